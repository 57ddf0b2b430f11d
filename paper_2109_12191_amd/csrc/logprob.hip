// Log probabilities of tokens under rows of logits x, the rows' entropies and most likely tokens, and their gradient:
//     m = max x,  d_v = scale (x_v - m),  s = sum exp(d_v),  t = sum exp(d_v) d_v
//     logp_v = d_v - log s,   H = log s - t / s   (two terms that are not negative: nothing cancels)
//     dx_v = scale (a ([v is the target] - p_v) - b p_v (logp_v + H))
//
// Bound by memory: 4096 rows of 32768 bf16 logits 50 us, 5.4 TB/s, with their gradient in the same call 107, 5.0.
// One pass: a thread keeps (m, s, t) of what it has seen, brought to a new m when one comes; two such triples are joined the same way, over the lanes,
// the waves of a workgroup, and the workgroups of a row where there are too few rows to fill the chip.
// Alternatives: a thread's m is its largest logit, so the k-th largest of the threads' m is a bound that the k largest logits do not fall below, and only
// threads whose m reaches it can have one.  Their logits alone are looked at again (k of 256 threads' as a rule), those that reach the bound go
// into a list, and a logit's place is the number of list entries before it.  A list that overflows (thousands of equal logits) is replaced
// by k searches for the largest that is left.
// Gradient: where the statistics are not given, a row is held in registers between its sums and its results, so that memory sees it once.
#include "lanes.h"
#include "values.h"

#include <algorithm>
#include <cfloat>

namespace dp {

namespace {

struct LogprobArgs {
    const void *logits;
    void *dlogits;
    const int32_t *targets, *lengths;
    const float *stats, *entropy, *d_logprobs, *d_entropy;
    float *logprobs_out, *entropy_out, *stats_out, *top_logprobs;
    int32_t *top_tokens;
    float *partials;                 // of rows that several workgroups share: [rows, part_words]
    int n, tokens, vocab, top;
    float scale;
    size_t row_stride;
    int splits, split_runs;          // workgroups of a row, and runs of eight of each
    int rows;                        // rows of the call
    unsigned first_block;            // workgroups of the launches before
};

// Words of a row's partial results, whole 16 bytes: they are written and read by those.
__host__ __device__ constexpr size_t part_words(int splits, int top) { return ((size_t)splits * (4 + 2 * top) + 3) & ~(size_t)3; }

// e^x, x at most 0: the hardware's 2^x of a product rounded to 32 bits, off by a share |x| 2^-24 and an ulp or two.  In a row's sum, whose largest term is 1, that
// is |x| e^x 2^-24 of a term, less than half of 2^-24; a derivative p is off by the share |logp| 2^-24.  Splitting the product would cost two operations a logit.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// What has been seen of a row: the largest logit, and over all the sums of exp(scale (x - largest)) and of that times its exponent.  No logit above -inf: s is 0.
struct Seen {
    float m, s, t;
    __device__ __forceinline__ void none() { m = -FLT_MAX; s = t = 0.0f; }
    // to another m, not below.  (An exponent below -10^4 has an exponential of zero; the bound keeps 0 * inf out.)
    __device__ __forceinline__ void move(float to, float scale)
    {
        const float d = fmaxf((m - to) * scale, -1e4f), r = exp_of(d);
        t = r * fmaf(d, s, t);
        s *= r;
        m = to;
    }
};

// Seen by the lanes of a wave together, in each of them.
__device__ __forceinline__ void wave_join(Seen &v, float scale)
{
    v.move(wave_all_max(v.m), scale);
    v.s = wave_all_sum(v.s);
    v.t = wave_all_sum(v.t);
}

// By the TPR threads of a row; `red` holds 3 words for each wave.  More than a wave: every thread of the workgroup calls it, once between two barriers.
template <int TPR>
__device__ __forceinline__ void row_join(Seen &v, float scale, float *red)
{
    wave_join(v, scale);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) { red[3 * wave] = v.m; red[3 * wave + 1] = v.s; red[3 * wave + 2] = v.t; }
        __syncthreads();
        const int lane = (int)threadIdx.x & 63;
        v.none();
        if (lane < TPR / 64) v = {red[3 * lane], red[3 * lane + 1], red[3 * lane + 2]};
        wave_join(v, scale);
    }
}

// A row of logits as runs of eight from its first whole dword on: run q holds values 8 q - lead .. 8 q - lead + 7, where lead is 1 for a bf16 row that
// begins in the middle of a dword.  Runs are loaded whole; what a run holds before the row and after it is unspecified (zeros beyond its last dword).
template <bool BF16>
struct LogitRow {
    typedef typename In<BF16>::type E;
    __amdgpu_buffer_rsrc_t buffer;
    E *first;
    int lead, count;
    __device__ __forceinline__ LogitRow(const void *p, size_t at, int count_) : first(static_cast<E *>(const_cast<void *>(p)) + at), count(count_)
    {
        const unsigned long long address = reinterpret_cast<unsigned long long>(first);
        lead = BF16 ? (int)(address >> 1) & 1 : 0;
        buffer = __builtin_amdgcn_make_buffer_rsrc(first - lead, 0, (int)(((unsigned)(count + lead) * (unsigned)sizeof(E) + 3u) & ~3u), 0x00020000);
    }
    __device__ __forceinline__ int runs() const { return (count + lead + 7) >> 3; }
    __device__ __forceinline__ int index(int q) const { return 8 * q - lead; }
    __device__ __forceinline__ void load(Raw8<BF16> &raw, int q) const
    {
        typedef uint32_t words __attribute__((ext_vector_type(4)));
        const int at = q * 8 * (int)sizeof(E);
        const words v = __builtin_bit_cast(words, __builtin_amdgcn_raw_buffer_load_b128(buffer, at, 0, 0));
        if constexpr (BF16) {
            raw.w = make_uint4(v.x, v.y, v.z, v.w);
        } else {
            const words w = __builtin_bit_cast(words, __builtin_amdgcn_raw_buffer_load_b128(buffer, at + 16, 0, 0));
            raw.w[0] = __uint_as_float(v.x); raw.w[1] = __uint_as_float(v.y); raw.w[2] = __uint_as_float(v.z); raw.w[3] = __uint_as_float(v.w);
            raw.w[4] = __uint_as_float(w.x); raw.w[5] = __uint_as_float(w.y); raw.w[6] = __uint_as_float(w.z); raw.w[7] = __uint_as_float(w.w);
        }
    }
    // values v0 .. v0 + 7, those of the row; v0 is where a run of the row that they were made from begins
    __device__ __forceinline__ void store(int v0, const float (&v)[8]) const
    {
        if (v0 >= 0 && v0 + 8 <= count) {
            if (((v0 + lead) & 7) == 0) {
                typedef uint32_t words __attribute__((ext_vector_type(4)));
                const int at = (v0 + lead) * (int)sizeof(E);
                if constexpr (BF16) {
                    const words w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
                    __builtin_amdgcn_raw_buffer_store_b128(w, buffer, at, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const words w = {__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
                        __builtin_amdgcn_raw_buffer_store_b128(w, buffer, at + 16 * i, 0, 0);
                    }
                }
            } else {
                store8(first + v0, 8, v);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v0 + i >= 0 && v0 + i < count) {
                    if constexpr (BF16) first[v0 + i] = float_to_bf16_any(v[i]);
                    else first[v0 + i] = v[i];
                }
        }
    }
    __device__ __forceinline__ static uint16_t float_to_bf16_any(float f) { return (uint16_t)pack_bf16(f, 0.0f); }
};

// A run's values; those outside the row are -inf (EDGES; else there are none).
template <bool BF16, bool EDGES>
__device__ __forceinline__ void run_values(const Raw8<BF16> &raw, int v0, int count, float (&x)[8])
{
    raw.get(x);
    if constexpr (EDGES)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (unsigned)(v0 + i) < (unsigned)count ? x[i] : -INFINITY;
}

template <int U>
__device__ __forceinline__ void see(Seen &v, const float (&x)[U][8], float scale, bool entropy)
{
    float top = v.m;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, x[u][i]);
    v.move(top, scale);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = (x[u][i] - top) * scale, e = exp_of(d);
            v.s += e;
            if (entropy) v.t = fmaf(e, fmaxf(d, -1e4f), v.t);
        }
}

// Runs q0 + t, q0 + t + TPR .. below q1, of a row, by TPR threads.  `raw`: a thread's last four.
template <bool BF16, int TPR>
__device__ __forceinline__ void see_runs(Seen &v, const LogitRow<BF16> &row, int q0, int q1, int t, float scale, bool entropy, Raw8<BF16> (&raw)[4])
{
    constexpr int U = 4;
    for (int q = q0; q < q1; q += U * TPR) {
#pragma unroll
        for (int u = 0; u < U; ++u) row.load(raw[u], q + t + u * TPR);
        float x[U][8];
        if (row.index(q) >= 0 && row.index(q + U * TPR) <= row.count && q + U * TPR <= q1) {
#pragma unroll
            for (int u = 0; u < U; ++u) run_values<BF16, false>(raw[u], 0, 0, x[u]);
        } else {
            const int end = min(row.count, row.index(q1));
#pragma unroll
            for (int u = 0; u < U; ++u) run_values<BF16, true>(raw[u], row.index(q + t + u * TPR), end, x[u]);
        }
        see<U>(v, x, scale, entropy);
    }
}

// Results of a row from what all have seen of it, by one thread.
struct RowResult { float m, log_sum, h; };
__device__ __forceinline__ RowResult row_result(const Seen &v)
{
    const bool broken = !(v.m < INFINITY) || !(v.s < INFINITY);          // a NaN or +inf among the logits
    const float log_sum = broken ? NAN : v.s > 0.0f ? logf(v.s) : INFINITY;
    return {broken ? NAN : v.s > 0.0f ? v.m : 0.0f, log_sum, broken ? NAN : v.s > 0.0f ? log_sum - v.t / v.s : 0.0f};
}
template <bool BF16>
__device__ __forceinline__ float target_logprob(const LogprobArgs &a, const typename In<BF16>::type *row, size_t r, const RowResult &res)
{
    const int target = a.targets[r];
    if (target < 0 || target >= a.vocab) return 0.0f;
    return (In<BF16>::ld(row + target) - res.m) * a.scale - res.log_sum;
}
template <bool BF16>
__device__ __forceinline__ void write_row(const LogprobArgs &a, const typename In<BF16>::type *row, size_t r, const RowResult &res)
{
    if (a.logprobs_out) a.logprobs_out[r] = target_logprob<BF16>(a, row, r, res);
    if (a.entropy_out) a.entropy_out[r] = res.h;
    if (a.stats_out) *reinterpret_cast<float2 *>(a.stats_out + 2 * r) = make_float2(res.m, res.log_sum);
}
__device__ __forceinline__ bool row_there(const LogprobArgs &a, unsigned r)
{
    if (!a.lengths) return true;
    const unsigned ex = r / (unsigned)a.tokens;
    return (int)(r - ex * (unsigned)a.tokens) < a.lengths[ex];
}
__device__ __forceinline__ void write_absent(const LogprobArgs &a, size_t r)
{
    if (a.logprobs_out) a.logprobs_out[r] = 0.0f;
    if (a.entropy_out) a.entropy_out[r] = 0.0f;
    if (a.stats_out) *reinterpret_cast<float2 *>(a.stats_out + 2 * r) = make_float2(0.0f, 0.0f);
    for (int k = 0; k < a.top; ++k) {
        a.top_tokens[r * a.top + k] = -1;
        if (a.top_logprobs) a.top_logprobs[r * a.top + k] = 0.0f;
    }
}

// Whether logit x of token i comes before logit y of token j among the alternatives.
__device__ __forceinline__ bool before(float x, int i, float y, int j) { return x > y || (x == y && i < j); }

constexpr int TOP_LIST = 1024;
struct TopShared {
    float bound[4];
    float list[TOP_LIST];
    int list_token[TOP_LIST];
    int threads[256];
    int thread_count, list_count;
    float best[LOGPROB_TOP];
    int best_token[LOGPROB_TOP];
    float wave_best[4];
    int wave_token[4];
};

// The k-th largest of a wave's values (equal ones count one by one), in every lane.
__device__ __forceinline__ float wave_kth(float v, int k)
{
    const int lane = (int)threadIdx.x & 63;
    float m = wave_all_max(v);
    for (; k > 1; --k) {
        if (lane == __ffsll((long long)__ballot(v == m)) - 1) v = -INFINITY;
        m = wave_all_max(v);
    }
    return m;
}

// The `top` largest logits of runs q0 .. q1 - 1 of a row, in order, into best / best_token (-inf and -1 beyond the last one above -inf).  `most`: the
// largest logit of this thread's runs, q0 + thread + 256 j.  HELD: `raw` are those runs.  By a workgroup of 256; ends with a barrier.
// The bound: of the waves whose threads all have a run (or the first), each holds a share of `top` logits that reach its share-th largest, so `top` reach the
// lowest of these.
template <bool BF16, bool HELD>
__device__ __forceinline__ void find_top(TopShared &sh, const LogitRow<BF16> &row, int q0, int q1, float most, int top, const Raw8<BF16> (&raw)[4])
{
    const int t = threadIdx.x, end = min(row.count, row.index(q1));
    const int waves = min(max((q1 - q0) >> 6, 1), 4);
    if (t < 64 * waves) {
        const float kth = wave_kth(most, (top + waves - 1) / waves);
        if ((t & 63) == 0) sh.bound[t >> 6] = kth;
    }
    if (t == 0) { sh.thread_count = 0; sh.list_count = 0; }
    if (t < LOGPROB_TOP) { sh.best[t] = -INFINITY; sh.best_token[t] = -1; }
    __syncthreads();
    float bound = sh.bound[0];
    for (int w = 1; w < waves; ++w) bound = fminf(bound, sh.bound[w]);
    auto enter = [&](float x, int v) {
        const int at = atomicAdd(&sh.list_count, 1);
        if (at < TOP_LIST) { sh.list[at] = x; sh.list_token[at] = v; }
    };
    if constexpr (HELD) {
        if (most >= bound)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int v0 = row.index(q0 + t + 256 * u);
                float x[8];
                run_values<BF16, true>(raw[u], v0, end, x);
                unsigned hits = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) hits |= x[i] >= bound && x[i] > -INFINITY ? 1u << i : 0u;
                for (; hits; hits &= hits - 1) {
                    const int at = __ffs((int)hits) - 1;
                    float y = x[0];
#pragma unroll
                    for (int i = 1; i < 8; ++i) y = at == i ? x[i] : y;
                    enter(y, v0 + at);
                }
            }
    } else {
        if (most >= bound) sh.threads[atomicAdd(&sh.thread_count, 1)] = t;
        __syncthreads();
        const int each = (q1 - q0 + 255) / 256 * 8, all = sh.thread_count * each;
        for (int e = t; e < all; e += 256) {
            const int which = e / each, in = e - which * each;
            const int v = row.index(q0 + sh.threads[which] + 256 * (in >> 3)) + (in & 7);
            if (v < 0 || v >= end) continue;
            const float x = In<BF16>::ld(row.first + v);
            if (x >= bound && x > -INFINITY) enter(x, v);
        }
    }
    __syncthreads();
    const int count = sh.list_count;
    if (count <= TOP_LIST) {
        for (int c = t; c < count; c += 256) {
            const float x = sh.list[c];
            const int v = sh.list_token[c];
            int place = 0;
#pragma unroll 8
            for (int o = 0; o < count; ++o) place += before(sh.list[o], sh.list_token[o], x, v);
            if (place < top) { sh.best[place] = x; sh.best_token[place] = v; }
        }
    } else {
        float last = INFINITY;
        int last_token = -1;
        for (int k = 0; k < top; ++k) {
            float x = -INFINITY;
            int token = -1;
            for (int v = max(row.index(q0), 0) + t; v < end; v += 256) {
                const float y = In<BF16>::ld(row.first + v);
                if (before(last, last_token, y, v) && y > -INFINITY && (token < 0 || before(y, v, x, token))) { x = y; token = v; }
            }
#pragma unroll
            for (int off = 32; off; off >>= 1) {
                const float y = __shfl_xor(x, off, 64);
                const int v = __shfl_xor(token, off, 64);
                if (v >= 0 && (token < 0 || before(y, v, x, token))) { x = y; token = v; }
            }
            if ((t & 63) == 0) { sh.wave_best[t >> 6] = x; sh.wave_token[t >> 6] = token; }
            __syncthreads();
            x = -INFINITY;
            token = -1;
            for (int w = 0; w < 4; ++w) {
                const float y = sh.wave_best[w];
                const int v = sh.wave_token[w];
                if (v >= 0 && (token < 0 || before(y, v, x, token))) { x = y; token = v; }
            }
            __syncthreads();
            if (token < 0) break;
            if (t == 0) { sh.best[k] = x; sh.best_token[k] = token; }
            last = x;
            last_token = token;
        }
    }
    __syncthreads();
}

// The alternatives of a row, from its `top` largest logits.
__device__ __forceinline__ void write_top(const LogprobArgs &a, size_t r, int k, float x, int token, const RowResult &res)
{
    const bool broken = !(res.h == res.h);
    a.top_tokens[r * a.top + k] = broken ? -1 : token;
    if (a.top_logprobs) a.top_logprobs[r * a.top + k] = broken ? NAN : token < 0 ? -INFINITY : (x - res.m) * a.scale - res.log_sum;
}

// Rows of which a workgroup of 256 has one (TPR 256), or each of its waves (TPR 64).  TOP: with alternatives (TPR 256).
template <bool BF16, int TPR, bool TOP>
__global__ void __launch_bounds__(256) logprob_kernel(const LogprobArgs a)
{
    __shared__ float red[12];
    const int slot = TPR == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0, t = (int)threadIdx.x % TPR;
    const size_t r = (size_t)(a.first_block + blockIdx.x) * (256 / TPR) + slot;
    if (r >= (size_t)a.rows) return;
    if (!row_there(a, (unsigned)r)) {
        if (t == 0) write_absent(a, r);
        return;
    }
    const LogitRow<BF16> row(a.logits, r * a.row_stride, a.vocab);
    Seen v;
    v.none();
    Raw8<BF16> raw[4];
    see_runs<BF16, TPR>(v, row, 0, row.runs(), t, a.scale, a.entropy_out != nullptr, raw);
    const float most = v.m;
    row_join<TPR>(v, a.scale, red);
    const RowResult res = row_result(v);
    if (t == 0) write_row<BF16>(a, row.first, r, res);
    if constexpr (TOP) {
        __shared__ TopShared sh;
        find_top<BF16, false>(sh, row, 0, row.runs(), most, a.top, raw);
        if (t < a.top) write_top(a, r, t, sh.best[t], sh.best_token[t], res);
    }
}

// Rows with alternatives, short enough for a wave to hold one: the largest logit is looked for `top` times, and taken out.  A lane knows the largest
// of each of its runs, so a search is two reductions over the lanes and one run of eight (us, a workgroup a row and this, 8192 rows of 1000 logits with 8
// alternatives 42 and 17, with 32 96 and 43; of 4000 logits, with twice the registers, 43 and 41, 68 and 92).
template <bool BF16, int NV>
__global__ void __launch_bounds__(256) logprob_wave_top_kernel(const LogprobArgs a)
{
    const int slot = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const size_t r = (size_t)(a.first_block + blockIdx.x) * 4 + slot;
    if (r >= (size_t)a.rows) return;
    if (!row_there(a, (unsigned)r)) {
        if (lane == 0) write_absent(a, r);
        return;
    }
    const LogitRow<BF16> row(a.logits, r * a.row_stride, a.vocab);
    float x[NV][8], run_most[NV];
    int run_at[NV];
    auto most_of = [&](int j) {                          // of a run, the first of the largest
        run_most[j] = x[j][0];
        run_at[j] = 0;
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            const bool more = x[j][i] > run_most[j];
            run_most[j] = more ? x[j][i] : run_most[j];
            run_at[j] = more ? i : run_at[j];
        }
    };
    {
        Raw8<BF16> raw[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) row.load(raw[j], lane + 64 * j);
#pragma unroll
        for (int j = 0; j < NV; ++j) run_values<BF16, true>(raw[j], row.index(lane + 64 * j), row.count, x[j]);
    }
    Seen v;
    v.none();
    see<NV>(v, x, a.scale, a.entropy_out != nullptr);
    wave_join(v, a.scale);
    const RowResult res = row_result(v);
    if (lane == 0) write_row<BF16>(a, row.first, r, res);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = x[j][i] == x[j][i] ? x[j][i] : -INFINITY;          // (rows with a NaN have no alternatives)
        most_of(j);
    }
    float best = -INFINITY;
    int best_token = -1;
    for (int k = 0; k < a.top; ++k) {
        float most = run_most[0];
        int at = run_at[0], run = 0;
#pragma unroll
        for (int j = 1; j < NV; ++j) {
            const bool more = run_most[j] > most;
            most = more ? run_most[j] : most;
            at = more ? run_at[j] : at;
            run = more ? j : run;
        }
        const float all = wave_all_max(most);
        if (!(all > -INFINITY)) break;
        const int mine = row.index(lane + 64 * run) + at;
        const int token = (int)-wave_all_max(most == all ? -(float)mine : -INFINITY);          // (below 2^24: a float exactly)
        if (lane == k) { best = all; best_token = token; }
        const int place = token + row.lead, taken = place >> 9;                                 // 64 runs of eight
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (taken == j) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (lane == ((place >> 3) & 63) && (place & 7) == i) x[j][i] = -INFINITY;
                most_of(j);
            }
    }
    if (lane < a.top) write_top(a, r, lane, best, best_token, res);
}

// Rows that several workgroups share: each leaves what it has seen, and its largest logits.  A row's partial results: (m, s, t) of its workgroups, four
// words each, then their largest logits, second largest and so on, then those logits' tokens.  TOP: 0, no alternatives; 1; 2, at most four runs a thread.
template <bool BF16, int TOP>
__global__ void __launch_bounds__(256) logprob_split_kernel(const LogprobArgs a)
{
    __shared__ float red[12];
    const unsigned block = a.first_block + blockIdx.x, r = block / (unsigned)a.splits;
    const int split = (int)(block - r * (unsigned)a.splits);
    if (!row_there(a, r)) return;
    const LogitRow<BF16> row(a.logits, (size_t)r * a.row_stride, a.vocab);
    const int q0 = split * a.split_runs, q1 = min(q0 + a.split_runs, row.runs());
    Seen v;
    v.none();
    Raw8<BF16> raw[4];
    see_runs<BF16, 256>(v, row, q0, q1, (int)threadIdx.x, a.scale, a.entropy_out != nullptr, raw);
    const float most = v.m;
    row_join<256>(v, a.scale, red);
    float *part = a.partials + (size_t)r * part_words(a.splits, a.top);
    if (threadIdx.x == 0) *reinterpret_cast<float4 *>(part + 4 * split) = make_float4(v.m, v.s, v.t, 0.0f);
    if constexpr (TOP) {
        __shared__ TopShared sh;
        find_top<BF16, TOP == 2>(sh, row, q0, q1, most, a.top, raw);
        if ((int)threadIdx.x < a.top) {
            part += 4 * a.splits + (int)threadIdx.x * a.splits + split;
            part[0] = sh.best[threadIdx.x];
            part[a.top * a.splits] = __int_as_float(sh.best_token[threadIdx.x]);
        }
    }
}

// What the workgroups of a row have left, joined by a workgroup a row, from as many loads at once as there are.  Alternatives: the k-th largest of the
// workgroups' first entries, as many of each as make 3 k together, is a bound as in find_top.
constexpr int MOST_SPLITS = 64;
template <bool BF16, bool TOP>
__global__ void __launch_bounds__(256) logprob_join_kernel(const LogprobArgs a)
{
    const size_t r = a.first_block + blockIdx.x;
    const int t = threadIdx.x;
    if (!row_there(a, (unsigned)r)) {
        if (t == 0) write_absent(a, r);
        return;
    }
    const float *part = a.partials + r * part_words(a.splits, a.top);
    Seen v;
    v.none();
    const int lane = t & 63, all = a.top * a.splits;
    if (lane < a.splits) {
        const float4 p = *reinterpret_cast<const float4 *>(part + 4 * lane);
        v = {p.x, p.y, p.z};
    }
    constexpr int MOST = MOST_SPLITS * LOGPROB_TOP / 256;
    float x[MOST];
    int token[MOST];
    if constexpr (TOP)
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            const int e = t + 256 * i;
            x[i] = e < all ? part[4 * a.splits + e] : -INFINITY;
            token[i] = e < all ? __float_as_int(part[4 * a.splits + all + e]) : -1;
        }
    wave_join(v, a.scale);
    const RowResult res = row_result(v);
    if (t == 0) write_row<BF16>(a, static_cast<const typename In<BF16>::type *>(a.logits) + r * a.row_stride, r, res);
    if constexpr (TOP) {
        __shared__ float list[MOST_SPLITS * LOGPROB_TOP], bound;
        __shared__ int list_token[MOST_SPLITS * LOGPROB_TOP], count;
        const int some = min(a.top, (3 * a.top + a.splits - 1) / a.splits) * a.splits;      // at most 3 top + splits, below 256
        if (t == 0) count = 0;
        if (t < some) list[t] = x[0];
        __syncthreads();
        if (t < some) {
            int place = 0;
#pragma unroll 8
            for (int o = 0; o < some; ++o) place += before(list[o], o, x[0], t);
            if (place == a.top - 1) bound = fmaxf(x[0], -FLT_MAX);
        }
        __syncthreads();
        const float least = bound;
#pragma unroll
        for (int i = 0; i < MOST; ++i)
            if (x[i] >= least) {
                const int at = atomicAdd(&count, 1);
                list[at] = x[i];
                list_token[at] = token[i];
            }
        __syncthreads();
        const int entries = count;
        for (int e = t; e < entries; e += 256) {
            const float y = list[e];
            const int w = list_token[e];
            int place = 0;
#pragma unroll 8
            for (int o = 0; o < entries; ++o) place += before(list[o], list_token[o], y, w);
            if (place < a.top) write_top(a, r, place, y, w, res);
        }
        if (t >= entries && t < a.top) write_top(a, r, t, -INFINITY, -1, res);
    }
}

constexpr int NO_TARGET = -(1 << 30);

// What the gradient of a row is made of.
struct RowGradient {
    float m, log_sum, h, a, b, scale;
    int target;
    // derivatives of eight values from v0 on
    template <bool ENTROPY>
    __device__ __forceinline__ void of(int v0, float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float logp = (x[i] - m) * scale - log_sum, p = exp_of(logp);
            float g = -a * p;
            if constexpr (ENTROPY) g = fmaf(-b * p, fmaxf(logp, -1e4f) + h, g);
            x[i] = g;
        }
    }
};
// The row's own part: which derivatives come in (zeros of a row that is empty), and the target's logit, whose derivative is a (1 - p): with p near 1, what is left of
// 1 - p comes out of its logarithm.
__device__ __forceinline__ void gradient_inputs(const LogprobArgs &a, size_t r, RowGradient &g)
{
    g.target = a.targets ? a.targets[r] : -1;
    const bool scored = g.target >= 0 && g.target < a.vocab, empty = g.log_sum == INFINITY;
    if (!scored) g.target = NO_TARGET;
    g.a = scored && a.d_logprobs && !empty ? a.d_logprobs[r] : 0.0f;
    g.b = a.d_entropy && !empty ? a.d_entropy[r] : 0.0f;
    g.scale = a.scale;
}
template <bool BF16, bool ENTROPY>
__device__ __forceinline__ void write_gradient(const RowGradient &g, const LogitRow<BF16> &row, const Raw8<BF16> &raw, int q, const LogitRow<BF16> &out,
                                               float *logprob)
{
    const int v0 = row.index(q);
    float x[8];
    raw.get(x);
    const unsigned at = (unsigned)(g.target - v0);
    float own = 0.0f;
    if (at < 8u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) own = at == (unsigned)i ? x[i] : own;
        const float logp = (own - g.m) * g.scale - g.log_sum;
        if (logprob) *logprob = logp;
        own = -g.a * expm1f(logp);
        if constexpr (ENTROPY) own = fmaf(-g.b * exp_of(logp), fmaxf(logp, -1e4f) + g.h, own);
    }
    g.of<ENTROPY>(v0, x);
    if (at < 8u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = at == (unsigned)i ? own : x[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= g.scale;
    out.store(v0, x);
}
// Zeros into runs q0 + t .. of a row.
template <bool BF16, int TPR>
__device__ __forceinline__ void write_zeros(const LogitRow<BF16> &out, int q0, int q1, int t)
{
    const float zeros[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (int q = q0 + t; q < q1; q += TPR) out.store(out.index(q), zeros);
}

// Gradient from statistics.  TPR threads take up to 4 TPR runs of a row.
template <bool BF16, int TPR, bool ENTROPY>
__global__ void __launch_bounds__(256) logprob_gradient_kernel(const LogprobArgs a)
{
    const int slot = TPR == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0, t = (int)threadIdx.x % TPR;
    const size_t part = (size_t)(a.first_block + blockIdx.x) * (256 / TPR) + slot, r = part / (unsigned)a.splits;
    if (r >= (size_t)a.rows) return;
    const LogitRow<BF16> row(a.logits, r * a.row_stride, a.vocab), out(a.dlogits, r * a.row_stride, a.vocab);
    const int q0 = (int)(part - r * (unsigned)a.splits) * 4 * TPR;
    if (!row_there(a, (unsigned)r)) {
        write_zeros<BF16, TPR>(out, q0, min(q0 + 4 * TPR, out.runs()), t);
        if (q0 == 0 && t == 0 && a.logprobs_out) a.logprobs_out[r] = 0.0f;
        return;
    }
    Raw8<BF16> raw[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) row.load(raw[u], q0 + t + u * TPR);
    RowGradient g;
    const float2 st = *reinterpret_cast<const float2 *>(a.stats + 2 * r);
    g.m = st.x;
    g.log_sum = st.y;
    g.h = ENTROPY ? a.entropy[r] : 0.0f;
    gradient_inputs(a, r, g);
    float *logprob = a.logprobs_out ? a.logprobs_out + r : nullptr;
    if (logprob && g.target == NO_TARGET && q0 == 0 && t == 0) *logprob = 0.0f;
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (q0 + t + u * TPR < row.runs()) write_gradient<BF16, ENTROPY>(g, row, raw[u], q0 + t + u * TPR, out, logprob);
}

// Raw values that the compiler takes for new ones: what was made of them in one pass over the registers is made again in the next, and not kept.
__device__ __forceinline__ void renew(Raw8<true> &raw) { asm volatile("" : "+v"(raw.w.x), "+v"(raw.w.y), "+v"(raw.w.z), "+v"(raw.w.w)); }
__device__ __forceinline__ void renew(Raw8<false> &raw)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(raw.w[i]));
}

// Statistics and gradient in one pass: a row in the registers of TPR threads, NV runs each.
template <bool BF16, int TPR, int NV, bool ENTROPY>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) logprob_held_kernel(const LogprobArgs a)
{
    __shared__ float red[3 * 16];
    constexpr int SLOTS = TPR > 256 ? 1 : 256 / TPR;
    const int slot = TPR == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0, t = (int)threadIdx.x % TPR;
    const size_t r = (size_t)(a.first_block + blockIdx.x) * SLOTS + slot;
    if (r >= (size_t)a.rows) return;
    const LogitRow<BF16> row(a.logits, r * a.row_stride, a.vocab), out(a.dlogits, r * a.row_stride, a.vocab);
    if (!row_there(a, (unsigned)r)) {
        write_zeros<BF16, TPR>(out, 0, out.runs(), t);
        if (t == 0 && a.logprobs_out) a.logprobs_out[r] = 0.0f;
        return;
    }
    Raw8<BF16> raw[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) row.load(raw[j], t + j * TPR);
    RowGradient g;
    g.log_sum = 0.0f;
    gradient_inputs(a, r, g);
    Seen v;
    v.none();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j && row.index(j * TPR) >= row.count) break;     // (the same for all threads)
        float x[8];
        run_values<BF16, true>(raw[j], row.index(t + j * TPR), row.count, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v.m = fmaxf(v.m, x[i]);
        if (NV > 4) __builtin_amdgcn_sched_barrier(0);       // (several runs' values at once would take the registers that hold rows)
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j && row.index(j * TPR) >= row.count) break;
        float x[8];
        renew(raw[j]);
        run_values<BF16, true>(raw[j], row.index(t + j * TPR), row.count, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = (x[i] - v.m) * a.scale, e = exp_of(d);
            v.s += e;
            if constexpr (ENTROPY) v.t = fmaf(e, fmaxf(d, -1e4f), v.t);
        }
        if (NV > 4) __builtin_amdgcn_sched_barrier(0);
    }
    row_join<TPR>(v, a.scale, red);
    const RowResult res = row_result(v);
    g.m = res.m;
    g.log_sum = res.log_sum;
    g.h = res.h;
    if (g.log_sum == INFINITY) g.a = g.b = 0.0f;
    float *logprob = a.logprobs_out ? a.logprobs_out + r : nullptr;
    if (logprob && g.target == NO_TARGET && t == 0) *logprob = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        renew(raw[j]);
        if (t + j * TPR < row.runs()) write_gradient<BF16, ENTROPY>(g, row, raw[j], t + j * TPR, out, logprob);
        if (NV > 4) __builtin_amdgcn_sched_barrier(0);
    }
}

size_t round16(size_t b) { return (b + 15) & ~(size_t)15; }

// Workgroups that share a row: as many as make 1024 together, of 4096 logits or more each, where the launch that joins them pays (us, shared and not: 8 rows
// of 20000 logits 6.2 and 5.6, of 40000 6.1 and 7.2, with 4 alternatives 12.3 and 11.3, of 60000 12.2 and 14.8; 100 rows of 40000 9.4 and 8.6, 150 of
// 131072 15.5 and 23.4, 300 of 50000 14.6 and 13.2, of 131072 24.4 and 27.0).
int logprob_splits(const LogprobGeo &g)
{
    const long long rows = (long long)g.n * g.tokens;
    if (rows >= 512 || g.vocab < 32768 + 128 * rows) return 1;
    return (int)std::min<long long>({MOST_SPLITS, 1024 / rows, g.vocab / 4096});
}

LogprobArgs logprob_args(const LogprobGeo &g)
{
    LogprobArgs a = {};
    a.n = g.n; a.tokens = g.tokens; a.vocab = g.vocab; a.top = g.top; a.scale = g.scale; a.row_stride = g.row_stride;
    a.rows = g.n * g.tokens;
    a.splits = logprob_splits(g);
    a.split_runs = ((g.vocab + 1 + 7) / 8 + a.splits - 1) / a.splits;      // (with the place before a row that begins inside a dword)
    return a;
}

size_t partial_bytes(const LogprobGeo &g)
{
    const int splits = logprob_splits(g);
    return splits > 1 ? (size_t)g.n * g.tokens * part_words(splits, g.top) * 4 : 0;
}

// Whether the gradient without statistics holds its rows in registers: rows that fit (with the place before them where they may begin inside a dword),
// and enough of them (us, workgroups that share a row, then a pass over all, and held rows: 8 rows of 131000 bf16 logits 11 and 22, 64 of them 16 and 25,
// 100 26 and 28, 200 40 and 34).
bool holds_rows(const LogprobGeo &g) { return g.vocab <= (g.bf16 ? 131071 : 65536) && ((long long)g.n * g.tokens >= 128 || logprob_splits(g) == 1); }
// Places of a row's runs.
int held_places(const LogprobArgs &a, bool bf16)
{
    const bool inside = bf16 && ((reinterpret_cast<uintptr_t>(a.logits) & 2) || (a.rows > 1 && a.row_stride % 2));
    return a.vocab + (inside ? 1 : 0);
}

template <bool BF16>
dp_status run_logprobs(const LogprobArgs &a, hipStream_t s)
{
    const size_t rows = (size_t)a.rows;
    if (a.splits > 1) {
        const dp_status st = !a.top ? launch_blocks<logprob_split_kernel<BF16, 0>>(rows * a.splits, 256, 0, s, a)
                             : a.split_runs > 1024 ? launch_blocks<logprob_split_kernel<BF16, 1>>(rows * a.splits, 256, 0, s, a)
                                                   : launch_blocks<logprob_split_kernel<BF16, 2>>(rows * a.splits, 256, 0, s, a);
        if (st != DP_OK) return st;
        return a.top ? launch_blocks<logprob_join_kernel<BF16, true>>(rows, 256, 0, s, a) : launch_blocks<logprob_join_kernel<BF16, false>>(rows, 256, 0, s, a);
    }
    if (a.top) {
        const int places = held_places(a, BF16);
        if (places <= 512) return launch_blocks<logprob_wave_top_kernel<BF16, 1>>((rows + 3) / 4, 256, 0, s, a);
        if (places <= 1024) return launch_blocks<logprob_wave_top_kernel<BF16, 2>>((rows + 3) / 4, 256, 0, s, a);
        if (places <= 2048) return launch_blocks<logprob_wave_top_kernel<BF16, 4>>((rows + 3) / 4, 256, 0, s, a);
        return launch_blocks<logprob_kernel<BF16, 256, true>>(rows, 256, 0, s, a);
    }
    if (a.vocab <= 4096) return launch_blocks<logprob_kernel<BF16, 64, false>>((rows + 3) / 4, 256, 0, s, a);
    return launch_blocks<logprob_kernel<BF16, 256, false>>(rows, 256, 0, s, a);
}

template <bool BF16, bool ENTROPY>
dp_status run_gradient(LogprobArgs a, hipStream_t s)
{
    const size_t rows = (size_t)a.rows, runs = ((size_t)a.vocab + 8) / 8;
    if (a.vocab <= 2048) {
        a.splits = (int)((runs + 255) / 256);
        return launch_blocks<logprob_gradient_kernel<BF16, 64, ENTROPY>>((rows * a.splits + 3) / 4, 256, 0, s, a);
    }
    a.splits = (int)((runs + 1023) / 1024);
    return launch_blocks<logprob_gradient_kernel<BF16, 256, ENTROPY>>(rows * a.splits, 256, 0, s, a);
}

template <bool BF16, bool ENTROPY>
dp_status run_held(const LogprobArgs &a, hipStream_t s)
{
    const size_t rows = (size_t)a.rows;
    const int places = held_places(a, BF16);
    if (places <= 512) return launch_blocks<logprob_held_kernel<BF16, 64, 1, ENTROPY>>((rows + 3) / 4, 256, 0, s, a);
    if (places <= 1024) return launch_blocks<logprob_held_kernel<BF16, 64, 2, ENTROPY>>((rows + 3) / 4, 256, 0, s, a);
    if (places <= 2048) return launch_blocks<logprob_held_kernel<BF16, 64, 4, ENTROPY>>((rows + 3) / 4, 256, 0, s, a);
    if (places <= 4096) return launch_blocks<logprob_held_kernel<BF16, 256, 2, ENTROPY>>(rows, 256, 0, s, a);
    if (places <= 8192) return launch_blocks<logprob_held_kernel<BF16, 256, 4, ENTROPY>>(rows, 256, 0, s, a);
    if (places <= 16384) return launch_blocks<logprob_held_kernel<BF16, 256, 8, ENTROPY>>(rows, 256, 0, s, a);
    if (places <= 32768) return launch_blocks<logprob_held_kernel<BF16, 512, 8, ENTROPY>>(rows, 512, 0, s, a);
    if (!BF16 || places <= 65536) return launch_blocks<logprob_held_kernel<BF16, 1024, 8, ENTROPY>>(rows, 1024, 0, s, a);
    if constexpr (BF16) return launch_blocks<logprob_held_kernel<BF16, 1024, 16, ENTROPY>>(rows, 1024, 0, s, a);
}

}  // namespace

// Partial results of rows that are shared; statistics and entropies of a gradient that has to make them first.
size_t logprob_ws_bytes(const LogprobGeo &g)
{
    const size_t rows = (size_t)g.n * g.tokens;
    return partial_bytes(g) + (g.top || holds_rows(g) ? 0 : round16(rows * 8) + round16(rows * 4));
}

dp_status launch_logprobs(const LogprobGeo &g, const void *logits, const int32_t *targets, const int32_t *lengths, float *logprobs, float *entropy,
                          float *stats, float *top_logprobs, int32_t *top_tokens, void *ws, hipStream_t s)
{
    LogprobArgs a = logprob_args(g);
    a.logits = logits; a.targets = targets; a.lengths = lengths;
    a.logprobs_out = logprobs; a.entropy_out = entropy; a.stats_out = stats; a.top_logprobs = top_logprobs; a.top_tokens = top_tokens;
    a.partials = static_cast<float *>(ws);
    return g.bf16 ? run_logprobs<true>(a, s) : run_logprobs<false>(a, s);
}

dp_status launch_logprobs_backward(const LogprobGeo &g, const void *logits, const int32_t *targets, const int32_t *lengths, const float *stats,
                                   const float *entropy, const float *d_logprobs, const float *d_entropy, float *logprobs, void *dlogits, void *ws,
                                   hipStream_t s)
{
    LogprobArgs a = logprob_args(g);
    a.logits = logits; a.dlogits = dlogits; a.targets = targets; a.lengths = lengths; a.d_logprobs = d_logprobs; a.d_entropy = d_entropy;
    if (!stats && holds_rows(g)) {
        a.logprobs_out = logprobs;
        if (g.bf16) return d_entropy ? run_held<true, true>(a, s) : run_held<true, false>(a, s);
        return d_entropy ? run_held<false, true>(a, s) : run_held<false, false>(a, s);
    }
    if (!stats) {
        char *room = static_cast<char *>(ws) + partial_bytes(g);
        float *made = reinterpret_cast<float *>(room), *made_h = reinterpret_cast<float *>(room + round16((size_t)g.n * g.tokens * 8));
        const dp_status st = launch_logprobs(g, logits, targets, lengths, logprobs, d_entropy ? made_h : nullptr, made, nullptr, nullptr, ws, s);
        if (st != DP_OK) return st;
        logprobs = nullptr;
        stats = made;
        entropy = made_h;
    }
    a.stats = stats; a.entropy = entropy; a.logprobs_out = logprobs;
    if (g.bf16) return d_entropy ? run_gradient<true, true>(a, s) : run_gradient<true, false>(a, s);
    return d_entropy ? run_gradient<false, true>(a, s) : run_gradient<false, false>(a, s);
}

}  // namespace dp
