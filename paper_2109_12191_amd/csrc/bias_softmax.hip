// Softmax of attention scores under a learned relative position bias, and its backward pass with the per-example gradient of the bias
// table:
//     z[q, k] = scale S[q, k] + table[bucket(qpos - k), h],   P = softmax_k z over the keys that count,
//     dz = P (dP - sum_k P dP),   dS = scale dz,   g_i[b, h] = sum of dz over the places of bucket b,   |g_i|^2.
//
// The keys that count for a query are the first `end` of its row (key length, causal mask), so a row is read up to there only and
// what lies beyond, whatever it holds, is replaced by zeros; a row with no such key is all zeros.
//
// A bucket holds a run of distances, and from `far` on all distances of a side are in one bucket.  A workgroup takes rows of one
// example and head.  Forward, it makes the biases of the distances in between once, in LDS.  Backward, a wave adds its rows'
// dz by distance into sums of its own in LDS (no two lanes meet in one place between two fences, so that the order is fixed), dz beyond
// `far` into registers, and the workgroup adds up the runs of its buckets at the end; bias_table_kernel adds up workgroups.
// A lane holds runs of eight keys, so the distances of a run go down by one from word to word: slot d + low + 16 lies in plane (slot mod 8)
// of eight, at slot / 8, lanes eight keys apart meet neighbouring words of a plane, and where a run's eight values lie is one number for the
// lane and eight that all lanes share.  The slots before -low and after far, which a run that straddles the border reaches, hold what
// belongs to the border's bucket.
//
// A row is held in registers between its two passes (its sums and its results), by one wave up to 2048 keys, by four up to
// 16384 and by sixteen up to 32768 (backward: by four up to 8192); longer ones are read twice.  Bound by memory: 16 x 12 x 512 x 512 bf16
// forward 44 us, 4.6 TB/s, backward 61, 4.9 (and 4 to join the tables); 4 x 8 x 1500 x 1500 fp32 backward, causal and ragged, 104.  Four
// waves to a row of 1100 keys: 97 us, one wave 68.
#include "lanes.h"
#include "values.h"

#include <algorithm>

namespace dp {

namespace {

struct BiasArgs {
    const void *in, *in2;            // scores; probabilities and their gradient
    void *out;
    const float *table;
    const int32_t *query_lengths, *key_lengths;
    float *partials;                 // backward: [n, heads, blocks, buckets]
    int n, heads, queries, keys, buckets, bidirectional, causal, query_offset;
    float scale;
    size_t row_stride;
    int near, border_count, far, low;    // low: distances from -low down are one bucket (0 where there is one side)
    int plane, last;                     // words of a plane of distances; slots at `last - 1` and beyond in each are beyond `far`
    int rows, blocks;                    // rows of a workgroup, workgroups of a head
    int share;                           // lanes that share a bucket's sum
    unsigned first_block;                // workgroups of the launches before
    int borders[BIAS_BORDERS];
};

// e^x of a logit's distance to the largest.  (The difference comes first: folded into one multiply-add, a largest logit near the
// type's lowest value, a row that a mask added to the scores leaves empty, would overflow.)
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

__device__ __forceinline__ int bias_bucket_of(const BiasArgs &a, int d)
{
    int side = 0;
    if (a.bidirectional) { side = d < 0 ? a.buckets / 2 : 0; d = abs(d); }
    else d = max(d, 0);
    int b = min(d, a.near);
    for (int k = 0; k < a.border_count; ++k) b += d >= a.borders[k] ? 1 : 0;
    return side + b;
}

// Where the values of a run that starts at distance d lie: value i at word `lane` + `shared[i]`.
struct RunWords {
    int lane, shared[8];
    __device__ __forceinline__ static int slot(const BiasArgs &a, int d) { return (int)((unsigned)d + (unsigned)a.low + 16u); }
    // the part that all lanes share, from any lane's distance (they differ by multiples of eight)
    __device__ __forceinline__ void set_shared(const BiasArgs &a, int d)
    {
        const int m = slot(a, d) & 7;
#pragma unroll
        for (int i = 0; i < 8; ++i) shared[i] = ((m - i) & 7) * a.plane + ((m - i) >> 31);      // (one row earlier where i > m)
    }
};
__device__ __forceinline__ int bias_word(const BiasArgs &a, int slot) { return (slot & 7) * a.plane + (slot >> 3); }

// What a workgroup works on.
struct Rows {
    unsigned block;
    int ex, head, q0, q1;            // queries q0 .. q1 - 1
    int first, query_length, key_length;
    size_t base;                     // row number of query 0
    // Position of query q.  Keys are below 2^30 and far below 2^12, so that a position beyond both together is as good as any further one, and a slot
    // stays below 2^31.
    __device__ __forceinline__ int position(int q) const { return first > 0 ? first + min(q, (1 << 30) + 8192 - first) : first + q; }
};

__device__ __forceinline__ Rows bias_rows(const BiasArgs &a)
{
    Rows r;
    r.block = a.first_block + blockIdx.x;
    const unsigned lines = r.block / (unsigned)a.blocks;           // example and head
    r.ex = (int)(lines / (unsigned)a.heads);
    r.head = (int)(lines - (unsigned)r.ex * (unsigned)a.heads);
    r.q0 = (int)(r.block - lines * (unsigned)a.blocks) * a.rows;
    r.q1 = min(r.q0 + a.rows, a.queries);
    r.key_length = a.key_lengths ? min(max(a.key_lengths[r.ex], 0), a.keys) : a.keys;
    r.query_length = a.query_lengths ? min(max(a.query_lengths[r.ex], 0), a.queries) : a.queries;
    r.first = a.query_offset < 0 ? r.key_length - r.query_length : a.query_offset;
    r.base = (size_t)lines * a.queries;
    return r;
}

// keys that count for query q
__device__ __forceinline__ int bias_end(const BiasArgs &a, const Rows &r, int q)
{
    if (q >= r.query_length) return 0;
    return max(min(r.key_length, a.causal ? r.first + q + 1 : a.keys), 0);
}

// Sums / maxima over the TPR threads of a row.  `red`: a word for each wave; every thread of the workgroup calls it.
template <int TPR, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float *red)
{
    v = MAX ? wave_all_max(v) : wave_all_sum(v);
    if constexpr (TPR > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) v = MAX ? fmaxf(v, red[w]) : v + red[w];
    }
    return v;
}

// The rows of a tensor as runs of eight keys.  WORDS: fp32 rows, and bf16 rows that begin at whole dwords and have an even number of keys: a row is
// a buffer that ends where the keys that count do (or the row), and the 16-byte accesses of a run leave out, dword by dword, what lies
// beyond: no branch, and masked keys are not read but for the other half of a last dword.  Else value by value where a run is cut.
// What a cut run holds after its keys is unspecified.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <bool BF16, bool WORDS>
struct RowOf {
    typedef typename In<BF16>::type E;
    __amdgpu_buffer_rsrc_t buffer;
    E *first;
    int keys;
    __device__ __forceinline__ RowOf(void *p, size_t row, int count) : first(static_cast<E *>(p) + row), keys(count)
    {
        if constexpr (WORDS) buffer = __builtin_amdgcn_make_buffer_rsrc(first, 0, (int)(((unsigned)count * (unsigned)sizeof(E) + 3u) & ~3u), 0x00020000);
    }
    __device__ __forceinline__ void load(Raw8<BF16> &raw, int k) const
    {
        if constexpr (!WORDS) {
            raw.load(first, (size_t)k, keys - k);
        } else {
            const u32x4_t v = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer, k * (int)sizeof(E), 0, 0));
            if constexpr (BF16) {
                raw.w = make_uint4(v.x, v.y, v.z, v.w);
            } else {
                const u32x4_t w = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer, k * (int)sizeof(E) + 16, 0, 0));
                raw.w[0] = __uint_as_float(v.x); raw.w[1] = __uint_as_float(v.y); raw.w[2] = __uint_as_float(v.z); raw.w[3] = __uint_as_float(v.w);
                raw.w[4] = __uint_as_float(w.x); raw.w[5] = __uint_as_float(w.y); raw.w[6] = __uint_as_float(w.z); raw.w[7] = __uint_as_float(w.w);
            }
        }
    }
    __device__ __forceinline__ void store(int k, const float (&v)[8]) const
    {
        if constexpr (!WORDS) {
            if (k < keys) store8(first + k, keys - k, v);
        } else if constexpr (BF16) {
            const u32x4_t w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
            __builtin_amdgcn_raw_buffer_store_b128(w, buffer, k * (int)sizeof(E), 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4_t w = {__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
                __builtin_amdgcn_raw_buffer_store_b128(w, buffer, k * (int)sizeof(E) + 16 * i, 0, 0);
            }
        }
    }
};

// The sums of a workgroup's four waves, by distance in LDS and beyond the borders in registers, by bucket into its place of the workspace:
// `share` lanes to a bucket, over the distances of its run.
__device__ __forceinline__ void bias_bucket_sums(const BiasArgs &a, const Rows &r, const float *lds, float sum_far, float sum_low, float (&ends)[4][2])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float far_wave = wave_all_sum(sum_far), low_wave = wave_all_sum(sum_low);
    if (lane == 0) { ends[wave][0] = far_wave; ends[wave][1] = low_wave; }
    __syncthreads();
    float *part = a.partials + (size_t)r.block * a.buckets;
    const int side_buckets = a.bidirectional ? a.buckets / 2 : a.buckets;
    auto start = [&](int m) { return m <= a.near ? m : a.borders[m - a.near - 1]; };       // smallest magnitude of a side's bucket m
    for (int b = (int)threadIdx.x / a.share; b < a.buckets; b += 256 / a.share) {
        const bool after = b >= side_buckets;                      // keys after the query
        const int m = after ? b - side_buckets : b;
        const bool outer = m == side_buckets - 1, inner = !a.bidirectional && b == 0;
        // magnitudes lo .. hi; the outer bucket's and, with one side, bucket 0's run on into the slots beyond the border (runs reach 13 beyond)
        const int hi = outer ? a.far + 13 : start(m + 1) - 1, lo = inner ? -13 : after ? max(start(m), 1) : start(m);
        // of those, the ones that some place of these rows has (seven places more, where runs end)
        const int first = after ? max(lo, -(r.first + r.q1 - 1)) : max(lo, r.first + r.q0 - a.keys - 6);
        const int last = after ? min(hi, a.keys + 6 - r.first - r.q0) : min(hi, r.first + r.q1 - 1);
        float s = 0.0f;
        const int mine = (int)threadIdx.x & (a.share - 1);
#pragma unroll 2
        for (int d = first + mine; d <= last; d += a.share) {
            const int word = bias_word(a, RunWords::slot(a, after ? -d : d));
#pragma unroll
            for (int w = 0; w < 4; ++w) s += lds[w * 8 * a.plane + word];
        }
        for (int off = a.share >> 1; off; off >>= 1) s += __shfl_xor(s, off, 64);
        if (outer || inner) {
            const int which = after || inner ? 1 : 0;
            s += ends[0][which] + ends[1][which] + ends[2][which] + ends[3][which];
        }
        if (mine == 0) part[b] = s;
    }
}

// NV > 0: a thread holds NV runs of eight keys, run j at 8 (thread + TPR j), and the next row's are on their way while it works on one.
// NV == 0: rows of any length, read twice.
template <bool BF16, bool WORDS, int TPR, int NV>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) bias_softmax_kernel(const BiasArgs a)
{
    extern __shared__ float bias_lds[];
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    __shared__ float red[THREADS / 64];
    typedef RowOf<BF16, WORDS> Row;
    const Rows r = bias_rows(a);
    for (int i = threadIdx.x; i < 8 * a.plane; i += THREADS)
        bias_lds[bias_word(a, i)] = a.table[(size_t)bias_bucket_of(a, min(max(i - 16 - a.low, -a.low), a.far)) * a.heads + r.head];
    __syncthreads();
    const int t = threadIdx.x % TPR;
    const int wave_first = __builtin_amdgcn_readfirstlane(t & ~63), row_first = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    constexpr int STEP = THREADS / TPR;                             // rows that are worked on together

    // the scores of a run of eight keys from key k on, as logits; `whole`: the same for the wave, every run of it counts to its end
    RunWords at;
    auto logits = [&](const Raw8<BF16> &raw, int k, bool whole, int position, int end, float (&z)[8]) {
        raw.get(z);
        at.lane = min(max(RunWords::slot(a, position - k) >> 3, 1), a.last);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = fmaf(z[i], a.scale, bias_lds[at.lane + at.shared[i]]);
        if (!whole) {
            asm volatile("");                                      // (a branch: most runs are whole)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = k + i < end ? z[i] : -INFINITY;
        }
    };

    // zeros at the places of a run that do not count
    auto cut = [&](float (&z)[8], int k, int end) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = k + i < end ? z[i] : 0.0f;
    };

    if constexpr (NV > 0) {
        Raw8<BF16> raw[NV];
        auto load_row = [&](int q) {
            const Row row(const_cast<void *>(a.in), (r.base + q) * a.row_stride, bias_end(a, r, q));
#pragma unroll
            for (int j = 0; j < NV; ++j) row.load(raw[j], 8 * (t + TPR * j));
        };
        if (r.q0 + row_first < r.q1) load_row(r.q0 + row_first);
        for (int q = r.q0 + row_first; q < r.q1; q += STEP) {
            const int end = bias_end(a, r, q), position = r.position(q);
            at.set_shared(a, position);
            float z[NV][8];
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < NV; ++j) logits(raw[j], 8 * (t + TPR * j), 8 * (wave_first + TPR * j + 64) <= end, position, end, z[j]);
            if (q + STEP < r.q1) load_row(q + STEP);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, z[j][i]);
            top = row_reduce<TPR, true>(top, red);
            top = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) { z[j][i] = exp_of(z[j][i] - top); sum += z[j][i]; }
            sum = row_reduce<TPR, false>(sum, red);
            const float inv = sum == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum);     // good to a step
            const bool broken = !(sum < INFINITY);                  // a NaN or +inf among the keys that count; the others are zeros all the same
            const Row out(a.out, (r.base + q) * a.row_stride, a.keys);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[j][i] *= inv;
                if (broken) cut(z[j], 8 * (t + TPR * j), end);
                out.store(8 * (t + TPR * j), z[j]);
            }
        }
    } else {
        for (int q = r.q0; q < r.q1; ++q) {
            const int end = bias_end(a, r, q), position = r.position(q);
            const RowOf<BF16, false> row(const_cast<void *>(a.in), (r.base + q) * a.row_stride, end), out(a.out, (r.base + q) * a.row_stride, a.keys);
            at.set_shared(a, position);
            float top = -INFINITY, sum = 0.0f;
            for (int k = 8 * t; k < end; k += 8 * TPR) {
                Raw8<BF16> raw;
                float z[8];
                row.load(raw, k);
                logits(raw, k, false, position, end, z);
                float here = z[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) here = fmaxf(here, z[i]);
                const float now = fmaxf(top, here), base = now == -INFINITY ? 0.0f : now;
                sum *= exp_of(top - base);
                top = now;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += exp_of(z[i] - base);
            }
            const float best = row_reduce<TPR, true>(top, red), base = best == -INFINITY ? 0.0f : best;
            sum = row_reduce<TPR, false>(sum * exp_of(top - base), red);
            const float inv = sum == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum);
            const bool broken = !(sum < INFINITY);
            for (int k = 8 * t; k < a.keys; k += 8 * TPR) {
                Raw8<BF16> raw;
                float z[8];
                row.load(raw, k);
                logits(raw, k, false, position, end, z);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = exp_of(z[i] - base) * inv;
                if (broken) cut(z, k, end);
                out.store(k, z);
            }
        }
    }
}

template <bool BF16, bool WORDS, int TPR, int NV>
__global__ void __launch_bounds__(256) bias_backward_kernel(const BiasArgs a)
{
    extern __shared__ float bias_lds[];                            // a wave's sums by distance, four times
    __shared__ float red[4], ends[4][2];
    typedef RowOf<BF16, WORDS> Row;
    const Rows r = bias_rows(a);
    const int wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < 4 * 8 * a.plane; i += 256) bias_lds[i] = 0.0f;
    __syncthreads();
    float *const mine = bias_lds + wave * 8 * a.plane;
    const int t = threadIdx.x % TPR;
    const int wave_first = __builtin_amdgcn_readfirstlane(t & ~63), row_first = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    constexpr int STEP = 256 / TPR;
    float sum_far = 0.0f, sum_low = 0.0f;

    // zeros at the places of a run that do not count; `whole`: the same for the wave, there is none
    auto cut = [&](float (&v)[8], int k, bool whole, int end) {
        if (!whole) {
            asm volatile("");                                      // (a branch: most runs are whole)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < end ? v[i] : 0.0f;
        }
    };
    // dz of a run from key k on into the sums
    RunWords at;
    auto add = [&](const float (&dz)[8], int k, int position) {
        const int d = position - k;                                // .. d - 7
        if (d - 7 >= a.far || d <= -a.low) {
            float s = dz[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) s += dz[i];
            sum_far += d > 0 ? s : 0.0f;
            sum_low += d > 0 ? 0.0f : s;
        } else {
            at.lane = RunWords::slot(a, d) >> 3;
            float sum[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = mine[at.lane + at.shared[i]];
#pragma unroll
            for (int i = 0; i < 8; ++i) mine[at.lane + at.shared[i]] = sum[i] + dz[i];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the next row's lanes meet other lanes' words
        }
    };

    if constexpr (NV > 0) {
        Raw8<BF16> rp[NV], rd[NV];
        auto load_row = [&](int q) {
            const int end = bias_end(a, r, q);
            const size_t row = (r.base + q) * a.row_stride;
            const Row p(const_cast<void *>(a.in), row, end), d(const_cast<void *>(a.in2), row, end);
#pragma unroll
            for (int j = 0; j < NV; ++j) { p.load(rp[j], 8 * (t + TPR * j)); d.load(rd[j], 8 * (t + TPR * j)); }
        };
        if (r.q0 + row_first < r.q1) load_row(r.q0 + row_first);
        for (int q = r.q0 + row_first; q < r.q1; q += STEP) {
            const int end = bias_end(a, r, q), position = r.first + q;
            at.set_shared(a, position);
            auto none_of = [&](int j) { return NV > 1 && 8 * (wave_first + TPR * j) >= end; };        // the wave's run j has no key that counts (108.5 us and 105.5)
            float p[NV][8], d[NV][8];
            float dot = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = 8 * (t + TPR * j);
                const bool whole = 8 * (wave_first + TPR * j + 64) <= end;
                if (none_of(j)) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) p[j][i] = 0.0f;
                    continue;
                }
                rp[j].get(p[j]); rd[j].get(d[j]);
                cut(p[j], k, whole, end);
                cut(d[j], k, whole, end);
#pragma unroll
                for (int i = 0; i < 8; ++i) dot = fmaf(p[j][i], d[j][i], dot);
            }
            if (q + STEP < r.q1) load_row(q + STEP);
            dot = row_reduce<TPR, false>(dot, red);
            const bool broken = !(fabsf(dot) < INFINITY);          // its places that do not count are zeros all the same
            const Row out(a.out, (r.base + q) * a.row_stride, a.keys);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = 8 * (t + TPR * j);
                if (!none_of(j)) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) p[j][i] *= d[j][i] - dot;
                    cut(p[j], k, !broken, end);
                    add(p[j], k, position);
#pragma unroll
                    for (int i = 0; i < 8; ++i) p[j][i] *= a.scale;
                }
                out.store(k, p[j]);
            }
        }
    } else {
        for (int q = r.q0; q < r.q1; ++q) {
            const int end = bias_end(a, r, q), position = r.first + q;
            const size_t row = (r.base + q) * a.row_stride;
            const RowOf<BF16, false> rows_p(const_cast<void *>(a.in), row, end), rows_d(const_cast<void *>(a.in2), row, end), out(a.out, row, a.keys);
            at.set_shared(a, position);
            float dot = 0.0f;
            for (int k = 8 * t; k < end; k += 8 * TPR) {
                Raw8<BF16> rp, rd;
                float p[8], d[8];
                rows_p.load(rp, k); rows_d.load(rd, k);
                rp.get(p); rd.get(d);
#pragma unroll
                for (int i = 0; i < 8; ++i) dot = fmaf(p[i], d[i], dot);
            }
            dot = row_reduce<TPR, false>(dot, red);
            for (int k = 8 * t; k < a.keys; k += 8 * TPR) {
                Raw8<BF16> rp, rd;
                float p[8], d[8];
                rows_p.load(rp, k); rows_d.load(rd, k);
                rp.get(p); rd.get(d);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= d[i] - dot;
                cut(p, k, false, end);
                if (k < end) add(p, k, position);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= a.scale;
                out.store(k, p);
            }
        }
    }

    bias_bucket_sums(a, r, bias_lds, sum_far, sum_low, ends);
}

// ---- rows of at most 256 keys: TPR lanes of a wave to a row, 64 / TPR rows of a wave together, and eight rows of each of these in turn.  The
// rows of a wave lie eight apart, so that the words of their runs have the shared part in common (RunWords).

// A workgroup's rows of a tensor, each lane with a run of a row of its own.  WORDS (as RowOf): buffer accesses, left out by an offset beyond the
// buffer.  A run that a row ends in is loaded whole, with the next row's first values, and stored dword by dword.
template <bool BF16, bool WORDS>
struct NarrowRows {
    typedef typename In<BF16>::type E;
    __amdgpu_buffer_rsrc_t buffer;
    E *first;
    size_t stride;
    int keys;
    __device__ __forceinline__ NarrowRows(void *p, const BiasArgs &a, const Rows &r) : first(static_cast<E *>(p) + (r.base + r.q0) * a.row_stride), stride(a.row_stride), keys(a.keys)
    {
        if constexpr (WORDS) buffer = __builtin_amdgcn_make_buffer_rsrc(first, 0, (int)(((r.q1 - r.q0 - 1) * (unsigned)stride + (unsigned)keys) * (unsigned)sizeof(E)), 0x00020000);
    }
    // row q of the workgroup's, keys k .. k + 7, of which those before `end` count; cut runs hold anything after them
    __device__ __forceinline__ void load(Raw8<BF16> &raw, int q, int k, int end) const
    {
        if constexpr (!WORDS) {
            raw.load(first, (size_t)q * stride + k, end - k);
        } else {
            const unsigned at = ((unsigned)q * (unsigned)stride + (unsigned)k) * (unsigned)sizeof(E);
            const u32x4_t v = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer, k < end ? at : NOWHERE, 0, 0));
            if constexpr (BF16) {
                raw.w = make_uint4(v.x, v.y, v.z, v.w);
            } else {
                const u32x4_t w = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer, k + 4 < end ? at + 16 : NOWHERE, 0, 0));
                raw.w[0] = __uint_as_float(v.x); raw.w[1] = __uint_as_float(v.y); raw.w[2] = __uint_as_float(v.z); raw.w[3] = __uint_as_float(v.w);
                raw.w[4] = __uint_as_float(w.x); raw.w[5] = __uint_as_float(w.y); raw.w[6] = __uint_as_float(w.z); raw.w[7] = __uint_as_float(w.w);
            }
        }
    }
    __device__ __forceinline__ void store(bool there, int q, int k, const float (&v)[8]) const
    {
        if constexpr (!WORDS) {
            if (there && k < keys) store8(first + (size_t)q * stride + k, keys - k, v);
        } else {
            const unsigned at = ((unsigned)q * (unsigned)stride + (unsigned)k) * (unsigned)sizeof(E);
            constexpr int PER = BF16 ? 2 : 1, WORDS_OF_RUN = 8 / PER;      // values of a dword, dwords of a run
            uint32_t w[WORDS_OF_RUN];
#pragma unroll
            for (int i = 0; i < WORDS_OF_RUN; ++i) w[i] = BF16 ? pack_bf16(v[PER * i], v[PER * i + PER - 1]) : __float_as_uint(v[i]);
            const bool whole = k + 8 <= keys;
#pragma unroll
            for (int i = 0; i < WORDS_OF_RUN; i += 4)
                __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{w[i], w[i + 1], w[i + 2], w[i + 3]}, buffer, there && whole ? at + 4 * i : NOWHERE, 0, 0);
            if (keys & 7) {
#pragma unroll
                for (int i = 0; i < WORDS_OF_RUN; ++i)
                    __builtin_amdgcn_raw_buffer_store_b32(w[i], buffer, there && !whole && k + PER * i < keys ? at + 4 * i : NOWHERE, 0, 0);
            }
        }
    }
    static constexpr unsigned NOWHERE = 0xFFFFFFE0u;
};

template <bool BF16, bool WORDS, int TPR>
__global__ void __launch_bounds__(256) bias_softmax_narrow_kernel(const BiasArgs a)
{
    extern __shared__ float bias_lds[];
    const Rows r = bias_rows(a);
    for (int i = threadIdx.x; i < 8 * a.plane; i += 256)
        bias_lds[bias_word(a, i)] = a.table[(size_t)bias_bucket_of(a, min(max(i - 16 - a.low, -a.low), a.far)) * a.heads + r.head];
    __syncthreads();
    const int k = 8 * (threadIdx.x % TPR), row0 = 8 * (threadIdx.x / TPR);         // of the workgroup's rows: row0 .. row0 + 7
    const NarrowRows<BF16, WORDS> in(const_cast<void *>(a.in), a, r), out(a.out, a, r);
    auto end_of = [&](int row) { return r.q0 + row < r.q1 ? bias_end(a, r, r.q0 + row) : 0; };
    Raw8<BF16> raw;
    in.load(raw, row0, k, end_of(row0));
    RunWords at;
    for (int s = 0; s < 8; ++s) {
        const int row = row0 + s, end = end_of(row), position = r.position(r.q0 + row);
        at.set_shared(a, r.position(r.q0 + s));                    // (beyond the last position that is told apart, all words hold the same)
        at.lane = min(max(RunWords::slot(a, position - k) >> 3, 1), a.last);
        float z[8];
        raw.get(z);
        if (s < 7) in.load(raw, row + 1, k, end_of(row + 1));      // on its way during this row
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            z[i] = fmaf(z[i], a.scale, bias_lds[at.lane + at.shared[i]]);
            z[i] = k + i < end ? z[i] : -INFINITY;
            top = fmaxf(top, z[i]);
        }
        top = lanes_reduce<TPR, true>(top);
        top = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) { z[i] = exp_of(z[i] - top); sum += z[i]; }
        sum = lanes_reduce<TPR, false>(sum);
        const float inv = sum == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= inv;
        if (!(sum < INFINITY)) {                                   // a NaN or +inf among the keys that count; the others are zeros all the same
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = k + i < end ? z[i] : 0.0f;
        }
        out.store(r.q0 + row < r.q1, row, k, z);
    }
}

// Backward: a lane's runs of its eight rows meet fifteen distances, row s's key i that of s - i; their sums stay in registers and go into the wave's
// words once, rows eight apart (whose runs have distances in common) one after the other.
template <bool BF16, bool WORDS, int TPR>
__global__ void __launch_bounds__(256) bias_backward_narrow_kernel(const BiasArgs a)
{
    extern __shared__ float bias_lds[];
    __shared__ float ends[4][2];
    const Rows r = bias_rows(a);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < 4 * 8 * a.plane; i += 256) bias_lds[i] = 0.0f;
    __syncthreads();
    float *const mine = bias_lds + wave * 8 * a.plane;
    const int k = 8 * (threadIdx.x % TPR), row0 = 8 * (threadIdx.x / TPR);
    const NarrowRows<BF16, WORDS> probs(const_cast<void *>(a.in), a, r), dprobs(const_cast<void *>(a.in2), a, r), out(a.out, a, r);
    auto end_of = [&](int row) { return r.q0 + row < r.q1 ? bias_end(a, r, r.q0 + row) : 0; };
    Raw8<BF16> rp, rd;
    probs.load(rp, row0, k, end_of(row0));
    dprobs.load(rd, row0, k, end_of(row0));
    float line[15];
#pragma unroll
    for (int c = 0; c < 15; ++c) line[c] = 0.0f;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        const int row = row0 + s, end = end_of(row);
        float p[8], d[8];
        rp.get(p); rd.get(d);
        if (s < 7) { probs.load(rp, row + 1, k, end_of(row + 1)); dprobs.load(rd, row + 1, k, end_of(row + 1)); }
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = k + i < end ? p[i] : 0.0f;
            d[i] = k + i < end ? d[i] : 0.0f;
            dot = fmaf(p[i], d[i], dot);
        }
        dot = lanes_reduce<TPR, false>(dot);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = k + i < end ? p[i] * (d[i] - dot) : 0.0f;
            line[7 + s - i] += p[i];
            p[i] *= a.scale;
        }
        out.store(r.q0 + row < r.q1, row, k, p);
    }
    const int d0 = r.first + r.q0 + row0 - k;                      // line c has distance d0 + c - 7
    float sum_far = 0.0f, sum_low = 0.0f;
    const bool beyond = d0 - 7 >= a.far || d0 <= -a.low - 7;
    if (beyond) {
        float s = line[0];
#pragma unroll
        for (int c = 1; c < 15; ++c) s += line[c];
        (d0 > 0 ? sum_far : sum_low) = s;
    }
    const int top = RunWords::slot(a, d0) + 7, m = (RunWords::slot(a, r.first + r.q0) + 7) & 7;
#pragma unroll 1
    for (int g = 0; g < 64 / TPR; ++g) {
        // A row's neighbouring lanes are eight keys apart: slots 8 .. 14 of a lane are 0 .. 6 of the next one, and in either half no two lanes
        // of a group have one in common.
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (lane / TPR == g && !beyond) {
#pragma unroll
                for (int c = 8 * half; c < 8 * half + 8 - half; ++c) {             // slots top - c, which line 14 - c goes to
                    float *word = mine + (top >> 3) + ((m - c) & 7) * a.plane + ((m - c) >> 3);
                    *word += line[14 - c];
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // what follows meets words of other lanes
        }
    }
    bias_bucket_sums(a, r, bias_lds, sum_far, sum_low, ends);
}
// Tables of an example from its workgroups' sums, and their squared norm: one workgroup an example.  Several threads share an
// entry's sums where there are fewer entries than threads; their shares are added in order.
__global__ void __launch_bounds__(1024) bias_table_kernel(const float *partials, int heads, int blocks, int buckets, float *g_table, size_t g_stride,
                                                          float *sqnorm)
{
    __shared__ float red[16], share[1024];
    const int entries = heads * buckets, parts = max(1, 1024 / entries);
    const float *p = partials + (size_t)blockIdx.x * entries * blocks;
    float *g = g_table + (size_t)blockIdx.x * g_stride;
    float ss = 0.0f;
    for (int e0 = 0; e0 < entries; e0 += 1024) {
        const int width = min(entries - e0, 1024);
        const int part = (int)threadIdx.x / width, e = e0 + (int)threadIdx.x - part * width, h = e / buckets, b = e - h * buckets;
        float s = 0.0f;
        if (part < parts) {
            const float *line = p + (size_t)h * blocks * buckets + b;
#pragma unroll 4
            for (int k = part; k < blocks; k += parts) s += line[(size_t)k * buckets];
        }
        share[threadIdx.x] = s;
        __syncthreads();
        if (part == 0) {
            for (int k = 1; k < parts; ++k) s += share[threadIdx.x + k * width];
            g[(size_t)b * heads + h] = s;
            ss += s * s;
        }
        __syncthreads();
    }
    ss = block_sum<16>(ss, red);
    if (threadIdx.x == 0 && sqnorm) sqnorm[blockIdx.x] = ss;
}

// Lanes of a wave that share a row in the kernels for short ones, or 0 where a row has a wave of its own or several: a call with fewer than eight
// queries would leave most of those lanes idle, and a few thousand rows are all under way at once that way (us, a wave to a row and
// several with eight in turn: backward, 64 keys, 8192 rows 7.6 and 10.8, 16384 11.4 and 11.6, 32768 15.7 and 11.3; 128 keys, 65536 rows 25.6 and
// 14.5; forward, 64 keys, 8192 rows 6.5 and 7.2, 16384 8.8 and 7.5, 65536 20.9 and 9.2).
int narrow_lanes(const BiasGeo &g)
{
    if (g.keys > 256 || g.queries < 8 || (long long)g.n * g.heads * g.queries < 16384 || g.row_stride > ((size_t)1 << 20)) return 0;
    return g.keys <= 64 ? 8 : g.keys <= 128 ? 16 : 32;
}

BiasArgs bias_args(const BiasGeo &g, bool backward)
{
    BiasArgs a = {};
    a.n = g.n; a.heads = g.heads; a.queries = g.queries; a.keys = g.keys; a.buckets = g.buckets; a.bidirectional = g.bidirectional;
    a.causal = g.causal; a.query_offset = g.query_offset; a.scale = g.scale; a.row_stride = g.row_stride;
    a.near = g.near; a.border_count = g.border_count; a.far = g.far; a.low = g.bidirectional ? g.far : 0;
    std::copy(g.borders, g.borders + BIAS_BORDERS, a.borders);
    a.last = (a.low + a.far + 16 + 7) / 8 + 1;
    a.plane = a.last + 1;
    if (const int lanes = narrow_lanes(g)) {
        a.rows = 8 * 256 / lanes;
    } else {
        // several rows, so that what a workgroup does once (the biases, or the sums by bucket) is shared by them, as long as there are 2048
        // workgroups; backward of rows of one run a lane, which leave more to what is done once, 1024 (512 keys, 98304 rows: 67.4 us and 61.6; 300
        // keys, 9600 rows: 11.2 and 9.6; but 512 keys, 4096 rows: 6.8 and 8.2; fp32 rows of 1024 keys, 32768 of them: 67.2 and 71.7).
        const long long workgroups = backward && g.keys <= 512 ? 1024 : 2048;
        const int at_once = g.keys <= 2048 ? 4 : 1;
        const long long rows = (long long)g.n * g.heads * g.queries;
        const long long each = std::max(1ll, std::min(rows / (workgroups * at_once), 64ll / at_once));
        a.rows = (int)std::min((long long)at_once * each, (long long)(g.queries + at_once - 1) / at_once * at_once);
    }
    a.blocks = (g.queries + a.rows - 1) / a.rows;
    // Lanes that share a bucket's sum: few where runs are short, so that all buckets are summed at once; a step over a run's distances against
    // steps of the exchange between the lanes, both about a trip to LDS.
    int longest = 14;                                              // the outer bucket's: beyond the border, as far as runs reach
    for (int i = 0; i < a.border_count; ++i) longest = std::max(longest, a.borders[i] - (i ? a.borders[i - 1] : a.near));
    longest = std::min(longest, a.keys + a.rows + 12);
    int best = 0;
    for (int share = 1, exchange = 0; share <= 64; share *= 2, ++exchange) {
        const int steps = ((a.buckets * share + 255) / 256) * ((longest + share - 1) / share + exchange + 2);
        if (!best || steps < best) { best = steps; a.share = share; }
    }
    return a;
}

// Whether a bf16 tensor's rows can be read by whole dwords (fp32 ones always can).
bool bias_words(const BiasGeo &g, const void *p)
{
    return (reinterpret_cast<uintptr_t>(p) & 3) == 0 && g.keys % 2 == 0 && g.row_stride % 2 == 0;
}

template <bool BF16, bool WORDS>
dp_status run_forward(const BiasGeo &g, const BiasArgs &a, hipStream_t s)
{
    const size_t grid = (size_t)g.n * g.heads * a.blocks;
    const unsigned lds = 8u * a.plane * 4u;
    const int lanes = narrow_lanes(g);
    if (lanes == 8) return launch_blocks<bias_softmax_narrow_kernel<BF16, WORDS, 8>>(grid, 256, lds, s, a);
    if (lanes == 16) return launch_blocks<bias_softmax_narrow_kernel<BF16, WORDS, 16>>(grid, 256, lds, s, a);
    if (lanes == 32) return launch_blocks<bias_softmax_narrow_kernel<BF16, WORDS, 32>>(grid, 256, lds, s, a);
    if (g.keys <= 512) return launch_blocks<bias_softmax_kernel<BF16, WORDS, 64, 1>>(grid, 256, lds, s, a);
    if (g.keys <= 1024) return launch_blocks<bias_softmax_kernel<BF16, WORDS, 64, 2>>(grid, 256, lds, s, a);
    if (g.keys <= 2048) return launch_blocks<bias_softmax_kernel<BF16, WORDS, 64, 4>>(grid, 256, lds, s, a);
    if (g.keys <= 4096) return launch_blocks<bias_softmax_kernel<BF16, WORDS, 256, 2>>(grid, 256, lds, s, a);
    if (g.keys <= 8192) return launch_blocks<bias_softmax_kernel<BF16, WORDS, 256, 4>>(grid, 256, lds, s, a);
    if (g.keys <= 16384) return launch_blocks<bias_softmax_kernel<BF16, WORDS, 256, 8>>(grid, 256, lds, s, a);
    // sixteen waves a row (16 rows, four waves and two passes against these: 60000 keys 27.2 us and 15.0, 131072 54.0 and 27.4)
    if (g.keys <= 32768) return launch_blocks<bias_softmax_kernel<BF16, WORDS, 1024, 4>>(grid, 1024, lds, s, a);
    return launch_blocks<bias_softmax_kernel<BF16, WORDS, 1024, 0>>(grid, 1024, lds, s, a);
}

template <bool BF16, bool WORDS>
dp_status run_backward(const BiasGeo &g, const BiasArgs &a, hipStream_t s)
{
    const size_t grid = (size_t)g.n * g.heads * a.blocks;
    const unsigned lds = 4u * 8u * a.plane * 4u;
    const int lanes = narrow_lanes(g);
    if (lanes == 8) return launch_blocks<bias_backward_narrow_kernel<BF16, WORDS, 8>>(grid, 256, lds, s, a);
    if (lanes == 16) return launch_blocks<bias_backward_narrow_kernel<BF16, WORDS, 16>>(grid, 256, lds, s, a);
    if (lanes == 32) return launch_blocks<bias_backward_narrow_kernel<BF16, WORDS, 32>>(grid, 256, lds, s, a);
    if (g.keys <= 512) return launch_blocks<bias_backward_kernel<BF16, WORDS, 64, 1>>(grid, 256, lds, s, a);
    if (g.keys <= 1024) return launch_blocks<bias_backward_kernel<BF16, WORDS, 64, 2>>(grid, 256, lds, s, a);
    if (g.keys <= 2048) return launch_blocks<bias_backward_kernel<BF16, WORDS, 64, 4>>(grid, 256, lds, s, a);
    if (g.keys <= 4096) return launch_blocks<bias_backward_kernel<BF16, WORDS, 256, 2>>(grid, 256, lds, s, a);
    if (g.keys <= 8192) return launch_blocks<bias_backward_kernel<BF16, WORDS, 256, 4>>(grid, 256, lds, s, a);
    return launch_blocks<bias_backward_kernel<BF16, WORDS, 256, 0>>(grid, 256, lds, s, a);
}

}  // namespace

size_t bias_ws_bytes(const BiasGeo &g)
{
    const BiasArgs a = bias_args(g, true);
    return ((size_t)g.n * g.heads * a.blocks * g.buckets * 4 + 15) & ~(size_t)15;
}

dp_status launch_bias_softmax(const BiasGeo &g, const void *scores, const float *table, const int32_t *query_lengths,
                              const int32_t *key_lengths, void *probs, hipStream_t s)
{
    BiasArgs a = bias_args(g, false);
    a.in = scores; a.out = probs; a.table = table; a.query_lengths = query_lengths; a.key_lengths = key_lengths;
    if (!g.bf16) return run_forward<false, true>(g, a, s);
    return bias_words(g, scores) && bias_words(g, probs) ? run_forward<true, true>(g, a, s) : run_forward<true, false>(g, a, s);
}

dp_status launch_bias_softmax_backward(const BiasGeo &g, const void *probs, const void *dprobs, const int32_t *query_lengths,
                                       const int32_t *key_lengths, void *dscores, float *g_table, size_t g_stride, float *sqnorm, void *ws,
                                       hipStream_t s)
{
    BiasArgs a = bias_args(g, true);
    a.in = probs; a.in2 = dprobs; a.out = dscores; a.query_lengths = query_lengths; a.key_lengths = key_lengths;
    a.partials = static_cast<float *>(ws);
    const bool words = bias_words(g, probs) && bias_words(g, dprobs) && bias_words(g, dscores);
    const dp_status st = !g.bf16 ? run_backward<false, true>(g, a, s) : words ? run_backward<true, true>(g, a, s) : run_backward<true, false>(g, a, s);
    if (st != DP_OK) return st;
    hipLaunchKernelGGL(bias_table_kernel, dim3((unsigned)g.n), dim3(1024), 0, s, a.partials, g.heads, a.blocks, g.buckets, g_table, g_stride, sqnorm);
    return check_launch("bias_table");
}

}  // namespace dp
