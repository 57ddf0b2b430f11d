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
// dz by distance into sums of its own in LDS (the lanes' distances differ, so no two lanes meet in one place and the order is fixed), dz beyond
// `far` into registers, and the workgroup adds up the runs of its buckets at the end; bias_table_kernel adds up workgroups.
// Distance d lies in plane d mod 8 of eight: lanes eight keys apart read neighbouring words.
//
// A row is held in registers between its two passes (its sums and its results), by one wave up to 2048 keys and by four up to
// 16384; longer ones are read twice.
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
    int plane;                           // words of a plane of distances
    int rows, blocks;                    // rows of a workgroup, workgroups of a head
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

__device__ __forceinline__ int bias_word(const BiasArgs &a, int index) { return (index & 7) * a.plane + (index >> 3); }

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}

// What a workgroup works on.
struct Rows {
    int ex, head, q0, q1;            // queries q0 .. q1 - 1
    int first, query_length, key_length;
    size_t base;                     // row number of query 0
};

__device__ __forceinline__ Rows bias_rows(const BiasArgs &a)
{
    Rows r;
    const unsigned lines = blockIdx.x / (unsigned)a.blocks;        // example and head
    r.ex = (int)(lines / (unsigned)a.heads);
    r.head = (int)(lines - (unsigned)r.ex * (unsigned)a.heads);
    r.q0 = (int)(blockIdx.x - lines * (unsigned)a.blocks) * a.rows;
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
    v = MAX ? wave_max(v) : wave_sum(v);
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

// NV > 0: a thread holds NV runs of eight keys, run j at 8 (thread + TPR j).  NV == 0: rows of any length, read twice.
template <bool BF16, int TPR, int NV>
__global__ void __launch_bounds__(256) bias_softmax_kernel(const BiasArgs a)
{
    typedef typename In<BF16>::type E;
    extern __shared__ float bias_lds[];
    __shared__ float red[4];
    const Rows r = bias_rows(a);
    for (int i = threadIdx.x; i <= a.low + a.far; i += 256)
        bias_lds[bias_word(a, i)] = a.table[(size_t)bias_bucket_of(a, i - a.low) * a.heads + r.head];
    __syncthreads();
    const float bias_far = bias_lds[bias_word(a, a.low + a.far)], bias_low = bias_lds[bias_word(a, 0)];
    const int t = threadIdx.x % TPR, wave_first = t & ~63;

    // the scores of a run of eight keys that starts at key k (the run of the wave's first lane at kw), as logits
    auto logits = [&](const Raw8<BF16> &raw, int k, int kw, int position, int end, float (&z)[8]) {
        raw.get(z);
        const int most = position - kw, least = most - 511;        // distances of the wave's runs
        if (least >= a.far || most <= -a.low) {
            const float b = least >= a.far ? bias_far : bias_low;
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = fmaf(z[i], a.scale, b);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = min(max(position - k - i, -a.low), a.far) + a.low;
                z[i] = fmaf(z[i], a.scale, bias_lds[bias_word(a, at)]);
            }
        }
        if (end - k < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = k + i < end ? z[i] : -INFINITY;
        }
    };

    for (int q = r.q0 + (int)(threadIdx.x / TPR); q < r.q1; q += 256 / TPR) {
        const int end = bias_end(a, r, q), position = r.first + q;
        const size_t row = (r.base + q) * a.row_stride;
        E *out = static_cast<E *>(a.out) + row;
        if constexpr (NV > 0) {
            Raw8<BF16> raw[NV];
            float z[NV][8];
#pragma unroll
            for (int j = 0; j < NV; ++j) raw[j].load(a.in, row + 8 * (t + TPR * j), end - 8 * (t + TPR * j));
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                logits(raw[j], 8 * (t + TPR * j), 8 * (wave_first + TPR * j), position, end, z[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, z[j][i]);
            }
            top = row_reduce<TPR, true>(top, red);
            top = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) { z[j][i] = exp_of(z[j][i] - top); sum += z[j][i]; }
            sum = row_reduce<TPR, false>(sum, red);
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = 8 * (t + TPR * j);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[j][i] *= inv;
                if (k < a.keys) store8(out + k, a.keys - k, z[j]);
            }
        } else {
            float top = -INFINITY, sum = 0.0f;
            for (int k = 8 * t; k < end; k += 8 * TPR) {
                Raw8<BF16> raw;
                float z[8];
                raw.load(a.in, row + k, end - k);
                logits(raw, k, k - 8 * (t - wave_first), position, end, z);
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
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            for (int k = 8 * t; k < a.keys; k += 8 * TPR) {
                Raw8<BF16> raw;
                float z[8];
                raw.load(a.in, row + k, end - k);
                logits(raw, k, k - 8 * (t - wave_first), position, end, z);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = exp_of(z[i] - base) * inv;
                store8(out + k, a.keys - k, z);
            }
        }
    }
}

template <bool BF16, int TPR, int NV>
__global__ void __launch_bounds__(256) bias_backward_kernel(const BiasArgs a)
{
    typedef typename In<BF16>::type E;
    extern __shared__ float bias_lds[];                            // a wave's sums by distance, four times
    __shared__ float red[4], ends[4][2];
    const Rows r = bias_rows(a);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < 4 * 8 * a.plane; i += 256) bias_lds[i] = 0.0f;
    __syncthreads();
    float *const mine = bias_lds + wave * 8 * a.plane;
    const int t = threadIdx.x % TPR, wave_first = t & ~63;
    float sum_far = 0.0f, sum_low = 0.0f;

    // zeros after the first `count` values (not 0 * dot: a broken row's sum may be NaN)
    auto cut = [&](float (&v)[8], int count) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? v[i] : 0.0f;
    };
    // dz of a run of eight keys into the sums; what does not count is zero there
    auto add = [&](const float (&dz)[8], int k, int kw, int position) {
        const int most = position - kw, least = most - 511;
        if (least >= a.far || most <= -a.low) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += dz[i];
            if (least >= a.far) sum_far += s;
            else sum_low += s;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = position - k - i;
                sum_far += d >= a.far ? dz[i] : 0.0f;
                sum_low += d <= -a.low ? dz[i] : 0.0f;
                if (d < a.far && d > -a.low) __hip_atomic_fetch_add(mine + bias_word(a, d + a.low), dz[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
            }
        }
    };

    for (int q = r.q0 + (int)(threadIdx.x / TPR); q < r.q1; q += 256 / TPR) {
        const int end = bias_end(a, r, q), position = r.first + q;
        const size_t row = (r.base + q) * a.row_stride;
        E *out = static_cast<E *>(a.out) + row;
        if constexpr (NV > 0) {
            Raw8<BF16> rp[NV], rd[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = 8 * (t + TPR * j);
                rp[j].load(a.in, row + k, end - k);
                rd[j].load(a.in2, row + k, end - k);
            }
            float dot = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float p[8], d[8];
                rp[j].get(p); rd[j].get(d);
#pragma unroll
                for (int i = 0; i < 8; ++i) dot = fmaf(p[i], d[i], dot);
            }
            dot = row_reduce<TPR, false>(dot, red);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = 8 * (t + TPR * j);
                float p[8], d[8];
                rp[j].get(p); rd[j].get(d);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= d[i] - dot;
                if (end - k < 8) cut(p, end - k);
                if (8 * (wave_first + TPR * j) < end) add(p, k, 8 * (wave_first + TPR * j), position);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= a.scale;
                if (k < a.keys) store8(out + k, a.keys - k, p);
            }
        } else {
            float dot = 0.0f;
            for (int k = 8 * t; k < end; k += 8 * TPR) {
                Raw8<BF16> rp, rd;
                float p[8], d[8];
                rp.load(a.in, row + k, end - k); rd.load(a.in2, row + k, end - k);
                rp.get(p); rd.get(d);
#pragma unroll
                for (int i = 0; i < 8; ++i) dot = fmaf(p[i], d[i], dot);
            }
            dot = row_reduce<TPR, false>(dot, red);
            for (int k = 8 * t; k < a.keys; k += 8 * TPR) {
                Raw8<BF16> rp, rd;
                float p[8], d[8];
                rp.load(a.in, row + k, end - k); rd.load(a.in2, row + k, end - k);
                rp.get(p); rd.get(d);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= d[i] - dot;
                if (end - k < 8) cut(p, end - k);
                if (k < end) add(p, k, k - 8 * (t - wave_first), position);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= a.scale;
                store8(out + k, a.keys - k, p);
            }
        }
    }

    // the workgroup's sums by bucket: a wave takes every fourth bucket, its lanes the distances of the run
    const float far_wave = wave_sum(sum_far), low_wave = wave_sum(sum_low);
    if (lane == 0) { ends[wave][0] = far_wave; ends[wave][1] = low_wave; }
    __syncthreads();
    float *part = a.partials + (size_t)blockIdx.x * a.buckets;
    const int side_buckets = a.bidirectional ? a.buckets / 2 : a.buckets;
    for (int b = wave; b < a.buckets; b += 4) {
        const bool after = b >= side_buckets;
        const int m = after ? b - side_buckets : b;
        int lo = m <= a.near ? m : a.borders[m - a.near - 1];      // magnitudes lo .. hi - 1
        const int next = m + 1, hi = m == side_buckets - 1 ? a.far : (next <= a.near ? next : a.borders[next - a.near - 1]);
        if (after || !a.bidirectional) lo = max(lo, 1);            // no distance of 0 on the side of later keys; 0 is in sum_low where there is one side
        float s = 0.0f;
        for (int d = lo + lane; d < hi; d += 64) {
            const int word = bias_word(a, (after ? -d : d) + a.low);
#pragma unroll
            for (int w = 0; w < 4; ++w) s += bias_lds[w * 8 * a.plane + word];
        }
        s = wave_sum(s);
        if (lane == 0) {
            if (m == side_buckets - 1) {
                const int which = after ? 1 : 0;
                s += ends[0][which] + ends[1][which] + ends[2][which] + ends[3][which];
            }
            if (!a.bidirectional && b == 0) s += ends[0][1] + ends[1][1] + ends[2][1] + ends[3][1];
            part[b] = s;
        }
    }
}

// Tables of an example from its workgroups' sums, in order, and their squared norm: one workgroup an example.
__global__ void __launch_bounds__(256) bias_table_kernel(const float *partials, int heads, int blocks, int buckets, float *g_table, size_t g_stride,
                                                         float *sqnorm)
{
    __shared__ float red[4];
    const float *p = partials + (size_t)blockIdx.x * heads * blocks * buckets;
    float *g = g_table + (size_t)blockIdx.x * g_stride;
    float ss = 0.0f;
    for (int e = threadIdx.x; e < heads * buckets; e += 256) {
        const int h = e / buckets, b = e - h * buckets;
        const float *line = p + (size_t)h * blocks * buckets + b;
        float s = 0.0f;
        for (int k = 0; k < blocks; ++k) s += line[(size_t)k * buckets];
        g[(size_t)b * heads + h] = s;
        ss += s * s;
    }
    ss = block_sum<4>(ss, red);
    if (threadIdx.x == 0 && sqnorm) sqnorm[blockIdx.x] = ss;
}

// Rows of a workgroup: several, so that what it does once (the biases, or the sums by bucket) is shared by them, as long as there
// are 2048 workgroups.
BiasArgs bias_args(const BiasGeo &g, int at_once)
{
    BiasArgs a = {};
    a.n = g.n; a.heads = g.heads; a.queries = g.queries; a.keys = g.keys; a.buckets = g.buckets; a.bidirectional = g.bidirectional;
    a.causal = g.causal; a.query_offset = g.query_offset; a.scale = g.scale; a.row_stride = g.row_stride;
    a.near = g.near; a.border_count = g.border_count; a.far = g.far; a.low = g.bidirectional ? g.far : 0;
    std::copy(g.borders, g.borders + BIAS_BORDERS, a.borders);
    a.plane = (a.low + a.far) / 8 + 1;
    const long long rows = (long long)g.n * g.heads * g.queries;
    const long long each = std::max(1ll, std::min(rows / (2048ll * at_once), 64ll / at_once));
    a.rows = (int)std::min((long long)at_once * each, (long long)(g.queries + at_once - 1) / at_once * at_once);
    a.blocks = (g.queries + a.rows - 1) / a.rows;
    return a;
}

int rows_at_once(const BiasGeo &g) { return g.keys <= 2048 ? 4 : 1; }

template <bool BF16>
dp_status run_forward(const BiasGeo &g, const BiasArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((size_t)g.n * g.heads * a.blocks));
    const unsigned lds = 8u * a.plane * 4u;
    if (g.keys <= 512) return launch_lds<bias_softmax_kernel<BF16, 64, 1>>(grid, 256, lds, s, a);
    if (g.keys <= 1024) return launch_lds<bias_softmax_kernel<BF16, 64, 2>>(grid, 256, lds, s, a);
    if (g.keys <= 2048) return launch_lds<bias_softmax_kernel<BF16, 64, 4>>(grid, 256, lds, s, a);
    if (g.keys <= 4096) return launch_lds<bias_softmax_kernel<BF16, 256, 2>>(grid, 256, lds, s, a);
    if (g.keys <= 8192) return launch_lds<bias_softmax_kernel<BF16, 256, 4>>(grid, 256, lds, s, a);
    if (g.keys <= 16384) return launch_lds<bias_softmax_kernel<BF16, 256, 8>>(grid, 256, lds, s, a);
    return launch_lds<bias_softmax_kernel<BF16, 256, 0>>(grid, 256, lds, s, a);
}

template <bool BF16>
dp_status run_backward(const BiasGeo &g, const BiasArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((size_t)g.n * g.heads * a.blocks));
    const unsigned lds = 4u * 8u * a.plane * 4u;
    if (g.keys <= 512) return launch_lds<bias_backward_kernel<BF16, 64, 1>>(grid, 256, lds, s, a);
    if (g.keys <= 1024) return launch_lds<bias_backward_kernel<BF16, 64, 2>>(grid, 256, lds, s, a);
    if (g.keys <= 2048) return launch_lds<bias_backward_kernel<BF16, 64, 4>>(grid, 256, lds, s, a);
    if (g.keys <= 4096) return launch_lds<bias_backward_kernel<BF16, 256, 2>>(grid, 256, lds, s, a);
    if (g.keys <= 8192) return launch_lds<bias_backward_kernel<BF16, 256, 4>>(grid, 256, lds, s, a);
    return launch_lds<bias_backward_kernel<BF16, 256, 0>>(grid, 256, lds, s, a);
}

}  // namespace

size_t bias_ws_bytes(const BiasGeo &g)
{
    const BiasArgs a = bias_args(g, rows_at_once(g));
    return ((size_t)g.n * g.heads * a.blocks * g.buckets * 4 + 15) & ~(size_t)15;
}

dp_status launch_bias_softmax(const BiasGeo &g, const void *scores, const float *table, const int32_t *query_lengths,
                              const int32_t *key_lengths, void *probs, hipStream_t s)
{
    BiasArgs a = bias_args(g, rows_at_once(g));
    a.in = scores; a.out = probs; a.table = table; a.query_lengths = query_lengths; a.key_lengths = key_lengths;
    return g.bf16 ? run_forward<true>(g, a, s) : run_forward<false>(g, a, s);
}

dp_status launch_bias_softmax_backward(const BiasGeo &g, const void *probs, const void *dprobs, const int32_t *query_lengths,
                                       const int32_t *key_lengths, void *dscores, float *g_table, size_t g_stride, float *sqnorm, void *ws,
                                       hipStream_t s)
{
    BiasArgs a = bias_args(g, rows_at_once(g));
    a.in = probs; a.in2 = dprobs; a.out = dscores; a.query_lengths = query_lengths; a.key_lengths = key_lengths;
    a.partials = static_cast<float *>(ws);
    const dp_status st = g.bf16 ? run_backward<true>(g, a, s) : run_backward<false>(g, a, s);
    if (st != DP_OK) return st;
    hipLaunchKernelGGL(bias_table_kernel, dim3((unsigned)g.n), dim3(256), 0, s, a.partials, g.heads, a.blocks, g.buckets, g_table, g_stride, sqnorm);
    return check_launch("bias_table");
}

}  // namespace dp
