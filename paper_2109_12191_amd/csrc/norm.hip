// Normalisation of tokens over their features, and its backward pass with the per-example gradients of scale and shift:
//     xhat = (x - mean) r,  r = 1 / sqrt(mean((x - mean)^2) + eps),  y = gamma xhat + beta          (RMS: the mean is taken as zero)
//     a = gamma dy,  dx = r (a - mean(a) - xhat mean(a xhat)),   g_w = sum_t dy xhat,  g_b = sum_t dy        (RMS: no mean(a))
//
// Bound by memory: 32768 tokens of 2048 bf16 features forward 52 us, 5.2 TB/s, backward 88, 4.8 (and 10 to join sums and add up squares).  A row's
// values are held in registers between its sums and its results, 8 to a lane and run, by as many lanes as have one, so that memory sees each value
// once.  The mean comes first; deviations from it are then summed with their squares, and what the mean's rounding left in their sum is taken out again
// (a mean of 1000 deviations costs no digits of the variance).  The backward pass works the statistics out again from x: two more sums of registers,
// nothing to keep from the forward pass.
// Gradients of scale and shift: a lane keeps its columns' sums over the workgroup's rows in registers, workgroups leave theirs in the workspace,
// and norm_join_kernel adds them up in order; where an example has one workgroup, it writes the results itself.
#include "lanes.h"
#include "token_rows.h"

#include <algorithm>

namespace dp {

namespace {

struct NormArgs {
    const void *x, *dy;
    void *out;
    const float *gamma, *beta;
    const int32_t *lengths;
    float *partials;                 // backward: [n, blocks, 2, padded features]
    int shift;                       // backward: gradients of the shift are wanted
    float *g_w, *g_b, *sqnorm;       // backward, where an example has one workgroup: its results (else `partials`)
    size_t g_stride;
    float *stats;                    // of rows too long for registers: [n * tokens, 4]
    int n, tokens, features, padded, rms;
    float eps, inv_features;
    size_t row_stride;
    int rows, blocks;                // rows of a workgroup; workgroups of an example (backward)
    unsigned first_block;            // workgroups of the launches before
};

// Of the `rows` rows from token `token` of example `ex` on, those that it has (none if below zero; a length may be any number).
__device__ __forceinline__ int rows_there(const NormArgs &a, unsigned ex, int token, int rows)
{
    return a.lengths ? min(max(a.lengths[ex], 0) - token, rows) : rows;
}

// Sums of N values over the TPR threads of a row, in each of them.  Rows of several waves: every thread of the workgroup calls it, and `red`
// has two places of 16 N words that are used in turn.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float *red, int &turn)
{
    if constexpr (TPR < 64) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_reduce<TPR, false>(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = wave_all_sum(v[i]);
    }
    if constexpr (TPR > 64) {
        float *here = red + turn * 16 * 4;
        turn ^= 1;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) here[wave * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = here[i];
#pragma unroll
            for (int w = 1; w < TPR / 64; ++w) v[i] += here[w * N + i];
        }
    }
}

// A thread's values of a row.  Runs beyond the row were loaded as zeros; in the run that the row ends in (there is one where its length is no multiple of
// eight, the same for all rows) the places after it become zeros.
template <bool BF16, int NV>
__device__ __forceinline__ void values(const Raw8<BF16> (&raw)[NV], int t, int step, int features, float (&v)[8 * NV])
{
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float w[8];
        raw[j].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[8 * j + i] = w[i];
    }
    if (features & 7) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int left = features - 8 * (t + step * j);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[8 * j + i] = i < left ? v[8 * j + i] : 0.0f;
        }
    }
}

// A thread's values of a row become less by `by`; zeros stay zeros beyond the row.
template <int TPR, int NV>
__device__ __forceinline__ void lower(const NormArgs &a, int t, float (&x)[8 * NV], float by)
{
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const float m = 8 * (t + TPR * j) < a.features ? by : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[8 * j + i] -= m;
    }
    if (a.features & 7) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int left = a.features - 8 * (t + TPR * j);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[8 * j + i] = i < left ? x[8 * j + i] : 0.0f;
        }
    }
}

// x becomes its deviations from the mean (but for the rounding of the mean, whose correction comes out of the next sums).
template <int TPR, int NV>
__device__ __forceinline__ void centre(const NormArgs &a, int t, float (&x)[8 * NV], float *red, int &turn)
{
    if (a.rms) return;
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) s[0] += x[i];
    row_sums<TPR, 1>(s, red, turn);
    lower<TPR, NV>(a, t, x, s[0] * a.inv_features);
}

// Whether what the mean's rounding left in the deviations, `off`, is much of them: a row of nearly one value, whose deviations are taken from their own
// mean once more (each time is good for 2^-18 of the value before).
constexpr int AGAIN = 3;
__device__ __forceinline__ bool once_more(float off, float mean_square) { return off * off > mean_square * 0x1p-8f; }

// 1 / sqrt(variance + eps), from deviations whose mean is `off`; NaN where their squares are no number below infinity.
__device__ __forceinline__ float inverse_size(float off, float mean_square, float eps)
{
    const float v = fmaf(-off, off, mean_square);
    return mean_square < INFINITY ? 1.0f / sqrtf((v < 0.0f ? 0.0f : v) + eps) : NAN;
}

// gamma or beta of eight columns from k on; `none` where there is no such tensor
__device__ __forceinline__ void columns8(const float *p, float none, int k, int features, float (&v)[8])
{
    if (p) {
        load8f(p + (k < features ? k : 0), features - k, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = none;
    }
}
template <int TPR, int NV>
__device__ __forceinline__ void columns(const float *p, float none, int t, int features, float (&v)[8 * NV])
{
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float w[8];
        columns8(p, none, 8 * (t + TPR * j), features, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[8 * j + i] = w[i];
    }
}

// Forward, rows of up to 8 TPR NV features; a workgroup's rows are consecutive ones of all examples.
template <bool BF16, bool WORDS, int TPR, int NV>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) norm_kernel(const NormArgs a)
{
    __shared__ float red[2 * 16 * 4];
    const int slots = TPR > 64 ? 1 : (int)blockDim.x / TPR;
    const int slot = TPR > 64 ? 0 : TPR == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / TPR) : (int)threadIdx.x / TPR;
    const int t = (int)threadIdx.x % TPR;
    const size_t first = (size_t)(a.first_block + blockIdx.x) * a.rows, all = (size_t)a.n * a.tokens;
    const int rows = (int)min((size_t)a.rows, all - first);
    const TokenRows<BF16, WORDS> in(a.x, first, rows, a.row_stride, a.features), out(a.out, first, rows, a.row_stride, a.features);
    auto is_there = [&](int row) {
        if (row >= rows) return false;
        if (!a.lengths) return true;
        const unsigned r = (unsigned)(first + row), ex = r / (unsigned)a.tokens;
        return (int)(r - ex * (unsigned)a.tokens) < a.lengths[ex];
    };
    float gamma[8 * NV], beta[8 * NV];
    columns<TPR, NV>(a.gamma, 1.0f, t, a.features, gamma);
    columns<TPR, NV>(a.beta, 0.0f, t, a.features, beta);
    Raw8<BF16> next[NV];
    bool there = is_there(slot);
#pragma unroll
    for (int j = 0; j < NV; ++j) in.load(next[j], there, slot, 8 * (t + TPR * j));
    int turn = 0;
    for (int row0 = 0; row0 < rows; row0 += slots) {
        const int row = row0 + slot;
        float x[8 * NV];
        values<BF16, NV>(next, t, TPR, a.features, x);
        const bool now = there;
        there = is_there(row + slots);
#pragma unroll
        for (int j = 0; j < NV; ++j) in.load(next[j], there, row + slots, 8 * (t + TPR * j));
        centre<TPR, NV>(a, t, x, red, turn);
        float s[2], off;
        for (int again = 0;; ++again) {
            s[0] = s[1] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8 * NV; ++i) { s[0] += x[i]; s[1] = fmaf(x[i], x[i], s[1]); }
            if (a.rms) s[0] = 0.0f;
            row_sums<TPR, 2>(s, red, turn);
            off = s[0] * a.inv_features;
            if (again == AGAIN || !once_more(off, s[1] * a.inv_features)) break;
            lower<TPR, NV>(a, t, x, off);
        }
        const float r = inverse_size(off, s[1] * a.inv_features, a.eps), shift = -off * r;
        if (row < rows) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = now ? fmaf(fmaf(x[8 * j + i], r, shift), gamma[8 * j + i], beta[8 * j + i]) : 0.0f;
                out.store(row, 8 * (t + TPR * j), y);
            }
        }
    }
}

// Backward, rows of up to 8 TPR NV features; a workgroup's rows are consecutive tokens of one example.
template <bool BF16, bool WORDS, int TPR, int NV>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) norm_backward_kernel(const NormArgs a)
{
    __shared__ float red[2 * 16 * 4];
    __shared__ float share[TPR > 64 ? 1 : 4 * 64 * 8];
    const int slots = TPR > 64 ? 1 : (int)blockDim.x / TPR;
    const int slot = TPR > 64 ? 0 : TPR == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / TPR) : (int)threadIdx.x / TPR;
    const int t = (int)threadIdx.x % TPR;
    const unsigned block = a.first_block + blockIdx.x, ex = block / (unsigned)a.blocks;
    const int token = (int)(block - ex * (unsigned)a.blocks) * a.rows, rows = min(a.rows, a.tokens - token);
    const int length = rows_there(a, ex, token, rows);
    const size_t first = (size_t)ex * a.tokens + token;
    const TokenRows<BF16, WORDS> in(a.x, first, rows, a.row_stride, a.features), in2(a.dy, first, rows, a.row_stride, a.features),
        out(a.out, first, rows, a.row_stride, a.features);
    // The scale of a thread's columns: in registers, or where those leave a compute unit room for one workgroup of eight waves only, in LDS (us, LDS and
    // registers: 300 x 20 tokens of 6000 features 74 and 88, 32 x 300 90 and 93; but in the kernel of four waves 64 x 200 of 4096 80.9 and 79.6).
    constexpr bool LDS = TPR == 512 && NV == 2;
    float gamma[LDS ? 1 : 8 * NV], sum_w[8 * NV], sum_b[8 * NV];
    __shared__ float4 scales[LDS ? NV * 2 : 1][LDS ? TPR : 1];
    if constexpr (LDS) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float v[8];
            columns8(a.gamma, 1.0f, 8 * (t + TPR * j), a.features, v);
            scales[2 * j][t] = make_float4(v[0], v[1], v[2], v[3]);
            scales[2 * j + 1][t] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
        columns<TPR, NV>(a.gamma, 1.0f, t, a.features, gamma);
    }
    auto scale_of = [&](int j, float (&v)[8]) {          // (a thread reads what it wrote)
        if constexpr (LDS) {
            const float4 lo = scales[2 * j][t], hi = scales[2 * j + 1][t];
            v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
            v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = gamma[8 * j + i];
        }
    };
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) sum_w[i] = sum_b[i] = 0.0f;
    Raw8<BF16> next[NV], next2[NV];
    auto fetch = [&](int row) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            in.load(next[j], row < length, row, 8 * (t + TPR * j));
            in2.load(next2[j], row < length, row, 8 * (t + TPR * j));
        }
    };
    fetch(slot);
    int turn = 0;
    for (int row0 = 0; row0 < rows; row0 += slots) {
        const int row = row0 + slot;
        if (TPR >= 64 ? row < length : row0 < length) {
            float x[8 * NV], d[8 * NV];
            values<BF16, NV>(next, t, TPR, a.features, x);
            values<BF16, NV>(next2, t, TPR, a.features, d);
            fetch(row + slots);
            centre<TPR, NV>(a, t, x, red, turn);
            float s[4], off;                             // of deviations, their squares, a, and a times deviations
            for (int again = 0;; ++again) {
                s[0] = s[1] = s[2] = s[3] = 0.0f;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    float scale[8];
                    scale_of(j, scale);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float dev = x[8 * j + i], g = d[8 * j + i] * scale[i];
                        s[0] += dev;
                        s[1] = fmaf(dev, dev, s[1]);
                        s[2] += g;
                        s[3] = fmaf(g, dev, s[3]);
                    }
                }
                if (a.rms) s[0] = s[2] = 0.0f;
                row_sums<TPR, 4>(s, red, turn);
                off = s[0] * a.inv_features;
                if (again == AGAIN || !once_more(off, s[1] * a.inv_features)) break;
                lower<TPR, NV>(a, t, x, off);
            }
            const float r = inverse_size(off, s[1] * a.inv_features, a.eps);
            const float level = s[2] * a.inv_features, along = r * (s[3] - off * s[2]) * a.inv_features;
            const float shift = -off * r, slope = -r * along, base = -r * level;
            const bool there = TPR >= 64 || row < length;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float g[8], scale[8];
                scale_of(j, scale);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xhat = fmaf(x[8 * j + i], r, shift), dy = d[8 * j + i];
                    sum_w[8 * j + i] = fmaf(dy, xhat, sum_w[8 * j + i]);          // (of a row that is not there: x, dy and xhat are zeros)
                    sum_b[8 * j + i] += dy;
                    g[i] = fmaf(dy * scale[i], r, fmaf(xhat, slope, base));
                    if (!there) g[i] = 0.0f;
                }
                if (a.out && row < rows) out.store(row, 8 * (t + TPR * j), g);
            }
        } else if (a.out && row < rows) {
            const float zeros[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < NV; ++j) out.store(row, 8 * (t + TPR * j), zeros);
        }
    }
    if (!a.partials && !a.g_w) return;
    float *part = a.partials + (size_t)block * 2 * a.padded, ss = 0.0f;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (which && !a.shift) break;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = which ? sum_b[8 * j + i] : sum_w[8 * j + i];
                if constexpr (TPR < 64)
#pragma unroll
                    for (int off = TPR; off < 64; off <<= 1) v[i] += __shfl_xor(v[i], off, 64);
            }
            const int k = 8 * (t + TPR * j);
            if constexpr (TPR <= 64) {                   // the waves' sums, in order
                const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
                __syncthreads();
                if (lane < TPR)
#pragma unroll
                    for (int i = 0; i < 8; ++i) share[(wave * 8 + i) * 64 + t] = v[i];
                __syncthreads();
                if (wave == 0 && lane < TPR) {
                    for (int w = 1; w < (int)blockDim.x / 64; ++w)
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] += share[(w * 8 + i) * 64 + t];
                }
                if (wave != 0 || lane >= TPR) continue;
            }
            if (a.g_w) {
                float *to = (which ? a.g_b : a.g_w) + (size_t)ex * a.g_stride + k;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (k + i < a.features) { to[i] = v[i]; ss = fmaf(v[i], v[i], ss); }
            } else if (k < a.padded) {
                float4 *to = reinterpret_cast<float4 *>(part + which * a.padded + k);
                to[0] = make_float4(v[0], v[1], v[2], v[3]);
                to[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
        }
    }
    if (!a.g_w || !a.sqnorm) return;
    if constexpr (TPR <= 64) {
        if ((threadIdx.x >> 6) != 0) return;
        ss = wave_all_sum(ss);
    } else {
        ss = block_sum<TPR / 64>(ss, red);
    }
    if (threadIdx.x == 0) a.sqnorm[ex] = ss;
}

// Rows too long for registers, a workgroup each, read three times.  Forward: all of it.  Backward: their statistics, and what dx needs.
template <bool BF16, bool BACKWARD>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormArgs a)
{
    __shared__ float red[2 * 16 * 4];
    const size_t row = a.first_block + blockIdx.x;
    const unsigned ex = (unsigned)row / (unsigned)a.tokens;
    const bool there = !a.lengths || (int)((unsigned)row - ex * (unsigned)a.tokens) < a.lengths[ex];
    typedef typename In<BF16>::type E;
    const E *x = static_cast<const E *>(a.x) + row * a.row_stride;
    const E *dy = BACKWARD ? static_cast<const E *>(a.dy) + row * a.row_stride : nullptr;
    E *out = static_cast<E *>(a.out) + row * a.row_stride;
    if (!there) {
        const float zeros[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (!BACKWARD)
            for (int k = 8 * (int)threadIdx.x; k < a.features; k += 8192) store8(out + k, a.features - k, zeros);
        return;
    }
    int turn = 0;
    float mean = 0.0f;
    if (!a.rms) {
        float s[1] = {0.0f};
        for (int k = 8 * (int)threadIdx.x; k < a.features; k += 8192) {
            Raw8<BF16> raw;
            raw.load(x, (size_t)k, a.features - k);
            float v[8];
            raw.get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += v[i];
        }
        row_sums<1024, 1>(s, red, turn);
        mean = s[0] * a.inv_features;
    }
    float s[4], off, taken = 0.0f;                   // taken: what the deviations have been lowered by
    for (int again = 0;; ++again) {
        s[0] = s[1] = s[2] = s[3] = 0.0f;
        for (int k = 8 * (int)threadIdx.x; k < a.features; k += 8192) {
            Raw8<BF16> raw;
            raw.load(x, (size_t)k, a.features - k);
            float v[8], g[8];
            raw.get(v);
            if constexpr (BACKWARD) {
                float gamma[8];
                raw.load(dy, (size_t)k, a.features - k);
                raw.get(g);
                columns8(a.gamma, 1.0f, k, a.features, gamma);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] *= gamma[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float dev = i < a.features - k ? v[i] - mean - taken : 0.0f;
                s[0] += dev;
                s[1] = fmaf(dev, dev, s[1]);
                if constexpr (BACKWARD) { s[2] += g[i]; s[3] = fmaf(g[i], dev, s[3]); }
            }
        }
        if (a.rms) s[0] = s[2] = 0.0f;
        row_sums<1024, 4>(s, red, turn);
        off = s[0] * a.inv_features;
        if (again == AGAIN || !once_more(off, s[1] * a.inv_features)) break;
        taken += off;
    }
    const float r = inverse_size(off, s[1] * a.inv_features, a.eps);
    if constexpr (BACKWARD) {
        // (the mean and its correction are kept apart: together they would be rounded to the mean's digits)
        if (threadIdx.x == 0) {
            *reinterpret_cast<float4 *>(a.stats + 4 * row) = make_float4(mean, taken + off, r, r * (s[3] - off * s[2]) * a.inv_features);
            a.stats[4 * (size_t)a.n * a.tokens + row] = s[2] * a.inv_features;
        }
        return;
    }
    for (int k = 8 * (int)threadIdx.x; k < a.features; k += 8192) {
        Raw8<BF16> raw;
        raw.load(x, (size_t)k, a.features - k);
        float v[8], gamma[8], beta[8];
        raw.get(v);
        columns8(a.gamma, 1.0f, k, a.features, gamma);
        columns8(a.beta, 0.0f, k, a.features, beta);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf((v[i] - mean - taken - off) * r, gamma[i], beta[i]);
        store8(out + k, a.features - k, v);
    }
}

// Their backward pass by columns: a thread has eight, a workgroup 2048 of consecutive tokens of one example.
template <bool BF16>
__global__ void __launch_bounds__(256) norm_columns_kernel(const NormArgs a)
{
    typedef typename In<BF16>::type E;
    const unsigned wide = (unsigned)(a.features + 2047) / 2048u, block = a.first_block + blockIdx.x, line = block / wide;
    const unsigned ex = line / (unsigned)a.blocks;
    const int token = (int)(line - ex * (unsigned)a.blocks) * a.rows, rows = min(a.rows, a.tokens - token);
    const int length = rows_there(a, ex, token, rows);
    const int k = (int)(block - line * wide) * 2048 + 8 * (int)threadIdx.x, count = a.features - k;
    if (count <= 0) return;
    float gamma[8], sum_w[8], sum_b[8];
    columns8(a.gamma, 1.0f, k, a.features, gamma);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum_w[i] = sum_b[i] = 0.0f;
    for (int t = 0; t < rows; ++t) {
        const size_t row = (size_t)ex * a.tokens + token + t, at = row * a.row_stride + (size_t)k;
        float out[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (t < length) {
            const float4 st = *reinterpret_cast<const float4 *>(a.stats + 4 * row);
            const float level = a.stats[4 * (size_t)a.n * a.tokens + row];
            Raw8<BF16> raw, raw2;
            raw.load(a.x, at, count);
            raw2.load(a.dy, at, count);
            float x[8], d[8];
            raw.get(x);
            raw2.get(d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xhat = (x[i] - st.x - st.y) * st.z;
                sum_w[i] = fmaf(d[i], xhat, sum_w[i]);
                sum_b[i] += d[i];
                out[i] = st.z * fmaf(-xhat, st.w, fmaf(d[i], gamma[i], -level));
            }
        }
        if (a.out) store8(static_cast<E *>(a.out) + at, count, out);
    }
    if (!a.partials) return;
    float4 *to = reinterpret_cast<float4 *>(a.partials + (size_t)line * 2 * a.padded + k);
    to[0] = make_float4(sum_w[0], sum_w[1], sum_w[2], sum_w[3]);
    to[1] = make_float4(sum_w[4], sum_w[5], sum_w[6], sum_w[7]);
    if (!a.shift) return;
    to += a.padded / 4;
    to[0] = make_float4(sum_b[0], sum_b[1], sum_b[2], sum_b[3]);
    to[1] = make_float4(sum_b[4], sum_b[5], sum_b[6], sum_b[7]);
}

// Gradients of an example from its workgroups' sums, and their squares.  A workgroup has 4 QUADS columns (WHOLE: all of an example's, and the squared norm is
// done); its THREADS / QUADS parts take ranges of the sums, which are added in order.  (A counter that tells a workgroup that it is an example's last, to
// spare the launch that adds up the squares, takes longer than the launch: 59 us for 2048 workgroups, its fences empty caches.)
struct NormJoinArgs {
    const float *partials;
    float *g_w, *g_b, *squares;      // squares: [n, groups]
    size_t g_stride;
    int blocks, features, padded, groups;
    unsigned first_block;
};
template <int THREADS, int QUADS, bool WHOLE>
__global__ void __launch_bounds__(THREADS) norm_join_kernel(const NormJoinArgs a)
{
    constexpr int PARTS = THREADS / QUADS;
    __shared__ float4 share[PARTS > 1 ? PARTS : 1][PARTS > 1 ? QUADS : 1];
    __shared__ float red[THREADS / 64];
    const unsigned block = a.first_block + blockIdx.x, ex = block / (unsigned)a.groups, group = block - ex * (unsigned)a.groups;
    const int part = (int)threadIdx.x / QUADS, column = (int)threadIdx.x % QUADS, quads = (a.g_b ? 2 : 1) * a.padded / 4;
    const float4 *from = reinterpret_cast<const float4 *>(a.partials + (size_t)ex * a.blocks * 2 * a.padded);
    const int each = (a.blocks + PARTS - 1) / PARTS, end = min((part + 1) * each, a.blocks);
    float ss = 0.0f;
    for (int q0 = QUADS * (int)group; q0 < (WHOLE ? quads : min(quads, QUADS * ((int)group + 1))); q0 += QUADS) {
        const int q = q0 + column;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (q < quads)
#pragma unroll 8
            for (int b = part * each; b < end; ++b) {
                const float4 v = from[(size_t)b * (a.padded / 2) + q];
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
        if constexpr (PARTS > 1) {
            if (WHOLE) __syncthreads();
            share[part][column] = s;
            __syncthreads();
        }
        if (part == 0 && q < quads) {
#pragma unroll
            for (int w = 1; w < PARTS; ++w) {
                const float4 v = share[w][column];
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
            const bool shift = q >= a.padded / 4;
            const int k = 4 * (shift ? q - a.padded / 4 : q);
            float *to = (shift ? a.g_b : a.g_w) + (size_t)ex * a.g_stride + k;
            const float v[4] = {s.x, s.y, s.z, s.w};
            if (k + 4 <= a.features) {
                to[0] = v[0]; to[1] = v[1]; to[2] = v[2]; to[3] = v[3];
#pragma unroll
                for (int i = 0; i < 4; ++i) ss = fmaf(v[i], v[i], ss);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (k + i < a.features) { to[i] = v[i]; ss = fmaf(v[i], v[i], ss); }
            }
        }
    }
    if (!a.squares) return;
    ss = block_sum<THREADS / 64>(ss, red);
    if (threadIdx.x == 0) a.squares[block] = ss;
}

constexpr int NORM_HELD = 16384;       // features that a workgroup of sixteen waves holds in registers
constexpr size_t JOIN_WHOLE = 16384;   // quads of sums that one workgroup adds up

// Threads that share a row: as many as have a run of eight, a wave for up to 1024 features (forward 2048), four for up to 4096 (forward 8192); then eight (forward sixteen).
int norm_lanes(int features, bool backward)
{
    if (features <= 64) return 8;
    if (features <= 128) return 16;
    if (features <= 256) return 32;
    if (features <= (backward ? 1024 : 2048)) return 64;
    return backward ? features <= 4096 ? 256 : 512 : features <= 8192 ? 256 : 1024;
}

// Forward, few rows of some length: four waves a row, which are done sooner (us, four waves and one: 8 rows of 768 features 3.4 and 3.7, 1024 rows 4.2 and 4.0;
// of 2048 features 8 rows 3.3 and 4.6, 4096 rows 9.4 and 10.5, 32768 rows 60 and 56).
bool norm_spread(const NormGeo &g, bool backward)
{
    const long long rows = (long long)g.n * g.tokens;
    return !backward && g.features > 512 && g.features <= 2048 && rows <= (g.features <= 1024 ? 512 : 4096);
}

NormArgs norm_args(const NormGeo &g, bool backward)
{
    NormArgs a = {};
    a.n = g.n; a.tokens = g.tokens; a.features = g.features; a.padded = (g.features + 7) & ~7; a.rms = g.rms;
    a.eps = g.eps; a.inv_features = 1.0f / (float)g.features; a.row_stride = g.row_stride;
    const long long all = (long long)g.n * g.tokens;
    const int lanes = norm_spread(g, backward) ? 256 : norm_lanes(g.features, backward), at_once = lanes > 64 ? 1 : 256 / lanes;
    if (!backward) {
        a.rows = (int)std::max(1ll, std::min(all / (2048ll * at_once), 64ll / at_once)) * at_once;
    } else {
        // as few sums as there may be, at two workgroups to a compute unit; five of the kernel that holds the least (us, 512 workgroups and 1024: 64 x 200
        // tokens of 4096 features 79 and 88, 32 x 500 of 768 23.6 and 27.4; but 16 x 2048 of 2048 98 and 96, 8 x 1000 of 2048 in fp32 53.7 and 51.1)
        const long long workgroups = g.features > 1024 && g.features <= 2048 && all * (g.bf16 ? 2 : 4) >= 32000 ? 1024 : 512;
        long long each = std::max(1ll, std::min((all + workgroups * at_once - 1) / (workgroups * at_once), 64ll));
        // at least a few rows where sums are wide or a few examples have them all, unless that leaves half the compute units idle (us: 3 x 511 tokens of
        // 5000 features in fp32, three rows 35.4, four 33.2; 2 x 300 of 8000 two 27.5, four 22.0; 1 x 2000 of 300 four 13.0, eight 11.6; but 32 x 64 of 768
        // four 10.4, eight 10.9)
        const long long least = g.features > 2048 ? 4 : g.n < 8 ? 2 : 1;
        if (all >= 128 * least * at_once) each = std::max(each, least);
        // Examples that one workgroup is soon done with have one, and need no launch to join its sums (us, joined and not: 1000 x 3 tokens of 100
        // features 12.0 and 4.6, 300 x 10 of 768 14.0 and 10.2, 150 x 5 of 768 9.3 and 7.2, 300 x 20 of 4096 in fp32 88.7 and 85.0; but 150 x 40 of 768
        // 15.1 and 16.8, 8 x 16 of 768 8.1 and 9.1, 300 x 60 of 2048 62 and 92; nothing was measured between 150 and 300 examples).
        const long long turns = (g.tokens + at_once - 1) / at_once;
        if (turns <= (g.n >= 256 ? 20 : 3)) each = turns;
        a.rows = (int)std::min(each * at_once, (long long)(g.tokens + at_once - 1) / at_once * at_once);
        a.blocks = (g.tokens + a.rows - 1) / a.rows;
    }
    if (backward && g.features > NORM_HELD) {
        a.rows = std::min(g.tokens, 32);
        a.blocks = (g.tokens + a.rows - 1) / a.rows;
    }
    return a;
}

template <bool BF16, bool WORDS>
dp_status run_forward(const NormGeo &g, const NormArgs &a, hipStream_t s)
{
    const size_t all = (size_t)g.n * g.tokens, grid = (all + a.rows - 1) / a.rows;
    if (g.features <= 64) return launch_blocks<norm_kernel<BF16, WORDS, 8, 1>>(grid, 256, 0, s, a);
    if (g.features <= 128) return launch_blocks<norm_kernel<BF16, WORDS, 16, 1>>(grid, 256, 0, s, a);
    if (g.features <= 256) return launch_blocks<norm_kernel<BF16, WORDS, 32, 1>>(grid, 256, 0, s, a);
    if (g.features <= 512) return launch_blocks<norm_kernel<BF16, WORDS, 64, 1>>(grid, 256, 0, s, a);
    if (norm_spread(g, false)) return launch_blocks<norm_kernel<BF16, WORDS, 256, 1>>(grid, 256, 0, s, a);
    if (g.features <= 1024) return launch_blocks<norm_kernel<BF16, WORDS, 64, 2>>(grid, 256, 0, s, a);
    if (g.features <= 2048) return launch_blocks<norm_kernel<BF16, WORDS, 64, 4>>(grid, 256, 0, s, a);
    if (g.features <= 4096) return launch_blocks<norm_kernel<BF16, WORDS, 256, 2>>(grid, 256, 0, s, a);
    if (g.features <= 8192) return launch_blocks<norm_kernel<BF16, WORDS, 256, 4>>(grid, 256, 0, s, a);
    return launch_blocks<norm_kernel<BF16, WORDS, 1024, 2>>(grid, 1024, 0, s, a);
}

template <bool BF16, bool WORDS>
dp_status run_backward(const NormGeo &g, const NormArgs &a, hipStream_t s)
{
    const size_t grid = (size_t)g.n * a.blocks;
    // waves of the kernels that have a row or several to a wave: none without a row
    const unsigned threads = (unsigned)std::min(256ll, ((long long)std::min(a.rows, g.tokens) * norm_lanes(g.features, true) + 63) / 64 * 64);
    if (g.features <= 64) return launch_blocks<norm_backward_kernel<BF16, WORDS, 8, 1>>(grid, threads, 0, s, a);
    if (g.features <= 128) return launch_blocks<norm_backward_kernel<BF16, WORDS, 16, 1>>(grid, threads, 0, s, a);
    if (g.features <= 256) return launch_blocks<norm_backward_kernel<BF16, WORDS, 32, 1>>(grid, threads, 0, s, a);
    if (g.features <= 512) return launch_blocks<norm_backward_kernel<BF16, WORDS, 64, 1>>(grid, threads, 0, s, a);
    if (g.features <= 1024) return launch_blocks<norm_backward_kernel<BF16, WORDS, 64, 2>>(grid, threads, 0, s, a);
    if (g.features <= 2048) return launch_blocks<norm_backward_kernel<BF16, WORDS, 256, 1>>(grid, 256, 0, s, a);
    if (g.features <= 4096) return launch_blocks<norm_backward_kernel<BF16, WORDS, 256, 2>>(grid, 256, 0, s, a);
    if (g.features <= 8192) return launch_blocks<norm_backward_kernel<BF16, WORDS, 512, 2>>(grid, 512, 0, s, a);
    return launch_blocks<norm_backward_kernel<BF16, WORDS, 512, 4>>(grid, 512, 0, s, a);
}

template <bool BF16, bool BACKWARD>
dp_status run_long(const NormGeo &g, const NormArgs &a, hipStream_t s)
{
    const size_t all = (size_t)g.n * g.tokens, wide = (size_t)(g.features + 2047) / 2048;
    const dp_status st = launch_blocks<norm_long_kernel<BF16, BACKWARD>>(all, 1024, 0, s, a);
    if (st != DP_OK || !BACKWARD) return st;
    return launch_blocks<norm_columns_kernel<BF16>>((size_t)g.n * a.blocks * wide, 256, 0, s, a);
}

size_t round16(size_t b) { return (b + 15) & ~(size_t)15; }

struct NormWs { size_t partials, squares, stats, total; int groups; };
// Workspace: the workgroups' sums, the squares of groups of columns, statistics of long rows.
NormWs norm_ws(const NormGeo &g, const NormArgs &a)
{
    NormWs w = {};
    const size_t all = (size_t)g.n * g.tokens;
    w.groups = (2 * a.padded / 4 + 31) / 32;
    w.partials = round16((size_t)g.n * a.blocks * 2 * a.padded * 4);
    w.squares = round16((size_t)g.n * w.groups * 4);
    w.stats = g.features > NORM_HELD ? round16(all * 20) : 0;
    w.total = w.partials + w.squares + w.stats;
    return w;
}

}  // namespace

size_t norm_ws_bytes(const NormGeo &g) { return norm_ws(g, norm_args(g, true)).total; }

dp_status launch_norm(const NormGeo &g, const void *x, const float *gamma, const float *beta, const int32_t *lengths, void *y, hipStream_t s)
{
    NormArgs a = norm_args(g, false);
    a.x = x; a.out = y; a.gamma = gamma; a.beta = beta; a.lengths = lengths;
    if (g.features > NORM_HELD) return g.bf16 ? run_long<true, false>(g, a, s) : run_long<false, false>(g, a, s);
    const size_t all = (size_t)g.n * g.tokens;
    const bool words = token_rows_by_words(x, g.bf16, g.row_stride, all, a.rows) && token_rows_by_words(y, g.bf16, g.row_stride, all, a.rows);
    if (!g.bf16) return words ? run_forward<false, true>(g, a, s) : run_forward<false, false>(g, a, s);
    return words ? run_forward<true, true>(g, a, s) : run_forward<true, false>(g, a, s);
}

dp_status launch_norm_backward(const NormGeo &g, const void *x, const float *gamma, const void *dy, const int32_t *lengths, void *dx, float *g_w,
                               float *g_b, size_t g_stride, float *sqnorm, void *ws, hipStream_t s)
{
    NormArgs a = norm_args(g, true);
    const NormWs w = norm_ws(g, a);
    char *room = static_cast<char *>(ws);
    a.x = x; a.dy = dy; a.out = dx; a.gamma = gamma; a.lengths = lengths;
    a.partials = g_w ? reinterpret_cast<float *>(room) : nullptr;
    a.shift = g_b != nullptr;
    a.stats = reinterpret_cast<float *>(room + w.partials + w.squares);
    const bool direct = g_w && a.blocks == 1 && g.features <= NORM_HELD;
    if (direct) { a.partials = nullptr; a.g_w = g_w; a.g_b = g_b; a.g_stride = g_stride; a.sqnorm = sqnorm; }
    dp_status st;
    if (g.features > NORM_HELD) {
        st = g.bf16 ? run_long<true, true>(g, a, s) : run_long<false, true>(g, a, s);
    } else {
        bool words = true;
        for (const void *p : {x, dy, static_cast<const void *>(dx)}) words = words && token_rows_by_words(p, g.bf16, g.row_stride, (size_t)g.n * g.tokens, a.rows);
        if (!g.bf16) st = words ? run_backward<false, true>(g, a, s) : run_backward<false, false>(g, a, s);
        else st = words ? run_backward<true, true>(g, a, s) : run_backward<true, false>(g, a, s);
    }
    if (st != DP_OK || !g_w || direct) return st;
    NormJoinArgs j = {};
    j.partials = a.partials; j.g_w = g_w; j.g_b = g_b; j.g_stride = g_stride; j.blocks = a.blocks; j.features = g.features; j.padded = a.padded;
    // one workgroup an example where it has little to add up, or where there are as many as compute units
    const int quads = (g_b ? 2 : 1) * a.padded / 4;
    if (g.n >= 256 || (size_t)a.blocks * quads <= JOIN_WHOLE) {
        j.groups = 1;
        j.squares = sqnorm;
        if (quads <= 128) return launch_blocks<norm_join_kernel<1024, 128, true>>((size_t)g.n, 1024, 0, s, j);
        return launch_blocks<norm_join_kernel<1024, 512, true>>((size_t)g.n, 1024, 0, s, j);
    }
    // few groups: of fewer columns, and more parts (1 x 4000 tokens of 2048 features 40 and 27 us)
    const bool narrow = (size_t)g.n * ((quads + 63) / 64) <= 64;
    j.groups = narrow ? (quads + 31) / 32 : (quads + 63) / 64;
    j.squares = sqnorm ? reinterpret_cast<float *>(room + w.partials) : nullptr;
    const size_t grid = (size_t)g.n * j.groups;
    if (narrow) st = launch_blocks<norm_join_kernel<1024, 32, false>>(grid, 1024, 0, s, j);
    else if (grid <= 512) st = launch_blocks<norm_join_kernel<1024, 64, false>>(grid, 1024, 0, s, j);
    else st = launch_blocks<norm_join_kernel<256, 64, false>>(grid, 256, 0, s, j);
    if (st != DP_OK || !sqnorm) return st;
    return launch_sum_partials(j.squares, g.n, j.groups, sqnorm, s);
}

}  // namespace dp
