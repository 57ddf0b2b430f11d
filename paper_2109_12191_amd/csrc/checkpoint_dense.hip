// Dense layers whose input activations are kept in 8 bits (checkpoint.h): per-example gradients and their squared norms, and the
// clipped sum, straight from the checkpoint:
//     dW_i[o, k] = sum_{t < len_i} dY_i[t, o] X_i[t, k],   db_i[o] = sum_{t < len_i} dY_i[t, o],   acc += sum_i f_i dW_i.
//
// A code times its power-of-two scale is a bf16 number, so the products are those of bf16 matrix instructions with fp32 sums, and no
// rounding is added to the checkpoint's own.  (The 8-bit matrix instructions, which take such codes and scales as they lie, align the
// products of an instruction to the largest one and drop what lies 2^-13 or so below it: 3e-5 of the sum of the magnitudes on random
// codes, where bf16 instructions gave 3e-8.  They are not used.)  fp32 values of dY are split into three bf16 numbers that add up to
// them exactly (8 + 8 + 8 significant bits), three products for one.
//
//   ck_gram_kernel     norms alone of short examples:  |dW_i|^2 = sum_{t, u} (X_t . X_u) (dY_t . dY_u)
//   ck_contract_kernel everything else
#include "checkpoint.h"

#include <algorithm>

namespace dp {

namespace {

struct CkDenseArgs {
    const uint8_t *codes, *scales;
    const void *dy;
    const int32_t *lengths;          // [n] or nullptr: every example has `tokens` of them
    float *out_w, *out_b;            // stored: example 0's; weighted: the accumulators, or the ranges' partial sums
    size_t stride_w, stride_b;       // from one example (weighted: one range) to the next
    float *partials;                 // per-example calls: [n, per_example]
    const float *group_sqnorm;
    float clip_c;
    int n, tokens, cin, cout, pitch;
    int dy_bf16, has_bias, stored, add;
    int tiles_k, tiles_o, columns;   // tiles along k, along o; tiles_k + 1 columns of tiles with a bias
    int per_range;                   // weighted: chunks of a range
    int chunks;                      // weighted: chunks in all (of examples, or of rows)
};

__device__ __forceinline__ int ck_length(const CkDenseArgs &a, int i)
{
    return a.lengths ? min(max(a.lengths[i], 0), a.tokens) : a.tokens;
}

// v = first + second + third, each a bf16 number: a difference of an fp32 number and the bf16 number nearest to it is exact, and what is
// left after two of them has at most eight bits.
__device__ __forceinline__ void split8(const float (&v)[8], uint4 (&planes)[3])
{
    uint32_t w[3][4];
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = v[i];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[q][i] = pack_bf16(rest[2 * i], rest[2 * i + 1]);
            rest[2 * i] -= __uint_as_float(w[q][i] << 16);
            rest[2 * i + 1] -= __uint_as_float(w[q][i] & 0xFFFF0000u);
        }
        planes[q] = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
    }
}

// ------------------------------------------------------------------------------------------
// Contraction over tokens.  A workgroup of four waves owns a 128 (o) x 128 (k) tile, a wave 64 x 64 of it (2 x 2 blocks of 32 x 32).
// A chunk is 32 tokens; both operands lie in LDS as they lie in memory, [token][feature], and the matrix operands, which want
// consecutive tokens of a feature, are read with the transposing LDS loads (four tokens of 16 features each).  A row is 16 pieces
// of 16 bytes; piece p of row r lies in slot p ^ 4 (r & 3): the four rows that a transposing load meets are in different banks.  Codes become bf16 on their
// way into LDS, once per workgroup.  Two LDS buffers, one barrier per chunk, the next chunk's loads in flight during the products.
//
// PLANES: 1: dY as bf16 numbers; 3: fp32 values of dY, split.
// Per-example call (WEIGHTED false): a workgroup contracts one example's tile, squares it, and stores it if asked.
// WEIGHTED, PLANES 1: a workgroup walks over the chunks of many examples.  With f_i = m_i 2^e_i, 1 <= m_i < 2, the power is put into
// the scales of X, exactly, and the running sum is kept in units of m_i: it is multiplied by m_(i-1) / m_i where an example begins, and by
// the last m at the end.  One set of accumulators for any number of examples, and each example meets its factor in fp32.
// WEIGHTED, PLANES 3: rows (example, token) of the whole call one after the other, dY times its factor in fp32, then split: for fp32 dY, and
// for examples of a few tokens, of which 32 rows hold several.
constexpr int CT = 128, CKC = 32, CK_ROW = 2 * CT, CK_PLANE = CKC * CK_ROW;      // bytes of a row, of an operand's chunk

template <int PLANES, bool WEIGHTED>
__global__ void __launch_bounds__(256, 2) ck_contract_kernel(const CkDenseArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char ck_lds[];
    __shared__ float red[4];
    constexpr bool ROWS = WEIGHTED && PLANES == 3;
    constexpr int STAGE = (PLANES + 1) * CK_PLANE;
    const int tiles = a.tiles_o * a.columns;
    const int slot = (int)(blockIdx.x / (unsigned)tiles), tile = (int)(blockIdx.x - (unsigned)slot * (unsigned)tiles);     // example or range
    const int tile_o = tile / a.columns, tile_k = tile - tile_o * a.columns;
    const int o0 = tile_o * CT, k0 = tile_k * CT;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wm = wave >> 1, wn = wave & 1;
    const int cpe = (a.tokens + CKC - 1) / CKC;                    // chunks of an example
    int c_begin = 0, c_end, len = 0;
    if constexpr (WEIGHTED) {
        c_begin = slot * a.per_range;
        c_end = min(c_begin + a.per_range, a.chunks);
    } else {
        len = ck_length(a, slot);
        c_end = (len + CKC - 1) / CKC;
    }

    if (tile_k == a.tiles_k) {                                     // the bias column: sums of dY, two threads to a feature
        const int o = o0 + (t & 127);
        float sum = 0.0f;
        if constexpr (WEIGHTED) {
            const long long total = (long long)a.n * a.tokens, per = ROWS ? CKC : 0;
            for (int c = c_begin; c < c_end; ++c) {
                const int ex = ROWS ? 0 : c / cpe;
                const long long first = ROWS ? c * per : (long long)ex * a.tokens + (c - ex * cpe) * CKC;
                const long long stop = ROWS ? min(first + CKC, total) : min(first + CKC, (long long)(ex + 1) * a.tokens);
                for (long long r = first + (t >> 7); r < stop; r += 2) {
                    const int i = (int)(r / a.tokens);
                    if (o >= a.cout || r - (long long)i * a.tokens >= ck_length(a, i)) continue;
                    const float f = clip_factor(a.group_sqnorm[i], a.clip_c);
                    if (f == 0.0f) continue;
                    const size_t at = (size_t)r * a.cout + o;
                    sum += f * (a.dy_bf16 ? bf16_bits_to_float(static_cast<const uint16_t *>(a.dy)[at]) : static_cast<const float *>(a.dy)[at]);
                }
            }
        } else if (o < a.cout) {
            for (int r = t >> 7; r < len; r += 2) {
                const size_t at = ((size_t)slot * a.tokens + r) * a.cout + o;
                sum += a.dy_bf16 ? bf16_bits_to_float(static_cast<const uint16_t *>(a.dy)[at]) : static_cast<const float *>(a.dy)[at];
            }
        }
        float *half = reinterpret_cast<float *>(ck_lds);
        half[t] = sum;
        __syncthreads();
        sum = t < 128 ? half[t] + half[t + 128] : 0.0f;
        const bool mine = t < 128 && o < a.cout;
        if constexpr (WEIGHTED) {
            if (mine) {
                float *out = a.out_b + (size_t)slot * a.stride_b + o;
                *out = a.add ? *out + sum : sum;
            }
        } else {
            if (mine && a.stored) a.out_b[(size_t)slot * a.stride_b + o] = sum;
            const float tot = block_sum<4>(mine ? sum * sum : 0.0f, red);
            if (t == 0) a.partials[(size_t)slot * tiles + tile] = tot;
        }
        return;
    }

    // this thread's pieces of a chunk: 16 codes of row t / 8; eight values of dY of rows t / 16 and t / 16 + 16
    const int xr = t >> 3, xp = t & 7, x_col = k0 + xp * 16;
    const int yr = t >> 4, yp = t & 15, y_col = o0 + yp * 8, y_count = a.cout - y_col;
    const bool x_there = x_col < a.pitch;

    uint4 x_raw;
    uint32_t x_exp = 0;                                            // biased exponent of the scale
    uint4 y_raw[PLANES == 1 ? 2 : 1];
    float y_val[PLANES == 1 ? 1 : 2][8];
    int f_ex = 0, f_c = 0, f_len = len;                            // example mode: next chunk to fetch
    bool f_first = false;                                          //   and whether an example begins with it
    int f_pow = 0;                                                 //   its factor's exponent
    float f_m = 1.0f;
    if constexpr (WEIGHTED && !ROWS) { f_ex = c_begin / cpe; f_c = c_begin - f_ex * cpe; }
    bool have;                                                     // the fetched chunk has rows

    auto fetch_rows = [&](size_t row0, int rows, int pow) {        // rows row0 .. row0 + rows of both operands
        x_raw = make_uint4(0, 0, 0, 0);
        x_exp = 127;
        if (xr < rows && x_there) {
            const size_t row = row0 + xr;
            x_raw = *reinterpret_cast<const uint4 *>(a.codes + row * a.pitch + x_col);
            x_exp = (uint32_t)max((int)a.scales[row * (unsigned)(a.pitch / CK_BLOCK) + (x_col / CK_BLOCK)] + pow, 1);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = yr + 16 * u, count = r < rows ? y_count : 0;
            const size_t at = (row0 + r) * a.cout + y_col;
            if constexpr (PLANES == 1) y_raw[u] = load8(static_cast<const uint16_t *>(a.dy) + at, count);
            else load8f(static_cast<const float *>(a.dy) + at, count, y_val[u]);
        }
    };
    auto fetch = [&](int c) {
        if constexpr (ROWS) {
            // rows of any examples: each has its own length and factor
            const long long total = (long long)a.n * a.tokens, row0 = (long long)c * CKC;
            auto factor = [&](long long row) {
                if (row >= total) return 0.0f;
                const int i = (int)(row / a.tokens);
                if (row - (long long)i * a.tokens >= ck_length(a, i)) return 0.0f;
                return clip_factor(a.group_sqnorm[i], a.clip_c);
            };
            have = true;
            x_raw = make_uint4(0, 0, 0, 0);
            x_exp = 127;
            const long long xrow = row0 + xr;
            if (x_there && factor(xrow) != 0.0f) {
                x_raw = *reinterpret_cast<const uint4 *>(a.codes + xrow * a.pitch + x_col);
                x_exp = a.scales[xrow * (a.pitch / CK_BLOCK) + (x_col / CK_BLOCK)];
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const long long row = row0 + yr + 16 * u;
                const float f = factor(row);
                const int count = f != 0.0f ? y_count : 0;
                const size_t at = (size_t)row * a.cout + y_col;
                if (a.dy_bf16) widen8(load8(static_cast<const uint16_t *>(a.dy) + at, count), y_val[u]);
                else load8f(static_cast<const float *>(a.dy) + at, count, y_val[u]);
#pragma unroll
                for (int j = 0; j < 8; ++j) y_val[u][j] *= f;
            }
        } else if constexpr (WEIGHTED) {
            f_first = f_c == 0 || c == c_begin;
            if (f_first) {
                f_len = ck_length(a, f_ex);
                const float f = clip_factor(a.group_sqnorm[f_ex], a.clip_c);
                if (f == 0.0f) f_len = 0;                          // adds nothing, and no 0 * inf
                f_pow = f > 0.0f ? (int)(__float_as_uint(f) >> 23) - 127 : 0;
                f_m = f > 0.0f ? f * pow2_of(127 - f_pow) : 1.0f;
            }
            const int rows = min(f_len - f_c * CKC, CKC);
            have = rows > 0;
            if (have) fetch_rows((size_t)f_ex * a.tokens + f_c * CKC, rows, f_pow);
            if (++f_c == cpe) { f_c = 0; ++f_ex; }
        } else {
            have = true;
            fetch_rows((size_t)slot * a.tokens + c * CKC, min(len - c * CKC, CKC), 0);
        }
    };
    auto stage = [&](int buf) {
        char *s = ck_lds + buf * STAGE;
        const float scale = pow2_of((int)x_exp);
        const uint2 w0 = ck_bf16(x_raw.x, scale), w1 = ck_bf16(x_raw.y, scale), w2 = ck_bf16(x_raw.z, scale), w3 = ck_bf16(x_raw.w, scale);
        char *x = s + PLANES * CK_PLANE + xr * CK_ROW;
        *reinterpret_cast<uint4 *>(x + (((2 * xp) ^ ((xr & 3) << 2)) << 4)) = make_uint4(w0.x, w0.y, w1.x, w1.y);
        *reinterpret_cast<uint4 *>(x + (((2 * xp + 1) ^ ((xr & 3) << 2)) << 4)) = make_uint4(w2.x, w2.y, w3.x, w3.y);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = yr + 16 * u;
            char *y = s + r * CK_ROW + ((yp ^ ((r & 3) << 2)) << 4);
            if constexpr (PLANES == 1) {
                *reinterpret_cast<uint4 *>(y) = y_raw[u];
            } else {
                uint4 p[3];
                split8(y_val[u], p);
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4 *>(y + q * CK_PLANE) = p[q];
            }
        }
    };

    // A lane's part of a transposing load: row (lane / 4) % 4 of four, features 4 (lane % 4) .. of 16; the second group of 16 lanes takes the
    // next 16 features, the upper half of the wave the tokens eight further on.
    const int tr = (lane >> 2) & 3, tf = ((lane >> 4) & 1) * 16 + (lane & 3) * 4, th = lane >> 5;
    auto operand = [&](const char *base, int f0, int ks) {         // features f0 .. f0 + 31, tokens 16 ks .. 16 ks + 15
        const int f = f0 + tf;
        const char *p = base + (ks * 16 + th * 8 + tr) * CK_ROW + (((f >> 3) ^ (tr << 2)) << 4) + ((f >> 2) & 1) * 8;
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * CK_ROW));
        return __builtin_bit_cast(bf16x8, s16x8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w});
    };

    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    float unit = 1.0f;                                             // the sum's unit (m of the last example that was added)
    if (c_begin < c_end) { fetch(c_begin); if (have) stage(0); }
    bool now = have && c_begin < c_end, begins = f_first;
    float m = f_m;
    int buf = 0;
    __syncthreads();
    for (int c = c_begin; c < c_end; ++c) {
        const bool more = c + 1 < c_end;
        if (more) fetch(c + 1);
        if (now) {
            if (WEIGHTED && !ROWS && begins) {
                const float ratio = unit / m;
                unit = m;
                if (ratio != 1.0f) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int r = 0; r < 16; ++r) acc[i][j][r] *= ratio;
                }
            }
            const char *s = ck_lds + buf * STAGE;
#pragma unroll
            for (int ks = 0; ks < CKC / 16; ++ks) {
                bf16x8 vb[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) vb[j] = operand(s + PLANES * CK_PLANE, wn * 64 + j * 32, ks);
#pragma unroll
                for (int q = 0; q < PLANES; ++q)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const bf16x8 va = operand(s + q * CK_PLANE, wm * 64 + i * 32, ks);
#pragma unroll
                        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, vb[j], acc[i][j], 0, 0, 0);
                    }
            }
        }
        now = more && have;
        begins = f_first;
        m = f_m;
        buf ^= 1;
        if (now) stage(buf);
        __syncthreads();
    }

    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int col = k0 + wn * 64 + j * 32 + (lane & 31), row0 = o0 + wm * 64 + i * 32 + (lane >> 5) * 4;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = row0 + (r >> 2) * 8 + (r & 3);
                const bool there = row < a.cout && col < a.cin;
                const float v = WEIGHTED && !ROWS ? acc[i][j][r] * unit : acc[i][j][r];
                if constexpr (WEIGHTED) {
                    if (there) {
                        float *out = a.out_w + (size_t)slot * a.stride_w + (size_t)row * a.cin + col;
                        *out = a.add ? *out + v : v;
                    }
                } else {
                    if (there) ss += v * v;
                    if (there && a.stored) a.out_w[(size_t)slot * a.stride_w + (size_t)row * a.cin + col] = v;
                }
            }
        }
    if constexpr (!WEIGHTED) {
        const float tot = block_sum<4>(ss, red);
        if (t == 0) a.partials[(size_t)slot * tiles + tile] = tot;
    }
}

// acc[e] += sum of the ranges' sums, in order (four values a thread where the count allows it)
__global__ void __launch_bounds__(256) ck_ranges_kernel(const float *part, size_t stride, int ranges, size_t count, float *acc)
{
    const size_t e = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (e >= count) return;
    if (e + 4 <= count) {
        float4 s = *reinterpret_cast<const float4 *>(part + e);
        for (int r = 1; r < ranges; ++r) {
            const float4 v = *reinterpret_cast<const float4 *>(part + r * stride + e);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        float4 *out = reinterpret_cast<float4 *>(acc + e);
        const float4 o = *out;
        *out = make_float4(o.x + s.x, o.y + s.y, o.z + s.z, o.w + s.w);
        return;
    }
    for (size_t i = e; i < count; ++i) {
        float s = part[i];
        for (int r = 1; r < ranges; ++r) s += part[r * stride + i];
        acc[i] += s;
    }
}

// ------------------------------------------------------------------------------------------
// Norms of short examples from the two Gram matrices of their tokens, T^2 (F + O) operations for 2 T F O:
//     |dW_i|^2 + |db_i|^2 = sum_{t, u} (dY_t . dY_u) (X_t . X_u + bias).
// A workgroup takes one pair of tiles of 32 B tokens of one example (those above the diagonal once, counted twice); its waves share the
// features, and their sums meet in LDS in the order of the waves.  Tokens and features both operands agree on need no order: a lane
// loads 16 consecutive features of a token, codes or bf16, and gives eight to each of two matrix instructions; nothing goes through
// LDS on the way in.
template <int B, int NW>
__global__ void __launch_bounds__(64 * NW) ck_gram_kernel(const CkDenseArgs a, int pairs)
{
    extern __shared__ __attribute__((aligned(16))) char ck_lds[];
    __shared__ float red[NW];
    const int ex = (int)(blockIdx.x / (unsigned)pairs);
    int pair = (int)(blockIdx.x - (unsigned)ex * (unsigned)pairs), tile_a = 0;
    while (pair > tile_a) { ++tile_a; pair -= tile_a; }            // pairs (0,0) (1,0) (1,1) (2,0) ...
    const int tile_b = pair;
    const bool diagonal = tile_a == tile_b;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, half = lane >> 5;
    const int len = ck_length(a, ex);
    if (tile_a * 32 * B >= len) {                                  // (tile_b is not the larger one)
        if (t == 0) a.partials[blockIdx.x] = 0.0f;
        return;
    }

    f32x16 gx[B][B], gy[B][B];
#pragma unroll
    for (int i = 0; i < B; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) gx[i][j][r] = gy[i][j][r] = 0.0f;

    size_t row[2][B];
    bool there[2][B];
#pragma unroll
    for (int i = 0; i < B; ++i) {
        const int ta = (tile_a * B + i) * 32 + (lane & 31), tb = (tile_b * B + i) * 32 + (lane & 31);
        there[0][i] = ta < len; row[0][i] = (size_t)ex * a.tokens + ta;
        there[1][i] = tb < len; row[1][i] = (size_t)ex * a.tokens + tb;
    }
    auto products = [&](const uint4 (&va)[B][2], const uint4 (&vb)[B][2], f32x16 (&g)[B][B]) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < B; ++i)
#pragma unroll
                for (int j = 0; j < B; ++j)
                    g[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, va[i][q]), __builtin_bit_cast(bf16x8, vb[j][q]), g[i][j], 0, 0, 0);
    };

    const int x_blocks = a.pitch / CK_BLOCK;
    auto load_x = [&](int side, int blk, uint4 (&v)[B][2]) {
#pragma unroll
        for (int i = 0; i < B; ++i) {
            uint4 c = make_uint4(0, 0, 0, 0);
            float scale = 1.0f;
            if (there[side][i]) {
                c = *reinterpret_cast<const uint4 *>(a.codes + row[side][i] * a.pitch + blk * 32 + half * 16);
                scale = pow2_of(a.scales[row[side][i] * (unsigned)x_blocks + blk]);
            }
            const uint2 w0 = ck_bf16(c.x, scale), w1 = ck_bf16(c.y, scale), w2 = ck_bf16(c.z, scale), w3 = ck_bf16(c.w, scale);
            v[i][0] = make_uint4(w0.x, w0.y, w1.x, w1.y);
            v[i][1] = make_uint4(w2.x, w2.y, w3.x, w3.y);
        }
    };
    for (int blk = wave; blk < x_blocks; blk += NW) {
        uint4 va[B][2], vb[B][2];
        load_x(0, blk, va);
        if (diagonal) products(va, va, gx);
        else { load_x(1, blk, vb); products(va, vb, gx); }
    }

    const int y_blocks = (a.cout + 31) / 32;
    auto load_y = [&](int side, int blk, uint4 (&v)[B][2]) {
        const int col = blk * 32 + half * 16;
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int count = there[side][i] ? a.cout - col : 0;
            const uint16_t *p = static_cast<const uint16_t *>(a.dy) + row[side][i] * a.cout + col;
            v[i][0] = load8(p, count);
            v[i][1] = load8(p + 8, count - 8);
        }
    };
    for (int blk = wave; blk < y_blocks; blk += NW) {
        uint4 va[B][2], vb[B][2];
        load_y(0, blk, va);
        if (diagonal) products(va, va, gy);
        else { load_y(1, blk, vb); products(va, vb, gy); }
    }

    // the waves' sums: wave w's value q of lane l at [w][q][l]; a thread adds up values of its own lane position
    float *buf = reinterpret_cast<float *>(ck_lds);
    constexpr int Q = 16 * B * B, MINE = Q / NW;                   // values of a lane; of which this wave adds up MINE
    static_assert(Q % NW == 0, "values are dealt to waves evenly");
    auto put = [&](const f32x16 (&g)[B][B]) {
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int j = 0; j < B; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) buf[(wave * Q + (i * B + j) * 16 + r) * 64 + lane] = g[i][j][r];
    };
    auto get = [&](float (&s)[MINE]) {
#pragma unroll
        for (int q = 0; q < MINE; ++q) {
            s[q] = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) s[q] += buf[(w * Q + wave * MINE + q) * 64 + lane];
        }
    };
    float sx[MINE], sy[MINE];
    put(gx);
    __syncthreads();
    get(sx);
    __syncthreads();
    put(gy);
    __syncthreads();
    get(sy);
    float ss = 0.0f;
#pragma unroll
    for (int q = 0; q < MINE; ++q) ss += (a.has_bias ? sx[q] + 1.0f : sx[q]) * sy[q];        // tokens that are not there: 0 dY . dY
    const float tot = block_sum<NW>(ss, red);
    if (t == 0) a.partials[blockIdx.x] = diagonal ? tot : 2.0f * tot;
}

// ---- plans --------------------------------------------------------------------------------

struct CkPlan {
    bool gram;
    int gram_tiles;                  // tiles of 32 B tokens of an example
    int gram_b;
    size_t per_example;              // partial squared norms
    int ranges, per_range, chunks;   // weighted
    bool rows;
};

int ck_tiles(int v) { return (v + CT - 1) / CT; }

// Gram matrices where they take fewer operations than the contraction, tiles counted whole.
CkPlan ck_plan(const Geo &g, int mode)
{
    CkPlan p = {};
    const int tiles_o = ck_tiles(g.cout), columns = ck_tiles(g.cin) + g.has_bias;
    if (mode == MODE_WEIGHTED) {
        // 32 rows hold several examples of a few tokens each, at three products for one
        p.rows = !g.bf16 || g.h < 16;
        const long long chunks = p.rows ? ((long long)g.n * g.h + CKC - 1) / CKC : (long long)g.n * ((g.h + CKC - 1) / CKC);
        p.chunks = (int)chunks;
        // ranges of the call's chunks until there are two workgroups for each compute unit; a range has eight chunks at least
        const long long want = (512 + tiles_o * columns - 1) / (tiles_o * columns);
        const long long ranges = std::max(1ll, std::min(want, chunks / 8));
        p.per_range = (int)((chunks + ranges - 1) / ranges);
        p.ranges = (int)((chunks + p.per_range - 1) / p.per_range);
        return p;
    }
    p.per_example = (size_t)tiles_o * columns;
    if (mode == MODE_NORM && g.bf16) {
        p.gram_b = g.h <= 32 ? 1 : 2;
        p.gram_tiles = (g.h + 32 * p.gram_b - 1) / (32 * p.gram_b);
        const double pairs = 0.5 * p.gram_tiles * (p.gram_tiles + 1), side = 32.0 * p.gram_b;
        const double gram = pairs * side * side * ((double)g.cin + g.cout);
        const double direct = (double)((g.h + CKC - 1) / CKC * CKC) * tiles_o * CT * (double)ck_tiles(g.cin) * CT;
        p.gram = gram < direct;
        if (p.gram) p.per_example = (size_t)p.gram_tiles * (p.gram_tiles + 1) / 2;
    }
    return p;
}

size_t align16(size_t b) { return (b + 15) & ~(size_t)15; }
size_t align4(size_t v) { return (v + 3) & ~(size_t)3; }

}  // namespace

size_t checkpoint_ws_bytes(const Geo &g, int mode)
{
    const CkPlan p = ck_plan(g, mode);
    if (mode == MODE_WEIGHTED) return p.ranges > 1 ? 4 * (size_t)p.ranges * (align4(g.pw) + align4(g.pb)) : 0;
    // both per-example forms: a caller sizes its workspace once
    const CkPlan q = ck_plan(g, mode == MODE_NORM ? MODE_MATERIALISE : MODE_NORM);
    return align16(4 * (size_t)g.n * std::max(p.per_example, q.per_example));
}

dp_status launch_checkpoint_dense(const Geo &g, int mode, const uint8_t *codes, const uint8_t *scales, const void *dy, const int32_t *lengths,
                                  float *out_w, float *out_b, size_t out_stride, float *sqnorm, const float *group_sqnorm, float clip_c,
                                  void *ws, hipStream_t s)
{
    const CkPlan p = ck_plan(g, mode);
    CkDenseArgs a = {};
    a.codes = codes; a.scales = scales; a.dy = dy; a.lengths = lengths;
    a.n = g.n; a.tokens = g.h; a.cin = g.cin; a.cout = g.cout; a.pitch = ck_pitch(g.cin);
    a.dy_bf16 = g.bf16; a.has_bias = g.has_bias;
    a.tiles_o = ck_tiles(g.cout); a.tiles_k = ck_tiles(g.cin); a.columns = a.tiles_k + g.has_bias;
    const size_t tiles = (size_t)a.tiles_o * a.columns;
    if (mode == MODE_WEIGHTED) {
        a.group_sqnorm = group_sqnorm; a.clip_c = clip_c;
        a.chunks = p.chunks; a.per_range = p.per_range;
        a.add = p.ranges == 1;
        a.out_w = out_w; a.out_b = out_b;
        if (p.ranges > 1) {
            a.out_w = static_cast<float *>(ws);
            a.stride_w = align4(g.pw);
            a.out_b = a.out_w + p.ranges * a.stride_w;
            a.stride_b = align4(g.pb);
        }
        const dim3 grid((unsigned)(tiles * p.ranges));
        profile_begin(s);
        dp_status st = p.rows ? launch_lds<ck_contract_kernel<3, true>>(grid, 256, 2 * 4 * CK_PLANE, s, a)
                              : launch_lds<ck_contract_kernel<1, true>>(grid, 256, 2 * 2 * CK_PLANE, s, a);
        profile_end(s);
        if (st != DP_OK || p.ranges == 1) return st;
        hipLaunchKernelGGL(ck_ranges_kernel, dim3((unsigned)((g.pw + 1023) / 1024)), dim3(256), 0, s, a.out_w, a.stride_w, p.ranges, g.pw, out_w);
        if (g.pb)
            hipLaunchKernelGGL(ck_ranges_kernel, dim3((unsigned)((g.pb + 1023) / 1024)), dim3(256), 0, s, a.out_b, a.stride_b, p.ranges, g.pb, out_b);
        return check_launch("checkpoint_ranges");
    }
    a.partials = static_cast<float *>(ws);
    a.stored = out_w != nullptr;
    a.out_w = out_w; a.out_b = out_b;
    a.stride_w = out_stride ? out_stride : g.pw;
    a.stride_b = out_stride ? out_stride : g.pb;
    dp_status st;
    profile_begin(s);
    if (p.gram) {
        const dim3 grid((unsigned)(g.n * p.per_example));
        st = p.gram_b == 1 ? launch_lds<ck_gram_kernel<1, 8>>(grid, 512, 8 * 16 * 64 * 4, s, a, (int)p.per_example)
                           : launch_lds<ck_gram_kernel<2, 4>>(grid, 256, 4 * 64 * 64 * 4, s, a, (int)p.per_example);
    } else {
        const dim3 grid((unsigned)(tiles * g.n));
        st = g.bf16 ? launch_lds<ck_contract_kernel<1, false>>(grid, 256, 2 * 2 * CK_PLANE, s, a)
                    : launch_lds<ck_contract_kernel<3, false>>(grid, 256, 2 * 4 * CK_PLANE, s, a);
    }
    profile_end(s);
    if (st != DP_OK || !sqnorm) return st;
    return launch_sum_partials(a.partials, g.n, (int)p.per_example, sqnorm, s);
}

}  // namespace dp
