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
//   ck_again_kernel    those of them that cancellation has left without digits, as sums of squares
//   ck_contract_kernel everything else
#include "checkpoint.h"

#include <algorithm>
#include <cmath>

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
    int has_bias, stored, add;
    int tiles_k, tiles_o, slots;     // tiles along k, along o; examples, or ranges
    int columns;                     // of tiles: tiles_k, and one more for a bias
    int chunks;                      // weighted, rows of any examples: chunks in all
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
// Contraction over tokens.  A workgroup of four waves owns a tile of 128 (o) x 64 NJ (k), NJ 2 or 4, a wave 64 x 32 NJ of it (2 x NJ blocks of
// 32 x 32).  A chunk is 64 tokens (NJ 4 or PLANES 3: 32); both operands lie in LDS as they lie in memory, [token][feature], and the matrix operands, which
// want consecutive tokens of a feature, are read with the transposing LDS loads (four tokens of 16 features each).  A row is 16 pieces
// of 16 bytes; piece p of row r lies in slot p ^ 4 (r & 3): the four rows that a transposing load meets are in different banks.  Codes
// become bf16 on their way into LDS, once per workgroup.  Two LDS buffers, one barrier per chunk; the loads of the two chunks after the next
// are in flight during the products.  The wider tile takes in two thirds of the bytes for a product (a code is one byte, dY's value two).
//
// PLANES: 1: dY as bf16 numbers; 3: fp32 values of dY, split.
// Per-example call (WEIGHTED false): a workgroup contracts one example's tile, squares it, and stores it if asked.
// WEIGHTED, PLANES 1: a workgroup walks over a range of the chunks of all examples, as many as any other range's; chunks after an example's
// last token are not among them.  With f_i = m_i 2^e_i, -16 <= e_i <= 0, 1 <= m_i < 2 (below 2^-16: m_i < 1), the power is put into
// the scales of X, exactly: values of a checkpoint times 2^-16 are normal bf16 numbers still (2^-9 2^-100 2^-16).  The running sum is kept in units of m_i: it is
// multiplied by m_(i-1) / m_i where an example begins, and by the last m at the end.  It stays below n times an example's norm, as
// f_i <= C / norm_i.  One set of accumulators for any number of examples, and each example meets its factor in fp32.  A factor that is no normal fp32
// number counts as 0 (m_(i-1) / m_i would pass fp32's range).
// WEIGHTED, PLANES 3: rows (example, token) of the whole call one after the other, dY times its factor in fp32, then split: for fp32 dY, and
// for examples of a few tokens, of which 32 rows hold several.
// Bias: a column of workgroups of its own adds up dY.
// Measured: norms of 8 x 1024 tokens 1024 -> 2048 34.8 us, 988 TFLOP/s (a library product of 8192^3: 1282); clipped sum of 16 x 512 tokens
// 2048 -> 2048 93.5 us, 735 TFLOP/s, and 11 us to join two ranges (factors worked out by every chunk instead of once: 94.4; 2 x 512 tokens
// 4096 -> 1024 24.6 instead of 23.2).  Bound by the LDS (a chunk's operands are 96 KB written and read for a workgroup, 0.3 us of its 0.75) and by
// the waits that two workgroups a compute unit leave uncovered (<1, 4, true, true, false>, wide sums of an odd number of features, keeps five registers
// in memory; no other instance does); 16 x 128 tokens 768 -> 768, 8 chunks a workgroup at most, by trips to memory one after
// the other.  Three stages of loads instead of two: no gain (registers); chunks of 32 with three workgroups: slower.
// WORDS: rows of dY begin at whole dwords: pieces by buffer loads, which give zeros beyond the chunk's last row (what a row's last piece takes
// from the next row is multiplied into features beyond the last, which nobody reads).  Else (bf16, an odd number of features) every other
// row begins in the middle of a dword: five dwords around a piece, shifted into place on their way into LDS.
constexpr int CT = 128;                                            // o of a tile
constexpr int ck_chunk(int planes, int nj) { return planes == 1 && nj == 2 ? 64 : 32; }
constexpr int ck_stage_bytes(int planes, int nj) { return ck_chunk(planes, nj) * (planes * 2 * CT + nj * 128); }
constexpr int CK_TABLE = 1024;                                     // examples of a weighted call
constexpr size_t CK_GROUPS = (size_t)1 << 23;                      // workgroups of a launch (fewer than 2^32 threads)
constexpr unsigned CK_NOWHERE = 0xFFFFFFE0u;                       // an offset beyond any buffer
constexpr int CK_POWER = 16;                                       // of a factor, in the scales of X
static_assert(CK_LOW - 9 - CK_POWER >= -126, "scaled values are normal bf16 numbers");
constexpr float CK_LEAST_FACTOR = 0x1p-126f;

template <int PLANES, int NJ, bool WEIGHTED, bool BF16, bool WORDS>
__global__ void __launch_bounds__(256, 2) ck_contract_kernel(const CkDenseArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char ck_lds[];
    __shared__ float red[4];
    typedef typename In<BF16>::type E;
    constexpr bool ROWS = WEIGHTED && PLANES == 3;
    constexpr int CK = ck_chunk(PLANES, NJ), STAGE = ck_stage_bytes(PLANES, NJ);
    constexpr int CTK = 64 * NJ, X_ROW = 2 * CTK, Y_ROW = 2 * CT, PLANE = CK * Y_ROW;      // k of a tile; bytes of a row of an operand, of a plane of dY
    constexpr int XW = CTK / 16, XS = 256 / XW, XP = CK / XS, YP = CK / 16;        // pieces of X (16 codes) in a row, rows between a thread's, pieces of a thread and chunk
    // workgroup -> XCD goes round robin: an XCD takes a run of consecutive tiles, which share an example's operands in its L2
    const unsigned per_xcd = gridDim.x >> 3, block = (blockIdx.x & 7u) * per_xcd + (blockIdx.x >> 3);
    const unsigned tiles = (unsigned)(a.tiles_o * a.columns);
    const int slot = (int)(block / tiles), tile = (int)(block - (unsigned)slot * tiles);     // example or range
    if (slot >= a.slots) return;
    const int tile_o = tile / a.columns, tile_k = tile - tile_o * a.columns;
    const int o0 = tile_o * CT, k0 = tile_k * CTK;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wm = wave >> 1, wn = wave & 1;
    int c_begin = 0, c_end = 0, len = 0;
    if constexpr (ROWS) {
        c_begin = (int)((long long)a.chunks * slot / a.slots);
        c_end = (int)((long long)a.chunks * (slot + 1) / a.slots);
    } else if constexpr (!WEIGHTED) {
        len = ck_length(a, slot);
        c_end = (len + CK - 1) / CK;
    }

    // this thread's pieces of a chunk: 16 codes of rows t / XW + XS u; eight values of dY of rows t / 16 + 16 u
    const int xr = t / XW, xp = t % XW, x_col = k0 + xp * 16;
    const int yr = t >> 4, yp = t & 15, y_col = o0 + yp * 8, y_count = a.cout - y_col;
    const unsigned x_off = x_col < a.pitch ? (unsigned)(xr * a.pitch + x_col) : CK_NOWHERE;
    const int s_pitch = a.pitch / CK_BLOCK;
    const unsigned s_off = x_col < a.pitch ? (unsigned)(xr * s_pitch + x_col / CK_BLOCK) : CK_NOWHERE;
    const unsigned y_off = y_count > 0 ? (unsigned)(yr * a.cout + y_col) * (unsigned)sizeof(E) : CK_NOWHERE;

    struct Slot {                                                  // a chunk on its way
        uint4 x[XP];
        uint32_t scale[XP];
        Raw8<BF16> y[YP];
        uint32_t y_more[WORDS ? 1 : YP];                           // odd rows: the dword after
        uint32_t odd;                                              //   and whether the chunk's first row begins in the middle of one
        int rows;                                                  // of the chunk (0: it adds nothing)
        bool begins;                                               // an example begins with it, of
        int ex;                                                    //   this number, hence
        int power;                                                 //   factor f = m 2^power
        float m, f;
    };
    int f_ex = 0, f_c = 0, f_len = len;                            // weighted, by example: what the next chunk belongs to
    // Ragged examples: lengths, and chunks of the examples before each, fetched together (one after the other they are a trip to memory each).
    // Factors as well, once for all chunks: an example that is left out is walked over without products.
    constexpr int TABLE = WEIGHTED && !ROWS ? CK_TABLE : 1;
    __shared__ int ex_len[TABLE], ex_before[TABLE], found, wave_chunks[4];
    __shared__ float ex_factor[TABLE];
    const __amdgpu_buffer_rsrc_t sq_buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.group_sqnorm), 0, (int)((unsigned)a.n * 4u), 0x00020000);
    float sq[4];
    if constexpr (WEIGHTED && !ROWS) {
#pragma unroll
        for (int u = 0; u < 4; ++u) sq[u] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sq_buffer, 16 * t + 4 * u, 0, 0));
    }
    auto place_factors = [&]() {                                   // (after the first chunks are on their way)
        if constexpr (WEIGHTED && !ROWS) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (4 * t + u < a.n) ex_factor[4 * t + u] = clip_factor(sq[u], a.clip_c);
            __syncthreads();
        }
    };
    if constexpr (WEIGHTED && !ROWS) {
        if (!a.lengths) {
            const int cpe = (a.tokens + CK - 1) / CK;
            c_begin = (int)((long long)a.n * cpe * slot / a.slots);
            c_end = (int)((long long)a.n * cpe * (slot + 1) / a.slots);
            f_ex = c_begin / cpe;
            f_c = c_begin - f_ex * cpe;
            f_len = a.tokens;
        } else {
            int mine = 0, before[4], count[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = 4 * t + u, l = i < a.n ? ck_length(a, i) : 0;
                if (i < a.n) ex_len[i] = l;
                before[u] = mine;
                mine += count[u] = (l + CK - 1) / CK;
            }
            int upto = mine;                                       // of this wave's threads up to this one
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int v = __shfl_up(upto, off, 64);
                upto += lane >= off ? v : 0;
            }
            if (lane == 63) wave_chunks[wave] = upto;
            if (t == 0) found = 0;
            __syncthreads();
            int base = upto - mine, total = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                base += w < wave ? wave_chunks[w] : 0;
                total += wave_chunks[w];
            }
            total = __builtin_amdgcn_readfirstlane(total);
            c_begin = (int)((long long)total * slot / a.slots);
            c_end = (int)((long long)total * (slot + 1) / a.slots);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = 4 * t + u, first = base + before[u];
                if (i < a.n) ex_before[i] = first;
                if (c_begin >= first && c_begin < first + count[u]) found = i;
            }
            __syncthreads();
            f_ex = __builtin_amdgcn_readfirstlane(found);
            f_c = c_begin - __builtin_amdgcn_readfirstlane(ex_before[f_ex]);
        }
    }

    auto load_rows = [&](Slot &s, unsigned row0_any, int rows_any) {
        // the same in every lane, which the compiler does not always see (and a buffer in vector registers is read lane by lane)
        const size_t row0 = (unsigned)__builtin_amdgcn_readfirstlane((int)row0_any);
        const int rows = __builtin_amdgcn_readfirstlane(rows_any);
        const __amdgpu_buffer_rsrc_t xb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.codes) + row0 * (unsigned)a.pitch, 0, rows * a.pitch, 0x00020000);
        const __amdgpu_buffer_rsrc_t sb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.scales) + row0 * (unsigned)s_pitch, 0, rows * s_pitch, 0x00020000);
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int u = 0; u < XP; ++u) {
            const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xb, x_off + (x_off == CK_NOWHERE ? 0u : (unsigned)(XS * u * a.pitch)), 0, 0));
            s.x[u] = make_uint4(v.x, v.y, v.z, v.w);
            s.scale[u] = __builtin_amdgcn_raw_buffer_load_b8(sb, s_off + (s_off == CK_NOWHERE ? 0u : (unsigned)(XS * u * s_pitch)), 0, 0);
        }
        const E *dy = static_cast<const E *>(a.dy) + row0 * (unsigned)a.cout;
        if constexpr (WORDS) {
            const __amdgpu_buffer_rsrc_t yb = __builtin_amdgcn_make_buffer_rsrc(const_cast<E *>(dy), 0, rows * a.cout * (int)sizeof(E), 0x00020000);
#pragma unroll
            for (int u = 0; u < YP; ++u) {
                const unsigned at = y_off + (y_off == CK_NOWHERE ? 0u : (unsigned)(16 * u * a.cout) * (unsigned)sizeof(E));
                const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(yb, at, 0, 0));
                if constexpr (BF16) {
                    s.y[u].w = make_uint4(v.x, v.y, v.z, v.w);
                } else {
                    const u32x4 n = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(yb, at == CK_NOWHERE ? at : at + 16u, 0, 0));
                    s.y[u].w[0] = __uint_as_float(v.x); s.y[u].w[1] = __uint_as_float(v.y); s.y[u].w[2] = __uint_as_float(v.z); s.y[u].w[3] = __uint_as_float(v.w);
                    s.y[u].w[4] = __uint_as_float(n.x); s.y[u].w[5] = __uint_as_float(n.y); s.y[u].w[6] = __uint_as_float(n.z); s.y[u].w[7] = __uint_as_float(n.w);
                }
            }
        } else {
            const uintptr_t first = reinterpret_cast<uintptr_t>(dy);
            s.odd = (uint32_t)(first >> 1) & 1u;
            const __amdgpu_buffer_rsrc_t yb = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(first & ~(uintptr_t)3), 0, ((rows * a.cout + (int)s.odd) * 2 + 3) & ~3, 0x00020000);
#pragma unroll
            for (int u = 0; u < YP; ++u) {
                // (the dword of the chunk's last value may hold the next row's first as well)
                const unsigned at = y_off == CK_NOWHERE || yr + 16 * u >= rows ? CK_NOWHERE : (y_off + (unsigned)(16 * u * a.cout) * 2u + 2u * s.odd) & ~3u;
                const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(yb, at, 0, 0));
                s.y[u].w = make_uint4(v.x, v.y, v.z, v.w);
                s.y_more[u] = __builtin_amdgcn_raw_buffer_load_b32(yb, at == CK_NOWHERE ? at : at + 16u, 0, 0);
            }
        }
    };
    auto fetch = [&](Slot &s, int c) {
        s.rows = 0;
        s.begins = false;
        s.ex = 0;
        if (c >= c_end) return;
        if constexpr (ROWS) {
            const unsigned row0 = (unsigned)c * CK;
            s.rows = (int)min((unsigned)a.n * (unsigned)a.tokens - row0, (unsigned)CK);
            load_rows(s, row0, s.rows);
        } else if constexpr (WEIGHTED) {
            s.begins = f_c == 0 || c == c_begin;
            if (s.begins && a.lengths) {
                while (__builtin_amdgcn_readfirstlane(ex_len[f_ex]) == 0) ++f_ex;         // (there are chunks: an example with some follows)
                f_len = __builtin_amdgcn_readfirstlane(ex_len[f_ex]);
            }
            s.ex = f_ex;
            s.rows = min(f_len - f_c * CK, CK);
            load_rows(s, (unsigned)f_ex * (unsigned)a.tokens + (unsigned)(f_c * CK), s.rows);
            if (++f_c * CK >= f_len) { f_c = 0; ++f_ex; }
        } else {
            s.rows = min(len - c * CK, CK);
            load_rows(s, (unsigned)slot * (unsigned)a.tokens + (unsigned)(c * CK), s.rows);
        }
    };
    // weighted, by example: the factor of a chunk that has arrived; one of factor 0 adds nothing (and no 0 * inf)
    auto ready = [&](Slot &s) {
        if constexpr (WEIGHTED && !ROWS) {
            s.f = __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(ex_factor[s.ex])));
            if (s.f < CK_LEAST_FACTOR) { s.f = 0.0f; s.rows = 0; }
            s.power = max((int)(__float_as_uint(s.f) >> 23) - 127, -CK_POWER);
            s.m = s.f * pow2_of(127 - s.power);
        }
    };
    auto piece_y = [&](const Slot &s, int u) {                     // piece u of dY as it is
        Raw8<BF16> y = s.y[u];
        if constexpr (!WORDS) {
            const uint32_t bits = ((((uint32_t)yr & 1u) ^ s.odd) & 1u) * 16u;         // (an odd number of features: rows take turns)
            y.w = make_uint4(funnel(y.w.y, y.w.x, bits), funnel(y.w.z, y.w.y, bits), funnel(y.w.w, y.w.z, bits), funnel(s.y_more[u], y.w.w, bits));
        }
        return y;
    };
    // rows of any examples: the factors of a chunk's rows (0 beyond lengths and the last row) in LDS, two chunks ahead, from what was loaded
    // four ahead; each row's example is a division, its factor a square root and another, once and not in every thread that holds a piece of it
    struct About { float sq; int token, len; };
    __shared__ float row_factors[2][ROWS ? 32 : 1];
    const __amdgpu_buffer_rsrc_t len_buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t *>(a.lengths), 0, a.lengths ? (int)((unsigned)a.n * 4u) : 0, 0x00020000);
    auto about = [&](About &b, int c) {
        if constexpr (ROWS) {
            const unsigned row = (unsigned)c * CK + (t & 31), i = row / (unsigned)a.tokens;        // beyond the last row: no squared norm there, token 0
            b.sq = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sq_buffer, 4 * i, 0, 0));
            b.len = (int)__builtin_amdgcn_raw_buffer_load_b32(len_buffer, 4 * i, 0, 0);
            b.token = i < (unsigned)a.n ? (int)(row - i * (unsigned)a.tokens) : a.tokens;
        }
    };
    auto place = [&](const About &b, int buf) {
        if constexpr (ROWS)
            if (t < 32) row_factors[buf][t] = b.token < (a.lengths ? b.len : a.tokens) ? clip_factor(b.sq, a.clip_c) : 0.0f;
    };
    About r0, r1;
    if constexpr (ROWS) {
        about(r0, c_begin);
        about(r1, c_begin + 1);
        place(r0, 0);
        place(r1, 1);
        about(r0, c_begin + 2);
        about(r1, c_begin + 3);
    }
    auto stage_x = [&](const Slot &s, int u, int buf) {            // piece u of X into LDS
        const int r = xr + XS * u;
        uint4 x = s.x[u];
        if constexpr (ROWS)
            if (row_factors[buf][r] == 0.0f) x = make_uint4(0, 0, 0, 0);
        // (beyond the checkpoint's rows scales are 0: no power of a factor there)
        const float scale = pow2_of(WEIGHTED && !ROWS ? max((int)s.scale[u] + s.power, 1) : (int)s.scale[u]);
        const uint2 w0 = ck_bf16(x.x, scale), w1 = ck_bf16(x.y, scale), w2 = ck_bf16(x.z, scale), w3 = ck_bf16(x.w, scale);
        char *to = ck_lds + buf * STAGE + PLANES * PLANE + r * X_ROW;
        *reinterpret_cast<uint4 *>(to + (((2 * xp) ^ ((r & 3) << 2)) << 4)) = make_uint4(w0.x, w0.y, w1.x, w1.y);
        *reinterpret_cast<uint4 *>(to + (((2 * xp + 1) ^ ((r & 3) << 2)) << 4)) = make_uint4(w2.x, w2.y, w3.x, w3.y);
    };
    auto stage_y = [&](const Slot &s, int u, int buf) {            // piece u of dY
        const int r = yr + 16 * u;
        char *to = ck_lds + buf * STAGE + r * Y_ROW + ((yp ^ ((r & 3) << 2)) << 4);
        if constexpr (PLANES == 1) {
            *reinterpret_cast<uint4 *>(to) = piece_y(s, u).w;
        } else {
            float v[8];
            piece_y(s, u).get(v);
            if constexpr (ROWS) {
                const float f = row_factors[buf][r];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = f == 0.0f ? 0.0f : v[j] * f;
            }
            uint4 p[3];
            split8(v, p);
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4 *>(to + q * PLANE) = p[q];
        }
    };
    auto stage = [&](const Slot &s, int buf) {
#pragma unroll
        for (int u = 0; u < XP; ++u) stage_x(s, u, buf);
#pragma unroll
        for (int u = 0; u < YP; ++u) stage_y(s, u, buf);
    };

    if (tile_k == a.tiles_k) {                                     // the column of the bias: sums of dY (X's pieces lie beyond its rows)
        float sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
        auto add = [&](Slot &s, int buf) {
            ready(s);
            if (s.rows <= 0) return;
#pragma unroll
            for (int u = 0; u < YP; ++u) {
                float v[8], f = 1.0f;
                piece_y(s, u).get(v);
                if constexpr (ROWS) f = row_factors[buf][yr + 16 * u];
                else if constexpr (WEIGHTED) f = s.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] = f == 0.0f ? sum[j] : fmaf(f, v[j], sum[j]);
            }
        };
        Slot b0, b1;
        fetch(b0, c_begin);
        place_factors();
        for (int c = c_begin; c < c_end; c += 2) {
            if constexpr (ROWS) __syncthreads();
            fetch(b1, c + 1);
            add(b0, 0);
            fetch(b0, c + 2);
            add(b1, 1);
            if constexpr (ROWS) {
                __syncthreads();
                place(r0, 0);
                place(r1, 1);
                about(r0, c + 4);
                about(r1, c + 5);
            }
        }
        float *sums = reinterpret_cast<float *>(ck_lds);
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[yr * CT + yp * 8 + j] = sum[j];
        __syncthreads();
        float ss = 0.0f;
        if (t < CT && o0 + t < a.cout) {
            float v = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) v += sums[r * CT + t];
            if constexpr (WEIGHTED) {
                float *out = a.out_b + (size_t)slot * a.stride_b + o0 + t;
                *out = a.add ? *out + v : v;
            } else {
                ss = v * v;
                if (a.stored) a.out_b[(size_t)slot * a.stride_b + o0 + t] = v;
            }
        }
        if constexpr (!WEIGHTED) {
            const float tot = block_sum<4>(ss, red);
            if (t == 0) a.partials[(size_t)slot * tiles + tile] = tot;
        }
        return;
    }

    // A lane's part of a transposing load: row (lane / 4) % 4 of four, features 4 (lane % 4) .. of 16; the second group of 16 lanes takes the
    // next 16 features, the upper half of the wave the tokens eight further on.
    const int tr = (lane >> 2) & 3, tf = ((lane >> 4) & 1) * 16 + (lane & 3) * 4, th = lane >> 5;
    auto operand = [&](const char *base, int row, int f0, int ks) {        // features f0 .. f0 + 31, tokens 16 ks .. 16 ks + 15, rows of `row` bytes
        const int f = f0 + tf;
        const char *p = base + (ks * 16 + th * 8 + tr) * row + (((f >> 3) ^ (tr << 2)) << 4) + ((f >> 2) & 1) * 8;
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * row));
        return __builtin_bit_cast(bf16x8, s16x8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w});
    };

    f32x16 acc[2][NJ];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    float unit = 1.0f;                                             // the sum's unit: m of the last example that was added

    struct Now { int rows; bool begins; float m; };                // of the chunk in LDS
    auto rescale = [&](const Now &now) {
        if constexpr (WEIGHTED && !ROWS) {
            const float ratio = now.begins && now.rows > 0 ? unit / now.m : 1.0f;
            unit = now.begins && now.rows > 0 ? now.m : unit;
            if (ratio != 1.0f) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i][j][r] *= ratio;
            }
        }
    };
    struct Operands { bf16x8 a[PLANES][2], b[NJ]; };               // of a K step (16 tokens)
    auto read = [&](Operands &o, int ks, int buf) {
        const char *base = ck_lds + buf * STAGE;
#pragma unroll
        for (int j = 0; j < NJ; ++j) o.b[j] = operand(base + PLANES * PLANE, X_ROW, wn * 32 * NJ + j * 32, ks);
#pragma unroll
        for (int q = 0; q < PLANES; ++q)
#pragma unroll
            for (int i = 0; i < 2; ++i) o.a[q][i] = operand(base + q * PLANE, Y_ROW, wm * 64 + i * 32, ks);
    };
    auto products = [&](const Operands &o) {
#pragma unroll
        for (int q = 0; q < PLANES; ++q)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(o.a[q][i], o.b[j], acc[i][j], 0, 0, 0);
    };
    // chunk c is in LDS buffer c & 1 (counted from the first), the two after it in registers; `next` holds c + 1 and takes c + 3
    Slot s0, s1;
    fetch(s0, c_begin);
    fetch(s1, c_begin + 1);
    place_factors();
    if constexpr (ROWS) __syncthreads();
    ready(s0);
    Now now = {s0.rows, s0.begins, s0.m};
    if (now.rows > 0) stage(s0, 0);
    fetch(s0, c_begin + 2);
    __syncthreads();
    // A chunk's products in two halves (the second one left out where no row reaches it), the next chunk staged in between: one set of
    // accumulators on every path.  Where the next chunk adds nothing, what is staged is not used.
    auto turn = [&](Slot &next, About &rows, int buf, int c) {
        rescale(now);
        ready(next);
        auto stage_xs = [&]() {
#pragma unroll
            for (int u = 0; u < XP; ++u) stage_x(next, u, buf ^ 1);
        };
        auto stage_ys = [&]() {
#pragma unroll
            for (int u = 0; u < YP; ++u) stage_y(next, u, buf ^ 1);
        };
        if constexpr (CK == 64) {
            if (now.rows > 0) {
                Operands p, q, r;
                read(p, 0, buf);
                read(q, 1, buf);
                products(p);
                stage_xs();
                read(r, 2, buf);
                products(q);
                if (now.rows > 32) {
                    read(p, 3, buf);
                    products(r);
                    stage_ys();
                    products(p);
                } else {
                    stage_ys();
                }
            } else {
                stage_xs();
                stage_ys();
            }
        } else {
            if (now.rows > 0) {
                Operands p, q;
                read(p, 0, buf);
                read(q, 1, buf);
                products(p);
                stage_xs();
                if (now.rows > 16) products(q);
                stage_ys();
            } else {
                stage_xs();
                stage_ys();
            }
        }
        now = {next.rows, next.begins, next.m};
        place(rows, buf);                                          // of chunk c + 2 (those of c were used before the last barrier)
        about(rows, c + 4);
        fetch(next, c + 3);
        __syncthreads();
    };
    for (int c = c_begin; c < c_end; c += 2) {
        turn(s1, r0, 0, c);
        if (c + 1 < c_end) turn(s0, r1, 1, c + 1);
    }

    // Rows beyond the last hold products of what followed in memory: gone.  (Columns beyond the last are sums of zeros.)
    const int out_row = wm * 64 + (lane >> 5) * 4, out_col = k0 + wn * 32 * NJ + (lane & 31);       // of the tile; row (r >> 2) * 8 + (r & 3) of a block
    if (o0 + CT > a.cout) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool there = o0 + out_row + i * 32 + (r >> 2) * 8 + (r & 3) < a.cout;
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j][r] = there ? acc[i][j][r] : 0.0f;
            }
    }
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if constexpr (WEIGHTED && !ROWS) acc[i][j][r] *= unit;
                if constexpr (!WEIGHTED) ss = fmaf(acc[i][j][r], acc[i][j][r], ss);
            }
    if (WEIGHTED || a.stored) {
        // the tile's rows as a buffer that ends with the last of them; columns beyond the last have no place in it
        float *first = a.out_w + (size_t)slot * a.stride_w + (size_t)o0 * a.cin;
        const __amdgpu_buffer_rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(first, 0, min(CT, a.cout - o0) * a.cin * 4, 0x00020000);
        const bool add = WEIGHTED && a.add;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int col = out_col + j * 32;
                const unsigned at = col < a.cin ? (unsigned)((out_row + i * 32) * a.cin + col) * 4u : CK_NOWHERE;
                const unsigned step = col < a.cin ? (unsigned)a.cin * 4u : 0u;
                float old[16];
                if (add) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) old[r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(out, at + step * ((r >> 2) * 8 + (r & 3)), 0, 0));
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] += old[r];
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float v = acc[i][j][r];
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), out, at + step * ((r >> 2) * 8 + (r & 3)), 0, 0);
                }
            }
    }
    if constexpr (!WEIGHTED) {
        const float tot = block_sum<4>(ss, red);
        if (t == 0) a.partials[(size_t)slot * tiles + tile] = tot;
    }
}

// acc[e] += sum of the ranges' sums, in order: `count_w` values of the weights, then those of the bias, which a range's sums hold one after the
// other (from `stride_w` on).
__global__ void __launch_bounds__(256) ck_ranges_kernel(const float *part, size_t stride, size_t stride_w, int ranges, size_t count_w, size_t count_b,
                                                        float *acc_w, float *acc_b)
{
    size_t e = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (e >= stride_w + count_b) return;
    const float *p = part + e;
    float4 s = *reinterpret_cast<const float4 *>(p);
#pragma unroll 8
    for (int r = 1; r < ranges; ++r) {
        const float4 v = *reinterpret_cast<const float4 *>(p + r * stride);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const bool bias = e >= stride_w;
    float *acc = bias ? acc_b : acc_w;
    const size_t count = bias ? count_b : count_w;
    if (bias) e -= stride_w;
    if (e + 4 <= count) {
        float4 *out = reinterpret_cast<float4 *>(acc + e);
        const float4 o = *out;
        *out = make_float4(o.x + s.x, o.y + s.y, o.z + s.z, o.w + s.w);
        return;
    }
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (e + i < count) acc[e + i] += v[i];
}

// ------------------------------------------------------------------------------------------
// Norms of short examples from the two Gram matrices of their tokens, T^2 (F + O) operations for 2 T F O:
//     |dW_i|^2 + |db_i|^2 = sum_{t, u} (dY_t . dY_u) (X_t . X_u + bias).
// A workgroup of four waves takes one pair of tiles of 64 tokens of one example (those above the diagonal once, counted twice), chunk by chunk of 128
// features: whole lines of memory into LDS, as bf16, the next chunk on its way; features both operands agree on need no order, so that
// operands are 16-byte reads of a token's row, and each wave takes a quarter of a chunk's features for the whole 64 x 64.  Bound by what a
// compute unit takes in, hence the tiles; where there are few pairs, several workgroups share a pair's features (splits) and
// ck_gram_join_kernel adds up their sums before it multiplies.
// fp32 dY: chunks of 64 features as they are, fp32 matrix instructions.  WORDS: as above.
//
// The terms have signs, and where they cancel the sum has lost its digits: tokens nearly alike whose dY add up to nothing (a key projection: a query's
// gradients of its scores add up to zero) can come out as 0, or less.  By Cauchy's inequality the terms add up to at most
//     B_i^2,   B_i = sum_t |dY_t| sqrt(|X_t|^2 + bias),
// which the diagonals hold, and every rounding is in proportion to it: with F / 4 or O / 4 additions in a row to an entry, the sum is off by
// (F + O) / 4 2^-23 B^2 if all err one way; 2^-23.9 B^2 is the most that was seen (2 to 500 tokens, 64 to 8192 features, tokens of their own to tokens all
// alike).  A sum stands if it is at least ck_resolution() of B^2: then it is within a quarter at worst, and within 2^-12 as measured.  Tokens of no common
// direction give B^2 / T.  The other examples' norms are made again from their gradients' values, on the device (ck_again_kernel).
// ONE: every example has one pair (64 tokens at most): half the operands, the products above the diagonal once, those of tokens from the 32nd on
// only where there are some, and three chunks on their way instead of one (32 x 64 tokens 768 -> 768 12.7 us and 11.3 before the bounds were summed
// here, 12.5 with them).  16 x 64 tokens 4096 -> 4096: 12.4, 8.5 to join; 400 x 64 768 -> 768: 17.2.
constexpr int GT = 64, GC = 128, G_ROW = 2 * GC + 16, G_SIDE = GT * G_ROW, G_STAGE = 2 * G_SIDE;      // tokens, features; bytes (16 of a row keep rows in different banks)
constexpr int G_VALUES = GT * GT;

// Whether value wave * 16 + q of lane `lane` is on the diagonal (of q's, one at most): four blocks of 32 x 32 one after the other, row
// (q >> 2) * 8 + (q & 3) + 4 (lane / 32) and column lane % 32 of a block.
__device__ __forceinline__ bool gram_diagonal(int wave, int q, int lane)
{
    return (wave == 0 || wave == 3) && (q >> 2) * 8 + (q & 3) + (lane >> 5) * 4 == (lane & 31);
}

// Sums of two values over a workgroup of NW waves, on thread 0.
template <int NW>
__device__ __forceinline__ float2 gram_sums(float v, float w, float (&red)[NW][2])
{
    v = wave_sum_last_lane(v);
    w = wave_sum_last_lane(w);
    if ((threadIdx.x & 63) == 63) { red[threadIdx.x >> 6][0] = v; red[threadIdx.x >> 6][1] = w; }
    __syncthreads();
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < NW; ++i) { s.x += red[i][0]; s.y += red[i][1]; }
    return s;
}

// bounds: [n, tiles of 64 tokens] shares of B_i; arrived: ck_again_kernel's counters, cleared for it
template <bool BF16, bool WORDS, bool ONE>
__global__ void __launch_bounds__(256, 2) ck_gram_kernel(const CkDenseArgs a, int pairs, int splits, float *tiles, float *bounds, unsigned *arrived)
{
    extern __shared__ __attribute__((aligned(16))) char ck_lds[];
    __shared__ float red[4][2];
    const unsigned whole = blockIdx.x / (unsigned)splits;          // example and pair
    const int split = (int)(blockIdx.x - whole * (unsigned)splits), ex = (int)(whole / (unsigned)pairs);
    int pair = (int)(whole - (unsigned)ex * (unsigned)pairs), tile_a = 0;
    if constexpr (!ONE)
        while (pair > tile_a) { ++tile_a; pair -= tile_a; }        // pairs (0,0) (1,0) (1,1) (2,0) ...
    const int tile_b = pair;
    const bool diagonal = ONE || tile_a == tile_b;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int len = __builtin_amdgcn_readfirstlane(ck_length(a, ex));
    if (t == 0 && pair == 0 && tile_a == 0 && split == 0) arrived[ex] = 0;
    float *const bound = bounds + (size_t)ex * (unsigned)((a.tokens + GT - 1) / GT) + tile_a;
    if (tile_a * GT >= len) {                                      // (tile_b is not the larger one)
        if (t == 0 && splits == 1) {
            a.partials[whole] = 0.0f;
            if (diagonal) *bound = 0.0f;
        }
        return;
    }
    const size_t row0 = (size_t)ex * (unsigned)a.tokens;
    const int s_pitch = a.pitch / CK_BLOCK;
    typedef typename In<BF16>::type E;
    constexpr int YC = BF16 ? GC : GC / 2, YV = YC / 16;           // features of a chunk of dY, of a piece (16 bytes)
    const uintptr_t y_at = reinterpret_cast<uintptr_t>(static_cast<const E *>(a.dy) + row0 * (unsigned)a.cout);
    const int odd = WORDS ? 0 : (int)(y_at >> 1) & 1;              // the first row begins in the middle of a dword
    // the example's tokens as buffers that end with its last one: those that are not there are zeros
    const __amdgpu_buffer_rsrc_t xb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.codes) + row0 * (unsigned)a.pitch, 0, len * a.pitch, 0x00020000);
    const __amdgpu_buffer_rsrc_t sb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.scales) + row0 * (unsigned)s_pitch, 0, len * s_pitch, 0x00020000);
    const int y_bytes = ((len * a.cout + odd) * (int)sizeof(E) + 3) & ~3;
    const __amdgpu_buffer_rsrc_t yb = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(y_at & ~(uintptr_t)3), 0, y_bytes, 0x00020000);
    // this workgroup's chunks, first those of X, then those of dY
    const int all_x = (a.pitch + GC - 1) / GC, all_y = (a.cout + YC - 1) / YC;
    const int x0 = all_x * split / splits, nx = all_x * (split + 1) / splits - x0, y0 = all_y * split / splits, ny = all_y * (split + 1) / splits - y0;
    const int xr = t >> 3, xp = t & 7, yr = t >> 4, yp = t & 15;   // pieces: 16 codes of rows xr + 32 u, YV values of dY of rows yr + 16 u

    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int SIDES = ONE ? 1 : 2, AHEAD = ONE ? 3 : 1;
    const int nx_up = (nx + AHEAD - 1) / AHEAD * AHEAD, all = nx_up + ny;          // chunk i: nx of X, none up to nx_up, then those of dY
    struct Held { uint4 v[SIDES][4]; };                            // a chunk on its way, X's scales, the dwords after dY's pieces
    struct Scale { uint32_t v[SIDES][2]; };                        // (one by one, not together, so that all of them are registers)
    struct More { uint32_t v[SIDES][WORDS ? 1 : 4]; };
    auto fetch = [&](Held &held, Scale &scale, More &more, int i) {
#pragma unroll
        for (int side = 0; side < SIDES; ++side) {
            if (side == 1 && diagonal) break;
            const int first = (side ? tile_b : tile_a) * GT;
            if (i < nx) {
                const int c = x0 + i;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int row = first + xr + 32 * u;
                    const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xb, row * a.pitch + xp * 16, c * GC, 0));
                    held.v[side][u] = make_uint4(v.x, v.y, v.z, v.w);
                    scale.v[side][u] = __builtin_amdgcn_raw_buffer_load_b8(sb, row * s_pitch + (xp >> 1), c * (GC / CK_BLOCK), 0);
                }
            } else if (i >= nx_up && i < all) {
                const int c = y0 + i - nx_up;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int row = first + yr + 16 * u;
                    unsigned at = (unsigned)(row * a.cout + yp * YV + odd) * (unsigned)sizeof(E) & ~3u;
                    if constexpr (!WORDS) at = row < len ? at : (unsigned)y_bytes;        // (the last value's dword may hold another)
                    const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(yb, at, c * YC * (int)sizeof(E), 0));
                    held.v[side][u] = make_uint4(v.x, v.y, v.z, v.w);
                    if constexpr (!WORDS) more.v[side][u] = __builtin_amdgcn_raw_buffer_load_b32(yb, at + 16u, c * YC * (int)sizeof(E), 0);
                }
            }
        }
    };
    auto stage = [&](const Held &held, const Scale &scale, const More &more, int i) {
#pragma unroll
        for (int side = 0; side < SIDES; ++side) {
            if (side == 1 && diagonal) break;
            char *to = ck_lds + (i & 1) * G_STAGE + side * G_SIDE;
            if (i < nx) {
                const bool there = (x0 + i) * GC + xp * 16 < a.pitch;      // (beyond: the next token's codes)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float f = pow2_of((int)scale.v[side][u]);
                    const uint4 c = there ? held.v[side][u] : make_uint4(0, 0, 0, 0);
                    const uint2 w0 = ck_bf16(c.x, f), w1 = ck_bf16(c.y, f), w2 = ck_bf16(c.z, f), w3 = ck_bf16(c.w, f);
                    uint4 *at = reinterpret_cast<uint4 *>(to + (xr + 32 * u) * G_ROW + xp * 32);
                    at[0] = make_uint4(w0.x, w0.y, w1.x, w1.y);
                    at[1] = make_uint4(w2.x, w2.y, w3.x, w3.y);
                }
            } else if (i >= nx_up && i < all) {
                const int left = a.cout - (y0 + i - nx_up) * YC - yp * YV;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    uint32_t w[4] = {held.v[side][u].x, held.v[side][u].y, held.v[side][u].z, held.v[side][u].w};
                    if constexpr (!WORDS) {                        // (an odd number of features: rows take turns)
                        const uint32_t bits = (uint32_t)((yr ^ odd) & 1) * 16u;
                        w[0] = funnel(w[1], w[0], bits); w[1] = funnel(w[2], w[1], bits); w[2] = funnel(w[3], w[2], bits); w[3] = funnel(more.v[side][u], w[3], bits);
                    }
                    if ((y0 + i - nx_up + 1) * YC > a.cout) mask_piece<BF16>(w, 0, left);       // beyond: the next token's values
                    *reinterpret_cast<uint4 *>(to + (yr + 16 * u) * G_ROW + yp * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
    };
    f32x16 gx[2][2], gy[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) gx[i][j][r] = gy[i][j][r] = 0.0f;
    auto products = [&](f32x16 (&g)[2][2], int buf) {
        const char *base_a = ck_lds + buf * G_STAGE + (lane & 31) * G_ROW + (lane >> 5) * 16 + wave * 64, *base_b = base_a + (diagonal ? 0 : G_SIDE);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            auto read = [&](const char *base, int i) { return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(base + i * 32 * G_ROW + ks * 32)); };
            const bf16x8 va = read(base_a, 0), vb = read(base_b, 0);
            g[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, vb, g[0][0], 0, 0, 0);
            if (!ONE || len > 32) {
                const bf16x8 wb = read(base_b, 1), wa = ONE ? wb : read(base_a, 1);
                g[0][1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, wb, g[0][1], 0, 0, 0);
                if (!ONE) g[1][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wa, vb, g[1][0], 0, 0, 0);
                g[1][1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wa, wb, g[1][1], 0, 0, 0);
            }
        }
    };
    // fp32 dY: a wave takes 16 of a chunk's 64 features, the halves of the wave eight each: a matrix instruction multiplies one of either half
    auto products_f32 = [&](int buf) {
        const char *base_a = ck_lds + buf * G_STAGE + (lane & 31) * G_ROW + (lane >> 5) * 32 + wave * 64, *base_b = base_a + (diagonal ? 0 : G_SIDE);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            auto read = [&](const char *base, int i) { return *reinterpret_cast<const float4 *>(base + i * 32 * G_ROW + q * 16); };
            auto step = [&](f32x16 &g, const float4 &a, const float4 &b) {
                g = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, b.x, g, 0, 0, 0);
                g = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, b.y, g, 0, 0, 0);
                g = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, b.z, g, 0, 0, 0);
                g = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, b.w, g, 0, 0, 0);
            };
            const float4 va = read(base_a, 0), vb = read(base_b, 0);
            step(gy[0][0], va, vb);
            if (!ONE || len > 32) {
                const float4 wb = read(base_b, 1), wa = ONE ? wb : read(base_a, 1);
                step(gy[0][1], va, wb);
                if (!ONE) step(gy[1][0], wa, vb);
                step(gy[1][1], wa, wb);
            }
        }
    };
    // chunk i is in LDS buffer i & 1, the AHEAD after it on their way
    auto after = [&](Held &held, Scale &scale, More &more, int i) {                             // chunk i + 1, and the next to be fetched there
        stage(held, scale, more, i + 1);
        fetch(held, scale, more, i + 1 + AHEAD);
        __syncthreads();
    };
    auto turn_x = [&](Held &held, Scale &scale, More &more, int i) {
        if (!ONE || i < nx) products(gx, i & 1);
        after(held, scale, more, i);
    };
    auto turn_y = [&](Held &held, Scale &scale, More &more, int i) {
        if constexpr (BF16) products(gy, i & 1);
        else products_f32(i & 1);
        after(held, scale, more, i);
    };
    Held h0, h1, h2;
    Scale c0, c1, c2;
    More m0, m1, m2;
    fetch(h0, c0, m0, 0);
    if constexpr (ONE) { fetch(h1, c1, m1, 1); fetch(h2, c2, m2, 2); }
    after(h0, c0, m0, -1);
    if constexpr (ONE) {
        for (int i = 0; i < nx_up; i += 3) { turn_x(h1, c1, m1, i); turn_x(h2, c2, m2, i + 1); turn_x(h0, c0, m0, i + 2); }
        for (int i = nx_up; i < all; i += 3) {
            turn_y(h1, c1, m1, i);
            if (i + 1 < all) turn_y(h2, c2, m2, i + 1);
            if (i + 2 < all) turn_y(h0, c0, m0, i + 2);
        }
    } else {
        for (int i = 0; i < nx; ++i) turn_x(h0, c0, m0, i);
        for (int i = nx; i < all; ++i) turn_y(h0, c0, m0, i);
    }

    // the waves' sums meet in LDS, in the order of the waves: a wave adds up sixteen of a lane's 64 values
    float *buf = reinterpret_cast<float *>(ck_lds);
    auto meet = [&](const f32x16 (&g)[2][2], float (&s)[16]) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) buf[(wave * 64 + (i * 2 + j) * 16 + r) * 64 + lane] = g[i][j][r];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            s[q] = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) s[q] += buf[(w * 64 + wave * 16 + q) * 64 + lane];
        }
        __syncthreads();
    };
    float sx[16], sy[16];
    meet(gx, sx);
    meet(gy, sy);
    if (splits > 1) {                                              // the other features' sums come first
        float *to = tiles + (size_t)blockIdx.x * 2 * G_VALUES + wave * 16 * 64 + lane;
#pragma unroll
        for (int q = 0; q < 16; ++q) { to[q * 64] = sx[q]; to[G_VALUES + q * 64] = sy[q]; }
        return;
    }
    float ss = 0.0f, own = 0.0f;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        const float p = (a.has_bias ? sx[q] + 1.0f : sx[q]) * sy[q];        // tokens that are not there: 0 dY . dY
        ss += p;
        own = gram_diagonal(wave, q, lane) ? p : own;
    }
    if (ONE && wave == 1) ss *= 2.0f;                              // a wave has one of the four blocks: block (0, 1), and (1, 0) is zeros
    const float2 sums = gram_sums<4>(ss, sqrtf(own), red);
    if (t == 0) {
        a.partials[whole] = diagonal ? sums.x : 2.0f * sums.x;
        if (diagonal) *bound = sums.y;
    }
}

// The products of a pair of tiles whose features several workgroups shared: their sums in order, then value by value.
__global__ void __launch_bounds__(512) ck_gram_join_kernel(const CkDenseArgs a, int pairs, int splits, const float *tiles, float *bounds)
{
    __shared__ float red[8][2];
    const int ex = (int)(blockIdx.x / (unsigned)pairs);
    int pair = (int)(blockIdx.x - (unsigned)ex * (unsigned)pairs), tile_a = 0;
    while (pair > tile_a) { ++tile_a; pair -= tile_a; }
    float ss = 0.0f, own = 0.0f;
    if (tile_a * GT < ck_length(a, ex)) {
        constexpr int values = G_VALUES;
        const float *p = tiles + (size_t)blockIdx.x * splits * 2 * values;
#pragma unroll 1
        for (int e = (int)threadIdx.x * 2; e < values; e += 1024) {
            float2 x = make_float2(0.0f, 0.0f), y = x;
#pragma unroll 4
            for (int k = 0; k < splits; ++k) {
                const float2 u = *reinterpret_cast<const float2 *>(p + (size_t)k * 2 * values + e), v = *reinterpret_cast<const float2 *>(p + (size_t)(2 * k + 1) * values + e);
                x.x += u.x; x.y += u.y; y.x += v.x; y.y += v.y;
            }
            if (a.has_bias) { x.x += 1.0f; x.y += 1.0f; }
            const float twice = pairs == 1 && e / (G_VALUES / 4) == 1 ? 2.0f : 1.0f;          // block (0, 1), and (1, 0) is zeros
            ss += twice * (x.x * y.x + x.y * y.y);
            const int wave = e >> 10, q = (e >> 6) & 15, lane = e & 63;
            if (gram_diagonal(wave, q, lane)) own += sqrtf(x.x * y.x);
            if (gram_diagonal(wave, q, lane + 1)) own += sqrtf(x.y * y.y);
        }
    }
    const float2 sums = gram_sums<8>(ss, own, red);
    if (threadIdx.x == 0) {
        a.partials[blockIdx.x] = tile_a == pair ? sums.x : 2.0f * sums.x;
        if (tile_a == pair) bounds[(size_t)ex * (unsigned)((a.tokens + GT - 1) / GT) + tile_a] = sums.y;
    }
}

// What the pairs of tiles of the examples left.
struct GramSums {
    const float *values, *bounds;    // [n, pairs], [n, tiles of 64 tokens]
    int pairs, tiles;
    float resolution;
    // example i's sum and the root of its bound
    __device__ __forceinline__ void load(int i, float &sum, float &bound) const
    {
        const float *v = values + (size_t)i * pairs, *b = bounds + (size_t)i * tiles;
        sum = bound = 0.0f;
#pragma unroll 4
        for (int k = 0; k < pairs; ++k) sum += v[k];
#pragma unroll 4
        for (int k = 0; k < tiles; ++k) bound += b[k];
    }
    __device__ __forceinline__ bool stands(float sum, float bound) const { return sum >= resolution * bound * bound; }        // (not: a NaN)
};

// Squared norms of the examples whose sums do not stand, from their gradients' values, dW_i and db_i as one product with a further feature of X that
// is 1.  `sharers` workgroups take an example's tiles of 64 x 64 in turn, a wave 32 x 32 of one, chunks of 32 tokens through LDS as [feature][token]; the
// last one to arrive adds up what they leave, in order.  Every workgroup walks over all examples, AGAIN_TURNS to a thread at a time; as many examples at
// once as fill the chip.  The first workgroup writes the norms that stand.  Small and with few registers, so that it costs little where there is nothing to
// do: a launch of 3.4 us (the contraction in its place: 20, for its registers in a loop).  Where all fall: 16 examples of 64 tokens 4096 -> 4096
// 529 us, the contraction 57; 512 of 8 tokens 768 -> 768 303 and 49.
constexpr int AGAIN = 64, AGAIN_TOKENS = 32, AGAIN_ROW = AGAIN_TOKENS * 2 + 16;        // features of a tile, tokens of a chunk; bytes (16 more: banks, alignment)

template <bool BF16, int AGAIN_TURNS>
__global__ void __launch_bounds__(256) ck_again_kernel(const CkDenseArgs a, const GramSums g, int sharers, unsigned *arrived, float *sqnorm)
{
    typedef typename In<BF16>::type E;
    constexpr int PLANES = BF16 ? 1 : 3;
    __shared__ __attribute__((aligned(16))) char xs[AGAIN * AGAIN_ROW], ys[PLANES][AGAIN * AGAIN_ROW];
    __shared__ uint32_t fallen[8 * AGAIN_TURNS];
    __shared__ float red[4];
    __shared__ unsigned before;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const unsigned at_once = gridDim.x / (unsigned)sharers, mine = blockIdx.x / (unsigned)sharers;
    const int sharer = (int)(blockIdx.x - mine * (unsigned)sharers);
    const int features = a.cin + a.has_bias, s_pitch = a.pitch / CK_BLOCK;

    auto squares = [&](int ex, int tile_o, int tile_k) {           // of a tile's values, this lane's share
        const int o0 = tile_o * AGAIN, k0 = tile_k * AGAIN, len = ck_length(a, ex);
        const size_t row0 = (size_t)ex * (unsigned)a.tokens;
        f32x16 acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
        for (int c = 0; c < len; c += AGAIN_TOKENS) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < AGAIN_TOKENS / 16; ++u) {          // token (t / 16) + 16 u, features 4 (t % 16) .. of either operand
                const int token = (t >> 4) + 16 * u, f = 4 * (t & 15), k = k0 + f, o = o0 + f;
                const bool there = c + token < len;
                const size_t row = row0 + (unsigned)(c + token);
                uint2 x = make_uint2(0, 0);
                if (there && k < a.pitch)
                    x = ck_bf16(*reinterpret_cast<const uint32_t *>(a.codes + row * (unsigned)a.pitch + k), pow2_of(a.scales[row * (unsigned)s_pitch + k / CK_BLOCK]));
                uint16_t xv[4] = {(uint16_t)x.x, (uint16_t)(x.x >> 16), (uint16_t)x.y, (uint16_t)(x.y >> 16)};
                char *to = xs + f * AGAIN_ROW + token * 2;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (k + i == a.cin && a.has_bias) xv[i] = there ? 0x3F80 : 0;
                    *reinterpret_cast<uint16_t *>(to + i * AGAIN_ROW) = xv[i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    E v = 0;
                    if (there && o + i < a.cout) v = static_cast<const E *>(a.dy)[row * (unsigned)a.cout + o + i];
                    to = &ys[0][(f + i) * AGAIN_ROW + token * 2];
                    if constexpr (BF16) {
                        *reinterpret_cast<uint16_t *>(to) = v;
                    } else {
                        float rest = v;
#pragma unroll
                        for (int q = 0; q < 3; ++q) {              // (split8)
                            const uint32_t w = pack_bf16(rest, 0.0f);
                            rest -= __uint_as_float(w << 16);
                            *reinterpret_cast<uint16_t *>(to + q * AGAIN * AGAIN_ROW) = (uint16_t)w;
                        }
                    }
                }
            }
            __syncthreads();
#pragma unroll
            for (int ks = 0; ks < AGAIN_TOKENS / 16; ++ks) {
                const int in_row = (lane & 31) * AGAIN_ROW + (lane >> 5) * 16 + ks * 32;
                const bf16x8 b = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(xs + (wave & 1) * 32 * AGAIN_ROW + in_row));
#pragma unroll
                for (int q = 0; q < PLANES; ++q) {
                    const bf16x8 y = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(&ys[q][(wave >> 1) * 32 * AGAIN_ROW + in_row]));
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, b, acc, 0, 0, 0);
                }
            }
        }
        float ss = 0.0f;                                           // (features beyond the last are zeros)
#pragma unroll
        for (int r = 0; r < 16; ++r) ss = fmaf(acc[r], acc[r], ss);
        return ss;
    };

    unsigned turn = 0;
    for (int first = 0; first < a.n; first += 256 * AGAIN_TURNS) {
        float sum[AGAIN_TURNS], bound[AGAIN_TURNS];
        unsigned long long those[AGAIN_TURNS];
#pragma unroll
        for (int u = 0; u < AGAIN_TURNS; ++u) sum[u] = bound[u] = 0.0f;
        if (g.pairs == 1) {                                        // all loads at once
#pragma unroll
            for (int u = 0; u < AGAIN_TURNS; ++u)
                if (first + 256 * u + t < a.n) { sum[u] = g.values[first + 256 * u + t]; bound[u] = g.bounds[first + 256 * u + t]; }
        } else {
#pragma unroll
            for (int u = 0; u < AGAIN_TURNS; ++u)
                if (first + 256 * u + t < a.n) g.load(first + 256 * u + t, sum[u], bound[u]);
        }
        bool any = false;
#pragma unroll
        for (int u = 0; u < AGAIN_TURNS; ++u) {
            const bool stands = g.stands(sum[u], bound[u]);
            if (blockIdx.x == 0 && stands && first + 256 * u + t < a.n) sqnorm[first + 256 * u + t] = sum[u];
            those[u] = __ballot(!stands);
            any |= !stands;
        }
        if (!__syncthreads_or(any)) continue;                      // (the last ones have been read, too)
#pragma unroll
        for (int u = 0; u < AGAIN_TURNS; ++u)
            if (lane == 0) {
                fallen[8 * u + 2 * wave] = (uint32_t)those[u];
                fallen[8 * u + 2 * wave + 1] = (uint32_t)(those[u] >> 32);
            }
        __syncthreads();
        for (int w = 0; w < 8 * AGAIN_TURNS; ++w)
            for (uint32_t left = (uint32_t)__builtin_amdgcn_readfirstlane((int)fallen[w]); left; left &= left - 1) {
                if (turn++ % at_once != mine) continue;
                const int ex = first + 32 * w + __builtin_ctz(left), tiles_k = (features + AGAIN - 1) / AGAIN, tiles = (a.cout + AGAIN - 1) / AGAIN * tiles_k;
                float ss = 0.0f;
                for (int tile = sharer; tile < tiles; tile += sharers) ss += squares(ex, tile / tiles_k, tile % tiles_k);
                const float tot = block_sum<4>(ss, red);
                float *const part = a.partials + (size_t)ex * sharers;
                if (t == 0) {
                    __hip_atomic_store(part + sharer, tot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    before = __hip_atomic_fetch_add(arrived + ex, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
                }
                __syncthreads();
                if (before + 1 == (unsigned)sharers) {             // all of them are there
                    const float v = t < sharers ? __hip_atomic_load(part + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0f;
                    const float sum = block_sum<4>(v, red);
                    if (t == 0) sqnorm[ex] = sum;
                }
            }
    }
}

// ---- plans --------------------------------------------------------------------------------

struct CkPlan {
    bool gram;
    int gram_splits;                 // workgroups that share a pair's features
    size_t per_example;              // partial squared norms
    int sharers;                     // workgroups of an example whose norm is made again
    int nj;                          // the contraction's tiles are 64 nj wide
    int ranges, chunks;              // weighted
    bool rows;
};

int ck_tiles(int v, int width) { return (v + width - 1) / width; }

// What a sum of the Gram form has to be of its bound (ck_gram_kernel).
float ck_resolution(const Geo &g) { return std::max(0x1p-11f, (float)(g.cin + g.cout) * 0x1p-23f); }

// Which of the two forms of norms: what they take, in microseconds a call.  bf16 (n, T, F, O: Gram form / contraction): 32, 64, 768, 768 15.0 / 9.9, with a
// bias 15.1 / 9.8; 400, 64, 768, 768 20.2 / 50.9; 8, 128, 2048, 2048 22.5 / 14.3; 16, 64, 2048, 2048 18.9 / 17.4; 64, 16, 2048, 2048 21.2 / 43.4;
// 8, 512, 2048, 2048 50.3 / 36.2; 16, 64, 4096, 4096 22.3 / 56.6; 16, 128, 4096, 4096 28.9 / 79.3; 16, 256, 4096, 4096 48.6 / 137.  fp32: 32, 64, 768, 768 21.6 / 14.8;
// 16, 64, 2048, 2048 24.6 / 36.2; 55, 2, 1792, 576 20.3 / 24.8; 16, 256, 4096, 4096 90.4 / 396.  512 workgroups of either kind fill the chip.
double gram_us(const Geo &g, double pairs, int splits, double chunks)
{
    const double groups = g.n * pairs * splits;
    const double chunk_us = pairs > 1.0 ? (g.bf16 ? 1.4 : 2.3) : groups <= 256.0 ? (g.bf16 ? 0.55 : g.h <= 32 ? 0.5 : 0.8) : (g.bf16 ? 1.0 : 1.65);
    return (pairs > 1.0 ? 9.0 : 10.0) + std::max(1.0, groups / 512.0) * chunk_us * chunks / splits + (splits > 1 ? 4.5 + groups / 85.0 : 0.0);
}
double contract_us(const Geo &g, double tiles, int chunk)
{
    return 5.5 + std::max(1.0, g.n * tiles / 512.0) * ((g.bf16 ? 1.5 : 1.15) + (g.bf16 ? 0.85 : 1.37) * ((g.h + chunk - 1) / chunk));
}

CkPlan ck_plan(const Geo &g, int mode)
{
    CkPlan p = {};
    const int tiles_o = ck_tiles(g.cout, CT);
    p.nj = 2;
    if (mode == MODE_WEIGHTED) {
        // 32 rows hold several examples of a few tokens each, at three products for one
        p.rows = !g.bf16 || g.h < 16;
        if (!p.rows && (long long)tiles_o * ck_tiles(g.cin, 256) >= 384) p.nj = 4;
        const int chunk = ck_chunk(p.rows ? 3 : 1, p.nj);
        const long long chunks = p.rows ? ((long long)g.n * g.h + chunk - 1) / chunk : (long long)std::min(g.n, CK_TABLE) * ((g.h + chunk - 1) / chunk);
        p.chunks = (int)chunks;
        // Ranges of the call's chunks: fewer chunks in a row against more sums to write and join.  What R of them take, in microseconds, fitted
        // to 16 x 128 tokens 768 -> 768 (R 1: 36, 3: 22.5, 6: 19.4, 16: 27), 16 x 512 2048 -> 2048 (1: 124, 2: 101, 4: 111, 8: 145) and
        // 64 x 64 512 -> 512 (1: 68, 4: 28, 16: 19): 9 at least, a chunk 0.85 where a workgroup has a compute unit to itself and 1.2 where two
        // share it (three products for one: 1.15 and 1.6), a value of a range's sums written and read at 4.5 TB/s.
        const double tiles = (double)tiles_o * ck_tiles(g.cin, 64 * p.nj), sums = 8.0 * g.pw / 4.5e6, one = p.rows ? 1.15 : 0.85, two = p.rows ? 1.6 : 1.2;
        double best = 0.0;
        for (int r = 1; r <= 64 && (r == 1 || r <= chunks / 2); ++r) {
            const double groups = tiles * r, chunk_us = groups <= 256.0 ? one : std::min(two, one + (two - one) * (groups - 256.0) / 256.0) * std::max(1.0, groups / 512.0);
            const double us = 9.0 + chunk_us * std::ceil((double)chunks / r) + (r > 1 ? sums * r : 0.0);
            if (r == 1 || us < best) { best = us; p.ranges = r; }
        }
        return p;
    }
    if (g.bf16 && (long long)g.n * tiles_o * ck_tiles(g.cin, 256) >= 384) p.nj = 4;
    const int tiles_k = ck_tiles(g.cin, 64 * p.nj);
    p.per_example = (size_t)tiles_o * (tiles_k + g.has_bias);
    if (mode == MODE_NORM && (long long)g.h * std::max(ck_pitch(g.cin), g.cout * (g.bf16 ? 2 : 4)) < (1ll << 31)) {        // (offsets of an example's values: 32 bits)
        const int yc = g.bf16 ? GC : GC / 2;
        const long long tiles = (g.h + GT - 1) / GT, pairs = tiles * (tiles + 1) / 2, chunks = (ck_pitch(g.cin) + GC - 1) / GC + (g.cout + yc - 1) / yc;
        p.gram_splits = (int)std::max(1ll, std::min({512 / (g.n * pairs), chunks / 8, 16ll}));
        // (tokens of no common direction have a sum of 1 / T of its bound: they stand with room for four times less)
        p.gram = g.n * pairs < (long long)CK_GROUPS && (double)g.h * ck_resolution(g) <= 0.25 &&
                 gram_us(g, (double)pairs, p.gram_splits, (double)chunks) < contract_us(g, (double)p.per_example, ck_chunk(g.bf16 ? 1 : 3, p.nj));
        if (p.gram) {
            p.per_example = (size_t)pairs;
            // (an example's workgroups meet on a counter, as long as a few tiles take: 16 tiles or more to each)
            p.sharers = (int)std::min(256ll, ((long long)ck_tiles(g.cin + g.has_bias, AGAIN) * ck_tiles(g.cout, AGAIN) + 15) / 16);
        }
    }
    return p;
}

template <int PLANES, int NJ, bool WEIGHTED, bool BF16>
dp_status run_contract(bool words, dim3 grid, const CkDenseArgs &a, hipStream_t s)
{
    constexpr unsigned lds = 2 * ck_stage_bytes(PLANES, NJ);
    if constexpr (BF16)
        if (!words) return launch_lds<ck_contract_kernel<PLANES, NJ, WEIGHTED, BF16, false>>(grid, 256, lds, s, a);
    return launch_lds<ck_contract_kernel<PLANES, NJ, WEIGHTED, BF16, true>>(grid, 256, lds, s, a);
}

size_t align16(size_t b) { return (b + 15) & ~(size_t)15; }
size_t align4(size_t v) { return (v + 3) & ~(size_t)3; }

}  // namespace

// Places in the workspace of norms by the Gram form, one after the other.
struct GramRoom { size_t bounds, partials, arrived, tiles, bytes; };
static GramRoom gram_room(const Geo &g, const CkPlan &p)
{
    const size_t n = (size_t)g.n;
    GramRoom r;
    r.bounds = align16(4 * n * p.per_example);                     // behind the pairs' sums
    r.partials = r.bounds + align16(4 * n * ((g.h + GT - 1) / GT));
    r.arrived = r.partials + align16(4 * n * p.sharers);
    r.tiles = r.arrived + align16(4 * n);
    r.bytes = r.tiles + (p.gram_splits > 1 ? n * p.per_example * p.gram_splits * 2 * G_VALUES * 4 : 0);
    return r;
}

// A weighted call goes in launches of CK_TABLE examples and one of those that are left, which plan their own ranges; ranges do not grow
// steadily with the chunks (645 examples of 64 tokens, 768 -> 768, take 15, 1024 of them 14): room for the most.
static size_t weighted_ws_bytes(const Geo &g)
{
    const CkPlan p = ck_plan(g, MODE_WEIGHTED);
    int most = p.ranges;
    if (!p.rows && g.n > CK_TABLE && g.n % CK_TABLE) {
        Geo rest = g;
        rest.n = g.n % CK_TABLE;
        most = std::max(most, ck_plan(rest, MODE_WEIGHTED).ranges);
    }
    return most > 1 ? 4 * (size_t)most * (align4(g.pw) + align4(g.pb)) : 0;
}

size_t checkpoint_ws_bytes(const Geo &g, int mode)
{
    if (mode == MODE_WEIGHTED) return weighted_ws_bytes(g);
    // both per-example forms: a caller sizes its workspace once
    const CkPlan p = ck_plan(g, MODE_NORM), q = ck_plan(g, MODE_MATERIALISE);
    return std::max(align16(4 * (size_t)g.n * q.per_example), p.gram ? gram_room(g, p).bytes : 0);
}

template <bool ONE>
static dp_status run_gram(bool bf16, bool words, dim3 grid, const CkDenseArgs &a, int pairs, int splits, float *tiles, float *bounds, unsigned *arrived,
                          hipStream_t s)
{
    if (!bf16) return launch_lds<ck_gram_kernel<false, true, ONE>>(grid, 256, 2 * G_STAGE, s, a, pairs, splits, tiles, bounds, arrived);
    if (!words) return launch_lds<ck_gram_kernel<true, false, ONE>>(grid, 256, 2 * G_STAGE, s, a, pairs, splits, tiles, bounds, arrived);
    return launch_lds<ck_gram_kernel<true, true, ONE>>(grid, 256, 2 * G_STAGE, s, a, pairs, splits, tiles, bounds, arrived);
}

static dp_status launch_gram(const Geo &g, const CkPlan &p, CkDenseArgs a, bool words, float *sqnorm, void *ws, hipStream_t s)
{
    const GramRoom room = gram_room(g, p);
    char *const base = static_cast<char *>(ws);
    float *const values = reinterpret_cast<float *>(base), *const bounds = reinterpret_cast<float *>(base + room.bounds);
    float *const tiles = reinterpret_cast<float *>(base + room.tiles);
    unsigned *const arrived = reinterpret_cast<unsigned *>(base + room.arrived);
    const int pairs = (int)p.per_example;
    const dim3 joins((unsigned)(g.n * p.per_example)), blocks(joins.x * (unsigned)p.gram_splits);
    a.partials = values;
    profile_begin(s);
    dp_status st = pairs == 1 ? run_gram<true>(g.bf16, words, blocks, a, pairs, p.gram_splits, tiles, bounds, arrived, s)
                              : run_gram<false>(g.bf16, words, blocks, a, pairs, p.gram_splits, tiles, bounds, arrived, s);
    if (st == DP_OK && p.gram_splits > 1) st = launch_lds<ck_gram_join_kernel>(joins, 512, 0, s, a, pairs, p.gram_splits, tiles, bounds);
    profile_end(s);
    if (st != DP_OK) return st;
    const GramSums sums = {values, bounds, pairs, (g.h + GT - 1) / GT, ck_resolution(g)};
    a.partials = reinterpret_cast<float *>(base + room.partials);
    const dim3 again((unsigned)(p.sharers * std::min(std::max(512 / p.sharers, 1), g.n)));
    // one example to a thread, or eight (16 x 64 tokens 4096 -> 4096: 22.4 us a call and 23.3; 400 x 64 768 -> 768 21.0 and 20.2; 65535 x 1
    // 256 -> 256 1227 and 938)
    if (g.n <= 256) return g.bf16 ? launch_lds<ck_again_kernel<true, 1>>(again, 256, 0, s, a, sums, p.sharers, arrived, sqnorm)
                                  : launch_lds<ck_again_kernel<false, 1>>(again, 256, 0, s, a, sums, p.sharers, arrived, sqnorm);
    return g.bf16 ? launch_lds<ck_again_kernel<true, 8>>(again, 256, 0, s, a, sums, p.sharers, arrived, sqnorm)
                  : launch_lds<ck_again_kernel<false, 8>>(again, 256, 0, s, a, sums, p.sharers, arrived, sqnorm);
}

static dp_status launch_weighted(const Geo &g, CkDenseArgs a, float *out_w, float *out_b, void *ws, hipStream_t s)
{
    const CkPlan p = ck_plan(g, MODE_WEIGHTED);
    a.tiles_k = ck_tiles(g.cin, 64 * p.nj); a.columns = a.tiles_k + g.has_bias;
    a.chunks = p.chunks; a.slots = p.ranges;
    a.add = p.ranges == 1;
    a.out_w = out_w; a.out_b = out_b;
    if (p.ranges > 1) {
        a.out_w = static_cast<float *>(ws);
        a.out_b = a.out_w + align4(g.pw);
        a.stride_w = a.stride_b = align4(g.pw) + align4(g.pb);
    }
    const bool words = !g.bf16 || g.cout % 2 == 0;
    const dim3 grid((unsigned)(((size_t)a.tiles_o * a.columns * p.ranges + 7) / 8 * 8));
    dp_status st;
    profile_begin(s);
    if (!p.rows) st = p.nj == 4 ? run_contract<1, 4, true, true>(words, grid, a, s) : run_contract<1, 2, true, true>(words, grid, a, s);
    else st = g.bf16 ? run_contract<3, 2, true, true>(words, grid, a, s) : run_contract<3, 2, true, false>(words, grid, a, s);
    profile_end(s);
    if (st != DP_OK || p.ranges == 1) return st;
    const size_t groups = (align4(g.pw) + align4(g.pb)) / 4;
    hipLaunchKernelGGL(ck_ranges_kernel, dim3((unsigned)((groups + 255) / 256)), dim3(256), 0, s, a.out_w, a.stride_w, align4(g.pw), p.ranges, g.pw, g.pb, out_w, out_b);
    return check_launch("checkpoint_ranges");
}

dp_status launch_checkpoint_dense(const Geo &g, int mode, const uint8_t *codes, const uint8_t *scales, const void *dy, const int32_t *lengths,
                                  float *out_w, float *out_b, size_t out_stride, float *sqnorm, const float *group_sqnorm, float clip_c,
                                  void *ws, hipStream_t s)
{
    const CkPlan p = ck_plan(g, mode);
    CkDenseArgs a = {};
    a.codes = codes; a.scales = scales; a.dy = dy; a.lengths = lengths;
    a.n = g.n; a.tokens = g.h; a.cin = g.cin; a.cout = g.cout; a.pitch = ck_pitch(g.cin);
    a.has_bias = g.has_bias;
    a.tiles_o = ck_tiles(g.cout, CT);
    if (mode == MODE_WEIGHTED) {
        a.group_sqnorm = group_sqnorm; a.clip_c = clip_c;
        if (p.rows) return launch_weighted(g, a, out_w, out_b, ws, s);
        // as many examples to a launch as the kernel's table has room for
        for (int i = 0; i < g.n; i += CK_TABLE) {
            Geo part = g;
            part.n = a.n = std::min(g.n - i, CK_TABLE);
            const dp_status st = launch_weighted(part, a, out_w, out_b, ws, s);
            if (st != DP_OK) return st;
            const size_t rows = (size_t)a.n * g.h;
            a.codes += rows * a.pitch;
            a.scales += rows * (a.pitch / CK_BLOCK);
            a.dy = static_cast<const uint16_t *>(a.dy) + rows * g.cout;
            if (a.lengths) a.lengths += a.n;
            a.group_sqnorm += a.n;
        }
        return DP_OK;
    }
    a.tiles_k = ck_tiles(g.cin, 64 * p.nj); a.columns = a.tiles_k + g.has_bias;
    const bool words = !g.bf16 || g.cout % 2 == 0;
    if (p.gram) return launch_gram(g, p, a, words, sqnorm, ws, s);
    dp_status st = DP_OK;
    const bool alone = p.per_example == 1 && sqnorm;               // an example's only partial sum is its squared norm
    a.partials = alone ? sqnorm : static_cast<float *>(ws);
    a.stored = out_w != nullptr;
    a.out_w = out_w; a.out_b = out_b;
    a.stride_w = out_stride ? out_stride : g.pw;
    a.stride_b = out_stride ? out_stride : g.pb;
    const float *const partials = a.partials;
    const int at_once = (int)std::max<size_t>(1, CK_GROUPS / p.per_example);       // examples of a launch
    profile_begin(s);
    for (int i = 0; i < g.n && st == DP_OK; i += at_once) {
        a.slots = std::min(g.n - i, at_once);
        // workgroups of all XCDs alike (the kernel's map), those beyond the last one end at once
        const dim3 grid((unsigned)((p.per_example * a.slots + 7) / 8 * 8));
        if (g.bf16) {
            st = p.nj == 4 ? run_contract<1, 4, false, true>(words, grid, a, s) : run_contract<1, 2, false, true>(words, grid, a, s);
        } else {
            st = run_contract<3, 2, false, false>(words, grid, a, s);
        }
        const size_t rows = (size_t)a.slots * g.h;
        a.codes += rows * a.pitch;
        a.scales += rows * (a.pitch / CK_BLOCK);
        a.dy = static_cast<const char *>(a.dy) + rows * g.cout * (g.bf16 ? 2 : 4);
        if (a.lengths) a.lengths += a.slots;
        a.partials += p.per_example * a.slots;
        if (a.out_w) a.out_w += a.stride_w * a.slots;
        if (a.out_b) a.out_b += a.stride_b * a.slots;
    }
    profile_end(s);
    if (st != DP_OK || !sqnorm || alone) return st;
    return launch_sum_partials(partials, g.n, (int)p.per_example, sqnorm, s);
}

}  // namespace dp
