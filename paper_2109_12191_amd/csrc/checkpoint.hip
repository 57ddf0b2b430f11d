// Activation checkpoints in 8 bits: what a layer saw in the forward pass, kept for the privatising backward pass in a little over a
// byte a value.
//
// A block is 32 consecutive features of one token.  With a the largest finite magnitude in it, its scale is the smallest power of
// two s with a <= 448 s, and a value x is kept as the e4m3 number nearest to x / s (ties to even): relative error at most 2^-4, or
// half of 2^-9 s in absolute terms.  Powers of two because x / s and code * s are then exact: the only rounding is the code's, and
// the contractions read the checkpoint as bf16 operands without another one.  Features, not tokens, share a scale, so that a token
// can be written by itself.
//
// Both kernels are bound by memory: a lane takes 16 bytes of activations, eight bf16 or four fp32 features, and its neighbours the next ones, so
// that either side of a wave's access is one run of whole lines; 4 or 8 neighbouring lanes hold a block.  (16 features to a lane: fp32
// stores 64 bytes apart, 6000 x 1003 read as fp32 in 11.6 us instead of 7.2.)  Every code of a row's pitch is written: the places after the
// last feature hold zeros.  32768 x 2048 bf16 written in 37 us, 5.5 TB/s in and out; a copy of 1 GiB runs at 5.2.
#include "checkpoint.h"

namespace dp {

namespace {

struct CkArgs {
    const void *x;
    void *out;
    uint8_t *codes, *scales;
    const uint8_t *codes_in, *scales_in;
    size_t rows, stride, pieces;     // pieces of V features of all rows
    int features, per_row;           // pieces of a row (whole blocks of them)
    size_t first_block;              // workgroups of the launches before
};

template <bool BF16> constexpr int ck_values() { return BF16 ? 8 : 4; }
constexpr int CK_TURNS = 2;                                        // pieces of a thread, a workgroup's width apart

// Row and piece of this thread's turn u.  One 64-bit division per workgroup (scalar), a 32-bit one per piece.
__device__ __forceinline__ bool ck_place(const CkArgs &a, int u, size_t &row, int &piece)
{
    const size_t first = (a.first_block + blockIdx.x) * (256 * CK_TURNS), row0 = first / (unsigned)a.per_row;
    const unsigned at = (unsigned)(first - row0 * (unsigned)a.per_row) + 256u * u + threadIdx.x, more = at / (unsigned)a.per_row;
    row = row0 + more;
    piece = (int)(at - more * (unsigned)a.per_row);
    return first + 256u * u + threadIdx.x < a.pieces;
}

__device__ __forceinline__ void load_piece(const uint16_t *p, int count, float (&v)[8]) { widen8(load8(p, count), v); }
__device__ __forceinline__ void load_piece(const float *p, int count, float (&v)[4])
{
    if (count >= 4) {
        const u32x4_a4 a = *reinterpret_cast<const u32x4_a4 *>(p);
        v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < count ? p[i] : 0.0f;
}

template <bool BF16>
__global__ void __launch_bounds__(256) checkpoint_write_kernel(const CkArgs a)
{
    typedef typename In<BF16>::type E;
    constexpr int V = ck_values<BF16>();
    size_t row[CK_TURNS];
    int piece[CK_TURNS];
    bool there[CK_TURNS];
    float v[CK_TURNS][V];
#pragma unroll
    for (int u = 0; u < CK_TURNS; ++u) {
        there[u] = ck_place(a, u, row[u], piece[u]);
        load_piece(static_cast<const E *>(a.x) + row[u] * a.stride + piece[u] * V, there[u] ? a.features - piece[u] * V : 0, v[u]);
    }
#pragma unroll
    for (int u = 0; u < CK_TURNS; ++u) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(v[u][i]) & 0x7FFFFFFFu);
        const bool broken = top >= 0x7F800000u;                    // an infinity or a NaN: no part in the scale, kept as NaN
        if (broken) {
            top = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t m = __float_as_uint(v[u][i]) & 0x7FFFFFFFu;
                top = max(top, m < 0x7F800000u ? m : 0u);
            }
        }
        // the block's other lanes: lane ^ 1, lane ^ 2 and, of eight, the other four
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true));
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, true));
        if constexpr (!BF16) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x141, 0xf, 0xf, true));
        // 448 = 1.75 * 2^8
        const int e = min(max((int)(top >> 23) - 135 + ((top & 0x7FFFFFu) > 0x600000u), CK_LOW), CK_HIGH);
        const float inv = pow2_of(127 - e);
        uint32_t w[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            float q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = __builtin_amdgcn_fmed3f(v[u][4 * i + j] * inv, -448.0f, 448.0f);
            int packed = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
            packed = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], packed, true);
            w[i] = (uint32_t)packed;
        }
        if (broken) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if ((__float_as_uint(v[u][i]) & 0x7FFFFFFFu) >= 0x7F800000u)
                    w[i >> 2] = (w[i >> 2] & ~(0xFFu << (8 * (i & 3)))) | (0x7Fu << (8 * (i & 3)));
        }
        if (there[u]) {
            const size_t at = row[u] * (unsigned)a.per_row + piece[u];
            if constexpr (BF16) reinterpret_cast<uint2 *>(a.codes)[at] = make_uint2(w[0], w[1]);
            else reinterpret_cast<uint32_t *>(a.codes)[at] = w[0];
            if (piece[u] % (CK_BLOCK / V) == 0) a.scales[at / (CK_BLOCK / V)] = (uint8_t)(e + 127);
        }
    }
}

template <bool BF16>
__global__ void __launch_bounds__(256) checkpoint_read_kernel(const CkArgs a)
{
    typedef typename In<BF16>::type E;
    constexpr int V = ck_values<BF16>();
    E *out[CK_TURNS];
    int count[CK_TURNS];
    uint32_t codes[CK_TURNS][V / 4], scale[CK_TURNS];
#pragma unroll
    for (int u = 0; u < CK_TURNS; ++u) {
        size_t row;
        int piece;
        const bool there = ck_place(a, u, row, piece);
        count[u] = there ? a.features - piece * V : 0;             // (none: after the last feature)
        out[u] = static_cast<E *>(a.out) + row * a.stride + piece * V;
        scale[u] = 127;
#pragma unroll
        for (int i = 0; i < V / 4; ++i) codes[u][i] = 0;
        if (count[u] > 0) {
            const size_t at = row * (unsigned)a.per_row + piece;
            if constexpr (BF16) {
                const uint2 c = reinterpret_cast<const uint2 *>(a.codes_in)[at];
                codes[u][0] = c.x; codes[u][1] = c.y;
            } else {
                codes[u][0] = reinterpret_cast<const uint32_t *>(a.codes_in)[at];
            }
            scale[u] = a.scales_in[at / (CK_BLOCK / V)];
        }
    }
#pragma unroll
    for (int u = 0; u < CK_TURNS; ++u) {
        if (count[u] <= 0) continue;
        const float s = pow2_of((int)scale[u]);
        float v[V];
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const uint2 d = ck_bf16(codes[u][i], s);
            v[4 * i] = __uint_as_float(d.x << 16); v[4 * i + 1] = __uint_as_float(d.x & 0xFFFF0000u);
            v[4 * i + 2] = __uint_as_float(d.y << 16); v[4 * i + 3] = __uint_as_float(d.y & 0xFFFF0000u);
        }
        if constexpr (BF16) {
            store8(out[u], count[u], v);                           // (rounds nothing: the values are bf16 numbers)
        } else if (count[u] >= 4) {
            *reinterpret_cast<u32x4_a4 *>(out[u]) = u32x4_a4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count[u]) out[u][i] = v[i];
        }
    }
}

CkArgs ck_args(size_t rows, int features, size_t stride, bool bf16)
{
    CkArgs a = {};
    a.rows = rows;
    a.stride = stride;
    a.features = features;
    a.per_row = ck_pitch(features) / (bf16 ? ck_values<true>() : ck_values<false>());
    a.pieces = rows * (size_t)a.per_row;
    return a;
}

}  // namespace

dp_status launch_checkpoint_write(const void *x, bool bf16, size_t rows, int features, size_t stride, uint8_t *codes, uint8_t *scales,
                                  hipStream_t s)
{
    CkArgs a = ck_args(rows, features, stride, bf16);
    a.x = x; a.codes = codes; a.scales = scales;
    const size_t grid = (a.pieces + 256 * CK_TURNS - 1) / (256 * CK_TURNS);
    return bf16 ? launch_blocks<checkpoint_write_kernel<true>>(grid, 256, 0, s, a) : launch_blocks<checkpoint_write_kernel<false>>(grid, 256, 0, s, a);
}

dp_status launch_checkpoint_read(const uint8_t *codes, const uint8_t *scales, bool bf16, size_t rows, int features, void *x, size_t stride,
                                 hipStream_t s)
{
    CkArgs a = ck_args(rows, features, stride, bf16);
    a.out = x; a.codes_in = codes; a.scales_in = scales;
    const size_t grid = (a.pieces + 256 * CK_TURNS - 1) / (256 * CK_TURNS);
    return bf16 ? launch_blocks<checkpoint_read_kernel<true>>(grid, 256, 0, s, a) : launch_blocks<checkpoint_read_kernel<false>>(grid, 256, 0, s, a);
}

}  // namespace dp
