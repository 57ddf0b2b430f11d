// Activation checkpoints in 8 bits: what a layer saw in the forward pass, kept for the privatising backward pass in a little over a
// byte a value.
//
// A block is 32 consecutive features of one token.  With a the largest finite magnitude in it, its scale is the smallest power of
// two s with a <= 448 s, and a value x is kept as the e4m3 number nearest to x / s (ties to even): relative error at most 2^-4, or
// half of 2^-9 s in absolute terms.  Powers of two because x / s and code * s are then exact: the only rounding is the code's, and
// the contractions read the checkpoint as bf16 operands without another one.  Features, not tokens, share a scale, so that a token
// can be written by itself.
//
// Both kernels are bound by memory: a lane takes 16 features, so that codes travel in 16-byte pieces and two neighbouring lanes hold
// a block.  Every code of a row's pitch is written: the places after the last feature hold zeros.
#include "checkpoint.h"

namespace dp {

namespace {

struct CkArgs {
    const void *x;
    void *out;
    uint8_t *codes, *scales;
    const uint8_t *codes_in, *scales_in;
    size_t rows, stride, pieces;     // pieces of 16 features of all rows
    int features, per_row;           // pieces of a row (even)
};

// Row and piece of this thread.  One 64-bit division per workgroup (scalar), a 32-bit one per thread.
__device__ __forceinline__ bool ck_place(const CkArgs &a, size_t &row, int &piece)
{
    const size_t first = (size_t)blockIdx.x * 256, row0 = first / (unsigned)a.per_row;
    const unsigned at = (unsigned)(first - row0 * (unsigned)a.per_row) + threadIdx.x, more = at / (unsigned)a.per_row;
    row = row0 + more;
    piece = (int)(at - more * (unsigned)a.per_row);
    return first + threadIdx.x < a.pieces;
}

template <bool BF16>
__global__ void __launch_bounds__(256) checkpoint_write_kernel(const CkArgs a)
{
    typedef typename In<BF16>::type E;
    size_t row;
    int piece;
    const bool there = ck_place(a, row, piece);
    const int count = there ? a.features - piece * 16 : 0;
    float v[16];
    load_values<BF16>(static_cast<const E *>(a.x) + row * a.stride + piece * 16, count, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    const bool broken = top >= 0x7F800000u;                        // an infinity or a NaN: no part in the scale, kept as NaN
    if (broken) {
        top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t m = __float_as_uint(v[i]) & 0x7FFFFFFFu;
            top = max(top, m < 0x7F800000u ? m : 0u);
        }
    }
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true));      // the block's other half: lane ^ 1
    // 448 = 1.75 * 2^8
    const int e = min(max((int)(top >> 23) - 135 + ((top & 0x7FFFFFu) > 0x600000u), CK_LOW), CK_HIGH);
    const float inv = pow2_of(127 - e);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = __builtin_amdgcn_fmed3f(v[4 * i + j] * inv, -448.0f, 448.0f);
        int packed = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
        packed = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], packed, true);
        w[i] = (uint32_t)packed;
    }
    if (broken) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if ((__float_as_uint(v[i]) & 0x7FFFFFFFu) >= 0x7F800000u)
                w[i >> 2] = (w[i >> 2] & ~(0xFFu << (8 * (i & 3)))) | (0x7Fu << (8 * (i & 3)));
    }
    if (!there) return;
    const size_t at = row * (unsigned)a.per_row + piece;
    reinterpret_cast<uint4 *>(a.codes)[at] = make_uint4(w[0], w[1], w[2], w[3]);
    if ((piece & 1) == 0) a.scales[at >> 1] = (uint8_t)(e + 127);
}

template <bool BF16>
__global__ void __launch_bounds__(256) checkpoint_read_kernel(const CkArgs a)
{
    typedef typename In<BF16>::type E;
    size_t row;
    int piece;
    if (!ck_place(a, row, piece)) return;
    const int count = a.features - piece * 16;
    if (count <= 0) return;                                        // the second half of a last block that ends in its first
    const size_t at = row * (unsigned)a.per_row + piece;
    const uint4 c = reinterpret_cast<const uint4 *>(a.codes_in)[at];
    const float scale = pow2_of(a.scales_in[at >> 1]);
    E *out = static_cast<E *>(a.out) + row * a.stride + piece * 16;
    const uint32_t codes[4] = {c.x, c.y, c.z, c.w};
    if constexpr (BF16) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const uint2 d = ck_bf16(codes[i], scale); w[2 * i] = d.x; w[2 * i + 1] = d.y; }
        if (count < 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < count) out[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        } else if ((reinterpret_cast<uintptr_t>(out) & 2) == 0) {
            *reinterpret_cast<u32x4_a4 *>(out) = u32x4_a4{w[0], w[1], w[2], w[3]};
            *reinterpret_cast<u32x4_a4 *>(out + 8) = u32x4_a4{w[4], w[5], w[6], w[7]};
        } else {                                                   // a value, seven dwords, a value
            uint32_t s[7];
#pragma unroll
            for (int i = 0; i < 7; ++i) s[i] = funnel(w[i + 1], w[i], 16);
            out[0] = (uint16_t)w[0];
            *reinterpret_cast<u32x4_a4 *>(out + 1) = u32x4_a4{s[0], s[1], s[2], s[3]};
            *reinterpret_cast<u32x2_a4 *>(out + 9) = u32x2_a4{s[4], s[5]};
            *reinterpret_cast<uint32_t *>(out + 13) = s[6];
            out[15] = (uint16_t)(w[7] >> 16);
        }
    } else {
        float v[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2 d = ck_bf16(codes[i], scale);
            v[4 * i] = __uint_as_float(d.x << 16); v[4 * i + 1] = __uint_as_float(d.x & 0xFFFF0000u);
            v[4 * i + 2] = __uint_as_float(d.y << 16); v[4 * i + 3] = __uint_as_float(d.y & 0xFFFF0000u);
        }
        if (count < 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < count) out[i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<u32x4_a4 *>(out + 4 * i) = u32x4_a4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                                                       __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
        }
    }
}

CkArgs ck_args(size_t rows, int features, size_t stride)
{
    CkArgs a = {};
    a.rows = rows;
    a.stride = stride;
    a.features = features;
    a.per_row = ck_pitch(features) / 16;
    a.pieces = rows * (size_t)a.per_row;
    return a;
}

}  // namespace

dp_status launch_checkpoint_write(const void *x, bool bf16, size_t rows, int features, size_t stride, uint8_t *codes, uint8_t *scales,
                                  hipStream_t s)
{
    CkArgs a = ck_args(rows, features, stride);
    a.x = x; a.codes = codes; a.scales = scales;
    const dim3 grid((unsigned)((a.pieces + 255) / 256));
    if (bf16) hipLaunchKernelGGL(checkpoint_write_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(checkpoint_write_kernel<false>, grid, dim3(256), 0, s, a);
    return check_launch("checkpoint_write");
}

dp_status launch_checkpoint_read(const uint8_t *codes, const uint8_t *scales, bool bf16, size_t rows, int features, void *x, size_t stride,
                                 hipStream_t s)
{
    CkArgs a = ck_args(rows, features, stride);
    a.out = x; a.codes_in = codes; a.scales_in = scales;
    const dim3 grid((unsigned)((a.pieces + 255) / 256));
    if (bf16) hipLaunchKernelGGL(checkpoint_read_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(checkpoint_read_kernel<false>, grid, dim3(256), 0, s, a);
    return check_launch("checkpoint_read");
}

}  // namespace dp
