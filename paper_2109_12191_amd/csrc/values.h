// Runs of consecutive values between memory and registers, from any element of a row on and of any count: bf16 rows of odd length
// start in the middle of a dword, and what lies outside a run is neither read nor written, so the ends of a tensor need no care.
// gfx950 only.
#pragma once

#include "pieces.h"

namespace dp {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2_a4 __attribute__((ext_vector_type(2), aligned(4)));

// Eight consecutive bf16 values, `count` of them there (any number; the others zero), from any element on.
__device__ __forceinline__ uint4 load8(const uint16_t *p, int count)
{
    if (count >= 8) {
        if ((reinterpret_cast<uintptr_t>(p) & 2) == 0) {
            const u32x4_a4 a = *reinterpret_cast<const u32x4_a4 *>(p);
            return make_uint4(a.x, a.y, a.z, a.w);
        }
        const uint32_t first = p[0], last = p[7];
        const u32x2_a4 a = *reinterpret_cast<const u32x2_a4 *>(p + 1);
        const uint32_t b = *reinterpret_cast<const uint32_t *>(p + 5);
        return make_uint4(funnel(a.x, first << 16, 16), funnel(a.y, a.x, 16), funnel(b, a.y, 16), funnel(last, b, 16));
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The same of fp32 values.
__device__ __forceinline__ void load8f(const float *p, int count, float (&v)[8])
{
    if (count >= 8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x4_a4 a = *reinterpret_cast<const u32x4_a4 *>(p + 4 * i);
            v[4 * i] = __uint_as_float(a.x); v[4 * i + 1] = __uint_as_float(a.y);
            v[4 * i + 2] = __uint_as_float(a.z); v[4 * i + 3] = __uint_as_float(a.w);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? p[i] : 0.0f;
}

__device__ __forceinline__ void widen8(const uint4 &w, float (&v)[8])
{
    const uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(d[i] << 16); v[2 * i + 1] = __uint_as_float(d[i] & 0xFFFF0000u); }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const f32x2_t p = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2_t));       // nearest, ties to even
}

// Eight values as they were loaded.
template <bool BF16> struct Raw8;
template <> struct Raw8<true> {
    uint4 w;
    __device__ __forceinline__ void load(const void *p, size_t at, int count) { w = load8(static_cast<const uint16_t *>(p) + at, count); }
    __device__ __forceinline__ void get(float (&v)[8]) const { widen8(w, v); }
};
template <> struct Raw8<false> {
    float w[8];
    __device__ __forceinline__ void load(const void *p, size_t at, int count) { load8f(static_cast<const float *>(p) + at, count, w); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w[i];
    }
};

// Eight values to memory, the first `count` of them.
__device__ __forceinline__ void store8(uint16_t *p, int count, const float (&v)[8])
{
    const uint32_t w[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    if (count < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    } else if ((reinterpret_cast<uintptr_t>(p) & 2) == 0) {
        *reinterpret_cast<u32x4_a4 *>(p) = u32x4_a4{w[0], w[1], w[2], w[3]};
    } else {
        p[0] = (uint16_t)w[0];
        *reinterpret_cast<u32x2_a4 *>(p + 1) = u32x2_a4{funnel(w[1], w[0], 16), funnel(w[2], w[1], 16)};
        *reinterpret_cast<uint32_t *>(p + 5) = funnel(w[3], w[2], 16);
        p[7] = (uint16_t)(w[3] >> 16);
    }
}
__device__ __forceinline__ void store8(float *p, int count, const float (&v)[8])
{
    if (count < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = v[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        *reinterpret_cast<u32x4_a4 *>(p + 4 * i) = u32x4_a4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                                             __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
}

}  // namespace dp
