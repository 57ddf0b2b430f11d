// A workgroup's rows of a tensor of tokens, in runs of eight consecutive values from any multiple of eight on.  gfx950 only.
#pragma once

#include "token_words.h"
#include "values.h"

namespace dp {

typedef uint32_t u32x4_v __attribute__((ext_vector_type(4)));

// Rows `first` .. `first + rows - 1` of a tensor, `width` values each.  WORDS: 16-byte buffer accesses, left out by an offset beyond the buffer;
// a run that a row ends in is loaded whole, with what follows it in memory (zeros after the last row, but for the other half of a last dword),
// and stored value by value.  Else by pointers, from any element on.  What a run holds after its row's values is unspecified.
template <bool BF16, bool WORDS>
struct TokenRows {
    typedef typename In<BF16>::type E;
    static constexpr unsigned AWAY = 0x80000000u;        // an offset beyond every buffer
    __amdgpu_buffer_rsrc_t buffer;
    E *base;
    size_t stride;
    int width;
    __device__ __forceinline__ TokenRows(const void *p, size_t first, int rows, size_t stride_, int width_)
        : base(static_cast<E *>(const_cast<void *>(p)) + first * stride_), stride(stride_), width(width_)
    {
        if constexpr (WORDS)
            buffer = __builtin_amdgcn_make_buffer_rsrc(base, 0, (int)((((unsigned)(rows - 1) * (unsigned)stride + (unsigned)width) * (unsigned)sizeof(E) + 3u) & ~3u), 0x00020000);
    }
    // `there`: whether there is anything to load (the run's values are zeros if not, by words)
    __device__ __forceinline__ void load(Raw8<BF16> &raw, bool there, int row, int k) const
    {
        if constexpr (WORDS) {
            const int at = (int)(there && k < width ? ((unsigned)row * (unsigned)stride + (unsigned)k) * (unsigned)sizeof(E) : AWAY);
            const u32x4_v v = __builtin_bit_cast(u32x4_v, __builtin_amdgcn_raw_buffer_load_b128(buffer, at, 0, 0));
            if constexpr (BF16) {
                raw.w = make_uint4(v.x, v.y, v.z, v.w);
            } else {
                const u32x4_v w = __builtin_bit_cast(u32x4_v, __builtin_amdgcn_raw_buffer_load_b128(buffer, at + 16, 0, 0));
                raw.w[0] = __uint_as_float(v.x); raw.w[1] = __uint_as_float(v.y); raw.w[2] = __uint_as_float(v.z); raw.w[3] = __uint_as_float(v.w);
                raw.w[4] = __uint_as_float(w.x); raw.w[5] = __uint_as_float(w.y); raw.w[6] = __uint_as_float(w.z); raw.w[7] = __uint_as_float(w.w);
            }
        } else {
            raw.load(base, there ? (size_t)row * stride + (size_t)k : 0, there ? width - k : 0);
        }
    }
    __device__ __forceinline__ void store(int row, int k, const float (&v)[8]) const
    {
        if (k >= width) return;
        if (WORDS && k + 8 <= width) {
            const int at = (int)(((unsigned)row * (unsigned)stride + (unsigned)k) * (unsigned)sizeof(E));
            if constexpr (BF16) {
                const u32x4_v w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
                __builtin_amdgcn_raw_buffer_store_b128(w, buffer, at, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x4_v w = {__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
                    __builtin_amdgcn_raw_buffer_store_b128(w, buffer, at + 16 * i, 0, 0);
                }
            }
        } else {
            store8(base + (size_t)row * stride + (size_t)k, width - k, v);
        }
    }
};

}  // namespace dp
