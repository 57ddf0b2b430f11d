// Which rows of tokens kernels take by whole dwords.  Host code only.
#pragma once

#include <cstddef>
#include <cstdint>

namespace dp {

// Whether the `all` rows of a call can be read by whole dwords from one buffer per workgroup of `rows` rows: every bf16 row has to begin at a whole
// dword -- a workgroup's buffer begins with its first row, which is any row of the call's, and ends with the dword that holds its last value --, and what a
// workgroup's rows span has to be below 2^31 bytes.  (Other rows go by pointers, which takes longer: 8 x 500 tokens of 5001 bf16 features 48 us forward, of 5000 28.)
inline bool token_rows_by_words(const void *p, bool bf16, size_t stride, size_t all, size_t rows)
{
    const size_t size = bf16 ? 2 : 4;
    if (bf16 && ((reinterpret_cast<uintptr_t>(p) & 3) || (all > 1 && stride % 2))) return false;
    return rows * stride <= ((size_t)1 << 30) / size;
}

}  // namespace dp
