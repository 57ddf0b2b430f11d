// Walks addresses, strides, widths and counts of rows and checks, wherever rows are taken by whole dwords, that each workgroup's buffer begins at a whole
// dword and ends with the dword that its last value lies in, and that byte offsets into it fit.
#include "token_words.h"

#include <cstdio>
#include <initializer_list>

using namespace dp;

int main()
{
    long long taken = 0, refused = 0, bad = 0;
    const size_t strides[] = {1, 2, 3, 7, 8, 1003, 1004, 2049, 2050, 5001, 16383, (1u << 24) + 1, 1u << 28, 1u << 29}, counts[] = {1, 2, 3, 5, 64, 1000, 100000};
    for (bool bf16 : {false, true})
        for (int address : {0x10000, 0x10002, 0x10004, 0x10006})
            for (size_t stride : strides)
                for (size_t all : counts)
                    for (size_t rows : {(size_t)1, (size_t)2, (size_t)4, (size_t)32, (size_t)64}) {
                        const size_t size = bf16 ? 2 : 4;
                        const uintptr_t at = address;
                        if (at % size || rows > all) continue;
                        if (!token_rows_by_words(reinterpret_cast<const void *>(at), bf16, stride, all, rows)) { ++refused; continue; }
                        ++taken;
                        for (size_t width : {stride, stride > 1 ? stride - 1 : stride})
                            for (size_t first = 0; first < all; first += rows) {
                                const size_t there = all - first < rows ? all - first : rows;
                                const uintptr_t base = at + first * stride * size, last = base + ((there - 1) * stride + width) * size;      // end of the last value
                                const uintptr_t end = base + ((((there - 1) * stride + width) * size + 3) & ~(size_t)3);
                                if (base % 4 == 0 && end / 4 == (last + 3) / 4 && end - base <= (size_t)1 << 30) continue;
                                if (!bad++) printf("%s at %zx, %zu rows of %zu every %zu, %zu to a workgroup: row %zu at %zx, buffer to %zx\n", bf16 ? "bf16" : "fp32", (size_t)at, all, width, stride, rows, first, (size_t)base, (size_t)end);
                            }
                    }
    // the ordinary calls are taken: packed rows of even width, single rows of any, fp32
    const void *even = reinterpret_cast<const void *>((uintptr_t)0x10000);
    const bool ordinary = token_rows_by_words(even, true, 768, 1000, 64) && token_rows_by_words(even, true, 1003, 1, 1) && token_rows_by_words(even, false, 1003, 1000, 64);
    printf("%lld calls by words, %lld not, %lld workgroups with a bad buffer\n", taken, refused, bad);
    return bad || !taken || !refused || !ordinary;
}
