// Which words of memory the training kernels read where an operand's rows start on any byte: plain functions, so that
// they can be run over all widths and alignments on the host.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define PG_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define PG_HOST_DEVICE inline
#endif

namespace pgt {

// Scales (one byte for 32 columns) that a row of `cols` columns has for the 128 columns from `col` on: none behind the row's end.
PG_HOST_DEVICE int scales_of_tile(int cols, int col) {
    const int left = col < cols ? (cols - col + 31) / 32 : 0;
    return left < 4 ? left : 4;
}
// Aligned 4-byte words, from the one that holds address `from` on, that hold `count` bytes from there (four at most).
PG_HOST_DEVICE int words_of_scales(uintptr_t from, int count) {
    return count <= 0 ? 0 : static_cast<int>(from & 3) + count > 4 ? 2 : 1;
}

}  // namespace pgt
