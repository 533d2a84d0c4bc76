// Pieces of rows of any length, on the host too, where a test reads rows that end where memory does.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace canvas {
namespace rows {

// Elements col .. col + 7 (col a multiple of 8) of a row of `cols`: zeros behind its end, where nothing is read.  Rows of a multiple of 8 are aligned to 16 bytes and
// read in whole vectors.
template <class T>
__host__ __device__ inline void load8(const T* row, int64_t col, int64_t cols, T (&v)[8]) {
    if ((cols & 7) != 0) {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = col + e < cols ? row[col + e] : T(0);
    } else if (col < cols) {  // (rows of 8 more than a multiple of 16 are followed by a piece without elements where pieces go in pairs)
        __builtin_memcpy(v, __builtin_assume_aligned(row + col, 16), sizeof(v));
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = T(0);
    }
}

}  // namespace rows
}  // namespace canvas
