// Products of bf16 matrices with fp32 sums, and of fp32 matrices as three bf16 planes each, for the operators whose hot part they are
// (include/canvas_gated.h, canvas_head.h): plans, and the launches that those operators share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace canvas {
namespace product {

// One operand.  In memory either rows of indexes with the summed index k along them, or rows of k with the indexes along them.  bf16: rows of a multiple of 8
// elements.  fp32 matrices: rows of pieces of 16 columns, each its first, second and third plane in turn, so that what a stage of a product takes of a
// row lies together.  From their end to the next multiple of 8 or 16 rows hold zeros.
struct Factor {
    const uint16_t* p[2] = {nullptr, nullptr};  // of the two halves of a sum over 2 * depth, or of the two results of a launch
    int64_t ld = 0;                             // elements of all planes from row to row
    int64_t count = 0;                          // indexes
};
__host__ __device__ inline int64_t padded(bool f32, int64_t cols) { return f32 ? (cols + 15) / 16 * 16 : (cols + 7) / 8 * 8; }
__host__ __device__ inline int64_t pitch(bool f32, int64_t cols) { return padded(f32, cols) * (f32 ? 3 : 1); }
// Where eight columns from `col` (a multiple of 8) on begin in their row, plane h.
template <int PLANES>
__host__ __device__ constexpr int64_t column(int64_t col, int h) { return PLANES == 1 ? col : col / 16 * 48 + h * 16 + col % 16; }

// How results are cut: tiles of `high` x `side`, the sum over k in `splits` parts.
struct Cut {
    int side = 128, high = 128, splits = 1;
    int64_t tiles_i = 0, tiles_j = 0;
    int64_t tiles() const { return tiles_i * tiles_j; }
};

// C[i][j] = sum_k A[i][k] B[j][k] for `results` pairs of matrices, or one sum over both of them.
struct Product {
    Factor a, b;
    bool a_rows = false;   // A as rows of indexes (B, and A without it, as rows of k)
    bool f32 = false;      // three planes, results in fp32; else one, results in bf16
    int64_t depth = 0;     // of one of them
    int segments = 1, results = 1;
    void* out[2] = {nullptr, nullptr};
    int64_t ld = 0;
    Cut cut;
    float* parts = nullptr;
    // A sum that several launches add to, in order: each leaves its part in `parts`; the last one's is followed by the sum's end.
    bool first = true, last = true;
};

// `us`: about what it takes.
Cut cut_of(bool f32, int64_t rows, int64_t cols, int64_t depth, int results, bool may_split, double* us = nullptr);
// Of two products that one launch may take if their tiles are alike.
struct Size {
    int64_t rows, cols, depth;
    int results;
};
void cuts_of(bool f32, const Size& x, const Size& y, Cut& cx, Cut& cy);
uint64_t parts_bytes(const Cut& c, int results, bool several);
// One product, or two that do not wait for each other, the first with a_rows.
void multiply(const Product& p, hipStream_t stream);
void multiply(const Product& x, const Product& y, hipStream_t stream);
// Launches of the latter; `several`: more than one adds to x.
int launches_of(const Cut& x, const Cut& y, bool several);

// A matrix of `rows` x `cols` elements laid out as a Factor.
// `live`: bytes by row, 0 for rows that are zeros in the copy whatever they hold.
struct Copy {
    const void* from = nullptr;
    uint16_t* to = nullptr;
    int64_t rows = 0, cols = 0;
    const uint8_t* live = nullptr;
};
void copy(bool f32, const Copy* copies, int n, hipStream_t stream);

}  // namespace product
}  // namespace canvas
