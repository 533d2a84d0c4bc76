// The inner part of a product of a weight [n][k] with few rows x [rows][k], 16 NT of them at a time: up to 32 rows bound by reading the weight, which goes from
// memory to the registers of the wave that multiplies it, in most bf16 products through that wave's piece of LDS (Lanes); more rows by the matrix units (92 TFLOP/s in fp32, workgroups of 32 x 64 results; 82 with the four products of a pair of loads one after the other on one sum).
//
// A workgroup takes R blocks of 16 rows of weights.  Its waves share out the summed index, AHEAD times 64 bytes of a row each in turn, and
// add up through LDS in the order of the waves.  bf16: the 16 x 16 x 32 product of the matrix units; fp32: their 16 x 16 x 4 one, whose products
// and sums are those of fp32.  Rows may begin at any element.
#pragma once
#include <hip/hip_runtime.h>

#include "product_device.hpp"
#include "tile_util.hpp"

namespace canvas {
namespace few {

using product::f32x4;
using tile::u32x4;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
// Loads of 64 bytes a row that are in flight, by what the registers of two or three waves a SIMD unit hold.
constexpr int ahead(int blocks, int nt) { return blocks * nt > 4 ? 2 : 4; }
// Whether this is the way for `rows` rows, by blocks of 64 of them, against `results` rows of weights.  Always up to 32.  More in fp32, where tiles need copies of both operands in planes first (10
// bytes an element, and a launch) and do not share out the summed index, if that takes 1.25 times as long (`tiles`: us of the products in tiles).  Both in us, without copies and
// with: pairs 64 x 1000 x 2 * 2731 16 and 55; 512 x 512 x 2 * 512 10 and 23; 250 x 4000 x 2 * 1000 50 and 146; 128 x 2000 x 2 * 8000 103 and 182; 256 x 2000 x 2 * 8000 194 and 173;
// heads 64 x 1000 x 50000 109 and 228; 256 x 512 x 1000 14 and 18; 2000 x 300 x 1000 30 and 22.  bf16: 64 x 2048 x 2 * 8192 24 and 14, 512 x 512 x 2 * 512 5.6 and 5.9.
constexpr int64_t kRows = 32, kMostRows = 4096;
inline bool fits(bool f32, int64_t rows, int64_t results, int64_t features, double tiles) {
    if (rows <= kRows || !f32 || rows > kMostRows) return rows <= kRows;
    const int64_t turns = ((results + 31) / 32 * ((rows + 63) / 64) + 255) / 256;
    const double here = 2 + (double)turns * (1.8 + 0.0114 * (double)features);
    return 1.25 * here < 1.15 * tiles + 6 + 10.0 * (double)(rows + results) * (double)features / 4e6;
}

template <class T>
struct Type;
template <>
struct Type<uint16_t> {
    static constexpr int kEach = 8;  // elements of 16 bytes
    static constexpr int kProducts = 1;  // of 16 bytes of each operand
    static __device__ __forceinline__ void multiply(const u32x4& a, const u32x4& b, int, f32x4& c) { c = tile::mfma32(a, b, c); }
};
template <>
struct Type<float> {
    static constexpr int kEach = 4;
    static constexpr int kProducts = 4;
    static __device__ __forceinline__ void multiply(const u32x4& a, const u32x4& b, int e, f32x4& c) {
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    }
};

// Nothing that a lane leaves in LDS for another of its wave changes places with what that one reads.
__device__ __forceinline__ void in_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
template <class T>
__device__ __forceinline__ u32x4 load16(const T* p) {
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
// Elements k .. of a row of `end`, zeros behind it.
template <class T>
__device__ __forceinline__ u32x4 load_end(const T* row, int64_t k, int64_t end) {
    T e[Type<T>::kEach];
#pragma unroll
    for (int i = 0; i < Type<T>::kEach; i++) e[i] = k + i < end ? row[k + i] : T(0);
    u32x4 v;
    __builtin_memcpy(&v, e, 16);
    return v;
}

// Which row of a block of 16 a lane loads, and which 16 of 64 bytes.  As the matrix units want them, lane % 16: no two lanes beside each other share a line, which the L1 serves one after the other.
// STAGED: four lanes beside each other take 64 bytes of a row, and the wave's own piece of LDS gives each lane its operands.  That is for bf16, most where rows begin anywhere: pairs, us,
// 7 x 3869 x 2 * 530 10 instead of 25, 27 x 3869 x 2 * 530 13 and 36, 32 x 2048 x 2 * 8192 15.3 and 17, 4 x 2048 x 2 * 8192 12 and 12; heads of 7 x 1001 x 50000 45 and 50, 32 x 2048 x 131072
// 117 and 121, but of 4 x 2048 x 131072 107 instead of 102.  fp32, whose matrix instructions take longer: 128 x 2000 x 2 * 8000 107 instead of 103, 512 x 512 x 2 * 512 8.8 and 10.3.
template <bool STAGED>
struct Lanes {
    static constexpr bool kStaged = STAGED;
    static __device__ __forceinline__ int row() { return kStaged ? (threadIdx.x & 63) >> 2 : threadIdx.x & 15; }
    static __device__ __forceinline__ int piece() { return kStaged ? threadIdx.x & 3 : (threadIdx.x & 63) >> 4; }
};
// Pieces of row r lie at place piece ^ (r / 4), so that 16 lanes read 16 pieces on different banks.
__device__ __forceinline__ int place_of(int row, int piece) { return row * 4 + (piece ^ (row >> 2)); }
// f32x4 elements of LDS that accumulate() takes.
template <bool STAGED, int R, int NT>
constexpr int kShared = kWaves * 64 * (R * NT > R + NT || !STAGED ? R * NT : R + NT);

// sums[r][t]: of weight rows `w[r]` (the row that this lane loads of the block) and rows `x[t]`; whole sums in waves 0 .. NT - 1, wave t those of rows 16 t ..:
// register e of a lane is weight row (lane / 16) * 4 + e, row lane % 16 of x.
template <bool STAGED, class T, int R, int NT, int AHEAD>
__device__ __forceinline__ void accumulate(const T* const (&w)[R], const T* const (&x)[NT], int64_t depth, f32x4 (&sums)[R], f32x4* shared) {
    using Y = Type<T>;
    constexpr int kStep = 4 * Y::kEach, kTurn = kStep * AHEAD;  // elements of a row that a wave takes per load, and per turn
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t mine = Lanes<STAGED>::piece() * Y::kEach;
    u32x4* const stage = reinterpret_cast<u32x4*>(shared) + wave * ((R + NT) * 64);
    const int put = place_of(Lanes<STAGED>::row(), Lanes<STAGED>::piece()), get = place_of(lane & 15, lane >> 4);
    f32x4 acc[R][NT] = {};
    struct Turn {
        u32x4 w[R][AHEAD], x[NT][AHEAD];
    };
    auto load = [&](int64_t k, Turn& t) {
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
#pragma unroll
            for (int r = 0; r < R; r++) t.w[r][u] = load16(w[r] + k + u * kStep + mine);
#pragma unroll
            for (int n = 0; n < NT; n++) t.x[n][u] = load16(x[n] + k + u * kStep + mine);
        }
    };
    // of 64 bytes of each row
    auto products = [&](const u32x4 (&a)[R], const u32x4 (&b)[NT]) {
#pragma unroll
        for (int e = 0; e < Y::kProducts; e++)
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
                for (int n = 0; n < NT; n++) Y::multiply(a[r], b[n], e, acc[r][n]);
    };
    auto step = [&](const u32x4 (&a)[R], const u32x4 (&b)[NT]) {
        if (!STAGED) return products(a, b);
        u32x4 p[R], q[NT];
        in_order();  // (a wave's accesses to LDS are)
#pragma unroll
        for (int r = 0; r < R; r++) stage[r * 64 + put] = a[r];
#pragma unroll
        for (int n = 0; n < NT; n++) stage[(R + n) * 64 + put] = b[n];
        in_order();
#pragma unroll
        for (int r = 0; r < R; r++) p[r] = stage[r * 64 + get];
#pragma unroll
        for (int n = 0; n < NT; n++) q[n] = stage[(R + n) * 64 + get];
        products(p, q);
    };
    auto multiply = [&](const Turn& t) {
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            u32x4 a[R], b[NT];
#pragma unroll
            for (int r = 0; r < R; r++) a[r] = t.w[r][u];
#pragma unroll
            for (int n = 0; n < NT; n++) b[n] = t.x[n][u];
            step(a, b);
        }
    };
    const int64_t whole = depth / kTurn;
    int64_t turn = wave;
    if (turn < whole) {
        Turn t[2];
        load(turn * kTurn, t[0]);
        for (; turn + kWaves < whole; turn += kWaves) {
            load((turn + kWaves) * kTurn, t[1]);
            multiply(t[0]);
            t[0] = t[1];
        }
        multiply(t[0]);
        turn += kWaves;
    }
    if (turn == whole) {  // what is left of the rows is one wave's
#pragma unroll 1
        for (int64_t k = whole * kTurn; k < depth; k += kStep) {
            u32x4 a[R], b[NT];
#pragma unroll
            for (int r = 0; r < R; r++) a[r] = load_end(w[r], k + mine, depth);
#pragma unroll
            for (int n = 0; n < NT; n++) b[n] = load_end(x[n], k + mine, depth);
            step(a, b);
        }
    }
    if (STAGED) __syncthreads();
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int n = 0; n < NT; n++) shared[((r * NT + n) * kWaves + wave) * 64 + lane] = acc[r][n];
    __syncthreads();
    if (wave >= NT) return;
#pragma unroll
    for (int r = 0; r < R; r++) {
        sums[r] = f32x4{};
#pragma unroll
        for (int v = 0; v < kWaves; v++) sums[r] += shared[((r * NT + wave) * kWaves + v) * 64 + lane];
    }
}

}  // namespace few
}  // namespace canvas
