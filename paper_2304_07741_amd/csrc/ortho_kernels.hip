// Newton-Schulz products of the orthogonalised update.
//
// A matrix of fp32 values v is held as two fp16 planes: hi = fp16(2^12 v), lo = fp16(2^12 v - hi).  |X| <= 1.3 and |b A + c A A + a I| <= 3.45
// in every step and the product of two of the latter below 12 (spectral norms bound the elements), so hi stays in fp16's range, and lo
// keeps 11 more bits of every element above 2^-15 of the largest possible one.  Where |v| is not far above the 1e-7 that is added to it, or
// below, X is small: its planes hold 2^up X with |2^up X| in [1/2, 1) at the start, and each step, which makes X at most 3.4445 times as
// large, takes as much from `up` until nothing is left.  A product of two such matrices is hi hi + hi lo + lo hi on the matrix units with fp32
// sums; lo lo is below 2^-22 of a term.
//
// Per step, with both X [m][n] and its transpose at hand so that every operand is read along the index that is summed over:
//   A = X X^T   (tiles on and below the diagonal, written on both sides of it)
//   B = a I + b A + c A A^T  (the same)
//   X = B X     (from the rows of B and of X^T; both X and X^T are written, or, in the last step, the outputs)
// Where the longer side is much longer, two steps at a time: with B0 and B1 polynomials of A, all these matrices commute, so
// A1 = B0 A B0 is the second step's A, and X = (B1 B0) X.  Three short symmetric products take the place of two long ones, one of
// them symmetric.  Rounding leaves the same error as step by step (what is wrong with B moves X by as much of X, also where X is
// weak); three steps at a time would leave two to three times that.
//
// Large matrices are bound by the matrix units, small ones by the launches that wait for each other.  2048 x 8192: the long products
// take 185-200 us each (1030-1110 TFLOP/s of fp16 products; a plain 8192 x 8192 x 8192 one of the library reaches 1145), Gram matrices 105 + 14 for the sums of
// their parts, short products 36 + 10 (740 TFLOP/s), momentum and splitting 85; five steps 1.48 ms.  256 x 2304: 22 launches of 4-8 us, 119-122 us.
#include "ortho_kernels.hpp"

#include <algorithm>
#include <atomic>

#include "device_util.hpp"
#include "launch.hpp"
#include "ortho_device.hpp"
#include "ortho_small_kernels.hpp"
#include "tile_util.hpp"

namespace canvas {
namespace ortho {
namespace {

constexpr int kThreads = 256;
constexpr float kScale = 4096.f;  // 2^12
constexpr int kDepth = 32;        // of one step of a product; leading dimensions are multiples of it, zeros behind the columns

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
using tile::u32x4;

// One matrix per group as two planes of rows; lo is `plane` elements behind hi, the next group's `step` behind this one's.
struct Pair {
    _Float16* hi;
    int64_t plane, step;
    int ld;
};

// What the planes of X are scaled by beyond 2^12, where the start's exponent is `up`, after steps that can have made X 2^grown times as large.
__device__ __forceinline__ int exponent_after(int up, int grown) { return up > grown ? up - grown : 0; }
constexpr int grown_by(int steps) { return (steps * 1785 + 999) / 1000; }  // log2(3.4445) = 1.7843 per step

__device__ __forceinline__ uint32_t pack_pair(float v) {  // v scaled: hi in the low half, lo in the high one
    const _Float16 h = (_Float16)v, l = (_Float16)(v - (float)h);
    return (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
}
__device__ __forceinline__ float of_half(uint32_t u) { return (float)__builtin_bit_cast(_Float16, (uint16_t)u); }

// 16 bytes per lane from `from` + voff + soff to LDS, lane after lane behind `to` (the same for the whole wave).
__device__ __forceinline__ tile::rsrc_t whole_memory(const void* from) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(from), 0, 0xffffffffu, 0x00020000); }
__device__ __forceinline__ void load_to_lds(tile::rsrc_t from, unsigned char* to, uint32_t voff, int soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, voff, soff, 0, 0);
}

// A barrier behind which everybody's loads to LDS have arrived.  (A barrier alone waits for them only where the compiler sees a read
// behind it that may concern them.)
__device__ __forceinline__ void loads_arrived() {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    __syncthreads();
}

// Momentum and the sum of squares of the direction, one part of a matrix per workgroup.
__global__ __launch_bounds__(kThreads) void k_mix(Shape s, Args a, double* sums) {
    __shared__ double buf[kThreads];
    const int64_t len = s.R * s.K, base = blockIdx.y * len, stride = (int64_t)gridDim.x * kThreads;
    const int64_t first = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    double t = 0;
    auto one = [&](int64_t i) {
        float m = 0.f;
        if (a.momentum) {
            m = (float)(a.mu * a.momentum[i] + a.grad[i]);
            a.momentum_out[i] = m;
        }
        const double v = direction(s, a, i, m);
        t += v * v;
    };
    if ((len & 3) == 0) {  // every matrix begins at 16 bytes
        for (int64_t k = first; k < len / 4; k += stride) {
            const int64_t i = base + 4 * k;
            const f32x4 g = *reinterpret_cast<const f32x4*>(a.grad + i);
            f32x4 v = g;
            if (a.momentum) {
                const f32x4 old = *reinterpret_cast<const f32x4*>(a.momentum + i);
                f32x4 m;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    m[e] = (float)(a.mu * old[e] + g[e]);
                    v[e] = s.nesterov ? (float)(g[e] + a.mu * m[e]) : m[e];
                }
                *reinterpret_cast<f32x4*>(a.momentum_out + i) = m;
            }
#pragma unroll
            for (int e = 0; e < 4; e++) t += (double)v[e] * v[e];
        }
    } else {
        for (int64_t k = first; k < len; k += stride) one(base + k);
    }
    buf[threadIdx.x] = t;
    __syncthreads();
    for (int o = kThreads / 2; o; o >>= 1) {
        if ((int)threadIdx.x < o) buf[threadIdx.x] += buf[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) sums[blockIdx.y * gridDim.x + blockIdx.x] = buf[0];
}

// 1 / (|v| + 1e-7) of this workgroup's matrix, and the power of two that brings |v| / (|v| + 1e-7) to [1/2, 1).
struct Norm {
    double inverse;
    int up;
};
__device__ Norm norm_of(const double* sums, int parts) {
    __shared__ double buf[kThreads / 64];
    double t = 0;
    for (int k = threadIdx.x; k < parts; k += kThreads) t += sums[k];
#pragma unroll
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = t;
    __syncthreads();
    t = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; w++) t += buf[w];
    const double inverse = inverse_norm(t), part = sqrt(t) * inverse;
    return Norm{inverse, part > 0 && part < 0.5 ? 1022 - (int)(__double_as_longlong(part) >> 52) : 0};
}

// X and X^T of the normalised direction, 64 x 64 elements per workgroup through LDS; zeros behind the columns.
__global__ __launch_bounds__(kThreads) void k_start(Shape s, Args a, const double* sums, int parts, int* ups, Pair x, Pair xt) {
    __shared__ uint32_t img[64][65];
    const unsigned wide = (unsigned)((s.K + 63) / 64), by = blockIdx.x / wide;
    const int64_t len = s.R * s.K, r0 = (int64_t)by * 64, c0 = (int64_t)(blockIdx.x - by * wide) * 64;
    const int c = (threadIdx.x & 15) * 4, r = threadIdx.x >> 4;
    const bool whole = (s.K & 3) == 0;  // four elements side by side are aligned and in one row
    const float* m = a.momentum ? a.momentum_out : nullptr;
    f32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int64_t row = r0 + r + 16 * k, col = c0 + c, i = blockIdx.y * len + row * s.K + col;
        v[k] = f32x4{};
        if (row >= s.R || col >= s.K) continue;
        if (whole) {
            const f32x4 g = !m || s.nesterov ? *reinterpret_cast<const f32x4*>(a.grad + i) : f32x4{}, w = m ? *reinterpret_cast<const f32x4*>(m + i) : f32x4{};
#pragma unroll
            for (int e = 0; e < 4; e++) v[k][e] = !m ? g[e] : s.nesterov ? (float)(g[e] + a.mu * w[e]) : w[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (col + e < s.K) v[k][e] = direction(s, a, i + e, m ? m[i + e] : 0.f);
        }
    }
    const Norm norm = norm_of(sums + (int64_t)blockIdx.y * parts, parts);
    const double inv = ldexp(norm.inverse, norm.up);
    if (blockIdx.x == 0 && threadIdx.x == 0) ups[blockIdx.y] = norm.up;
    // four pairs side by side
    auto put = [&](const Pair& to, int64_t row, int64_t col, const uint32_t (&p)[4]) {
        _Float16* at = to.hi + blockIdx.y * to.step + row * to.ld + col;
        const uint32_t hi[2] = {__builtin_amdgcn_perm(p[1], p[0], 0x05040100u), __builtin_amdgcn_perm(p[3], p[2], 0x05040100u)};
        const uint32_t lo[2] = {__builtin_amdgcn_perm(p[1], p[0], 0x07060302u), __builtin_amdgcn_perm(p[3], p[2], 0x07060302u)};
        __builtin_memcpy(at, hi, 8);
        __builtin_memcpy(at + to.plane, lo, 8);
    };
    // orig: the planes laid out as the gradient is; turned: its transpose
    const Pair orig = s.tall ? xt : x, turned = s.tall ? x : xt;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int64_t row = r0 + r + 16 * k, col = c0 + c;
        uint32_t p[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            p[e] = pack_pair((float)(v[k][e] * inv) * kScale);
            img[r + 16 * k][c + e] = p[e];
        }
        if (row < s.R && col < orig.ld) put(orig, row, col, p);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int64_t row = c0 + r + 16 * k, col = r0 + c;  // of the transpose
        uint32_t p[4];
#pragma unroll
        for (int e = 0; e < 4; e++) p[e] = img[c + e][r + 16 * k];
        if (row < s.K && col < turned.ld) put(turned, row, col, p);
    }
}

// Plans without products: the normalised direction itself.
__global__ __launch_bounds__(kThreads) void k_normalised(Shape s, Args a, const double* sums, int parts) {
    const double inv = norm_of(sums + (int64_t)blockIdx.y * parts, parts).inverse;
    const int64_t len = s.R * s.K, k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (k >= len) return;
    const int64_t i = blockIdx.y * len + k;
    finish_one(s, a, i, (float)(direction(s, a, i, a.momentum ? a.momentum_out[i] : 0.f) * inv));
}

enum Kind { kGram, kSquare, kUpdate, kLast };  // kGram: all symmetric products that nothing is added to

// C[i][j] = sum_k P[i][k] Q[j][k], rows of P x rows of Q, over `depth` (a multiple of kDepth, zeros at its end).
struct Product {
    Pair p, q;
    int rows, cols, depth;
    Pair out;   // kGram, kSquare: C, both sides; kUpdate: X
    Pair turn;  // kUpdate: X^T
    int tiles_i, tiles_j, tiles;
    // The sum over k cut into `splits` parts, a workgroup each, where there are few tiles.  Parts are left in memory for a launch
    // that adds them in their order.  (One launch in which the last workgroup at a tile adds them needs a fence over all XCDs
    // per workgroup, which writes back its L2: 89 us against 10 for the Gram matrix of 512 x 2048.)
    int splits;
    f32x4* parts;
    // Products with X: the exponents of the matrices, by how much the X that is read and the X that is written can have grown.
    const int* ups = nullptr;
    int grown_in = 0, grown_out = 0;
};
// The power of two that takes results from the scale of the operands' planes to that of the result's, apart from 2^12 (kLast: 2^24).
template <Kind KIND>
__device__ __forceinline__ int exponent_of(const Product& g, int grp) {
    if (KIND == kSquare || !g.ups) return 0;
    const int up = g.ups[grp], in = exponent_after(up, g.grown_in);
    return KIND == kGram ? -2 * in : KIND == kUpdate ? exponent_after(up, g.grown_out) - in : -in;
}

struct Tile {
    int grp, i0, j0;
    bool diagonal;
};
// A way of cutting products: tiles of BM x BN by WI x WJ waves, SUB times kDepth summands at a time.
template <int BM_, int BN_, int WI_, int WJ_, int SUB_>
struct Form {
    static constexpr int BM = BM_, BN = BN_, WI = WI_, WJ = WJ_, SUB = SUB_;
    static constexpr int kThreads = 64 * WI * WJ, TM = BM / WI / 32, TN = BN / WJ / 32;
    static constexpr int kOpA = BM * 64, kOpB = BN * 64;  // bytes of one plane of kDepth summands
    static constexpr int kPart = 2 * (kOpA + kOpB), kStage = SUB * kPart;
    static constexpr int kRows = BM * BN * 4 > kStage ? kStage / (BN * 4) : BM;  // of results that one buffer takes at once
};
using Large = Form<256, 256, 2, 4, 1>;
using Middle = Form<128, 128, 2, 2, 1>;
using Small = Form<64, 64, 2, 2, 2>;

template <int BM, int BN, Kind KIND>
__device__ __forceinline__ Tile tile_of(const Product& g, int task) {
    const int grp = task / g.tiles, t = task - grp * g.tiles;
    int bi, bj;
    if (KIND == kGram || KIND == kSquare) {  // row by row of the triangle
        bi = (int)((__fsqrt_rn(8.f * t + 1.f) - 1.f) * 0.5f);
        while (bi * (bi + 1) / 2 > t) bi--;
        while ((bi + 1) * (bi + 2) / 2 <= t) bi++;
        bj = t - bi * (bi + 1) / 2;
    } else {
        bj = t / g.tiles_i;
        bi = t - bj * g.tiles_i;
    }
    return Tile{grp, bi * BM, bj * BN, bi == bj};
}

// Where element (r, c) of an image of rows of BN results is.  Columns are exchanged in pieces of 16 by bits of the row, so that
// eight rows of a column, and the rows that the halves of a wave write at once, fall on different banks.
template <int BN>
__device__ __forceinline__ int place(int r, int c) {
    return r * BN + (c ^ (((((r >> 3) & 3) << 4) ^ (((r >> 2) & 1) << 5)) & (BN - 1)));
}
// A block of 32 x 32 results, as the matrix units leave it, to its place.
template <int BN>
__device__ __forceinline__ void to_image(uint32_t* img, const f32x16& acc, int r0, int c0) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < 16; k++) img[place<BN>(r0 + (k >> 2) * 8 + (lane >> 5) * 4 + (k & 3), c0 + (lane & 31))] = __float_as_uint(acc[k]);
}

// Eight results side by side to two pieces of 16 bytes.
__device__ __forceinline__ void put_pairs(_Float16* to, int64_t plane, const uint32_t (&p)[8]) {
    u32x4 hi, lo;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        hi[k] = __builtin_amdgcn_perm(p[2 * k + 1], p[2 * k], 0x05040100u);
        lo[k] = __builtin_amdgcn_perm(p[2 * k + 1], p[2 * k], 0x07060302u);
    }
    *reinterpret_cast<u32x4*>(to) = hi;
    *reinterpret_cast<u32x4*>(to + plane) = lo;
}

// An image of BM x BN results, complete in LDS, to where it belongs: first as fp32, row by row; pairs are left in the same places,
// which the transpose is written from.
template <int BM, int BN, int THREADS, Kind KIND>
__device__ __forceinline__ void emit(const Shape& s, const Args& args, const Product& g, int grp, int exponent, int i0, int j0, bool diagonal, uint32_t* img) {
    constexpr int kChunks = BN / 8;
#pragma unroll 2
    for (int e = threadIdx.x; e < BM * kChunks; e += THREADS) {
        const int r = e / kChunks, c = (e - r * kChunks) * 8, i = i0 + r, j = j0 + c;
        u32x4* from = reinterpret_cast<u32x4*>(img + place<BN>(r, c));  // (pieces of 16 columns stay together)
        const u32x4 raw[2] = {from[0], from[1]};
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; k++) v[k] = __uint_as_float(raw[k >> 2][k & 3]);
        if (KIND == kLast) {
            if (i >= g.rows || j >= g.cols) continue;
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] = ldexpf(v[k], exponent - 24);
            const int64_t first = (int64_t)grp * s.R * s.K + (int64_t)i * s.K + j;
            if ((s.K & 7) == 0)
                finish_eight(s, args, first, v);
            else
                for (int k = 0; k < 8 && j + k < g.cols; k++) finish_one(s, args, first + k, v[k]);
            continue;
        }
        const bool in = i < g.rows && j < g.out.ld;
        u32x4 ah = {}, al = {};
        if (KIND == kSquare && in) {
            const _Float16* a = g.p.hi + grp * g.p.step + (int64_t)i * g.p.ld + j;
            ah = *reinterpret_cast<const u32x4*>(a);
            al = *reinterpret_cast<const u32x4*>(a + g.p.plane);
        }
        uint32_t p[8];
#pragma unroll
        for (int k = 0; k < 8; k++) {
            float w = KIND == kSquare ? v[k] * (1.f / kScale) : ldexpf(v[k], exponent - 12);
            if (KIND == kSquare) {
                const uint32_t hw = ah[k >> 1] >> ((k & 1) * 16), lw = al[k >> 1] >> ((k & 1) * 16);
                w = kC * w + (kB * (of_half(hw & 0xffffu) + of_half(lw & 0xffffu)) + (i == j + k ? kA * kScale : 0.f));
            }
            p[k] = i < g.rows && j + k < g.cols ? pack_pair(w) : 0u;
        }
        from[0] = u32x4{p[0], p[1], p[2], p[3]};
        from[1] = u32x4{p[4], p[5], p[6], p[7]};
        if (in) put_pairs(g.out.hi + grp * g.out.step + (int64_t)i * g.out.ld + j, g.out.plane, p);
    }
    if (KIND == kLast || (KIND != kUpdate && diagonal)) return;
    __syncthreads();
    const Pair turn = KIND == kUpdate ? g.turn : g.out;
#pragma unroll 2
    for (int e = threadIdx.x; e < BN * (BM / 8); e += THREADS) {
        // four pieces of eight rows side by side, then the columns
        const int piece4 = e & 3, rest = e >> 2, c = rest % BN, r = (rest / BN) * 32 + piece4 * 8, i = i0 + r, j = j0 + c;
        if (j >= g.cols || i >= turn.ld) continue;
        uint32_t p[8];
#pragma unroll
        for (int k = 0; k < 8; k++) p[k] = img[place<BN>(r + k, c)];
        put_pairs(turn.hi + grp * turn.step + (int64_t)j * turn.ld + i, turn.plane, p);
    }
}

// One tile of results, or one part of its sum, per workgroup.  Both planes of both operands are loaded straight into LDS, SUB
// times 32 summands at a time, a whole stage ahead of their use.  Rows of
// 64 bytes lie four to a line of all banks; a 16-byte piece c of row r lies at place c ^ (r / 4) % 4, so that the pieces that
// eight rows read together fall on different banks.
template <class F, Kind KIND>
__global__ __launch_bounds__(F::kThreads) void k_product(Shape s, Args args, Product g) {
    constexpr int BM = F::BM, BN = F::BN, SUB = F::SUB, TM = F::TM, TN = F::TN, kThreads = F::kThreads;
    constexpr int kOpA = F::kOpA, kOpB = F::kOpB, kPart = F::kPart, kStage = F::kStage;
    constexpr int kTimesA = BM * 4 / kThreads, kTimesB = BN * 4 / kThreads;  // 16-byte pieces of a thread in a plane
    // (two arrays, not one: the compiler has to see that loads into the one do not concern reads of the other)
    __shared__ __align__(16) unsigned char first_buffer[kStage], second_buffer[kStage];

    const unsigned seq = tile::xcd_sequence();
    const int task = seq / g.splits, split = seq - task * g.splits;
    const Tile at_tile = tile_of<BM, BN, KIND>(g, task);
    const int grp = at_tile.grp, i0 = at_tile.i0, j0 = at_tile.j0, exponent = exponent_of<KIND>(g, grp);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / F::WJ * (TM * 32), wj = wave % F::WJ * (TN * 32);

    // 16-byte pieces of this thread in a plane of a step; rows past the end are the last one again
    auto piece = [&](int q, int first, int rows, int ld) {
        const int at = tid + q * kThreads, r = at >> 2, c = (at & 3) ^ ((r >> 2) & 3);
        const int row = first + r < rows ? r : rows - 1 - first;
        return (uint32_t)row * (uint32_t)ld * 2u + (uint32_t)c * 16u;
    };
    uint32_t va[kTimesA], vb[kTimesB];
#pragma unroll
    for (int q = 0; q < kTimesA; q++) va[q] = piece(q, i0, g.rows, g.p.ld);
#pragma unroll
    for (int q = 0; q < kTimesB; q++) vb[q] = piece(q, j0, g.cols, g.q.ld);
    const _Float16* pa = g.p.hi + grp * g.p.step + (int64_t)i0 * g.p.ld;
    const _Float16* pb = g.q.hi + grp * g.q.step + (int64_t)j0 * g.q.ld;
    const tile::rsrc_t ra[2] = {whole_memory(pa), whole_memory(pa + g.p.plane)};
    const tile::rsrc_t rb[2] = {whole_memory(pb), whole_memory(pb + g.q.plane)};
    const int all = g.depth / kDepth, begin = (int)((int64_t)all * split / g.splits), end = (int)((int64_t)all * (split + 1) / g.splits);
    auto load = [&](int first, unsigned char* buffer) {
#pragma unroll
        for (int u = 0; u < SUB; u++) {
            if (first + u >= end) break;
            unsigned char* to = buffer + u * kPart + wave * 1024;
            const int k = (first + u) * (kDepth * 2);
#pragma unroll
            for (int h = 0; h < 2; h++) {
#pragma unroll
                for (int q = 0; q < kTimesA; q++) load_to_lds(ra[h], to + h * kOpA + q * (kThreads * 16), va[q], k);
#pragma unroll
                for (int q = 0; q < kTimesB; q++) load_to_lds(rb[h], to + 2 * kOpA + h * kOpB + q * (kThreads * 16), vb[q], k);
            }
        }
    };

    // (products that add to one block of results wait for each other: with one block per wave the three pairings go apart)
    constexpr int kChains = TM * TN == 1 ? 3 : 1;
    f32x16 acc[TM][TN] = {}, apart[kChains - 1 ? kChains - 1 : 1] = {};
    // the operands of 16 summands: half of those of one part of a stage
    struct Operands {
        half8 a[TM][2], b[TN][2];
    };
    auto read = [&](const unsigned char* buffer, int unit, Operands& o) {
        const unsigned char* at = buffer + (unit >> 1) * kPart;
        const int c = (unit & 1) * 2 + (lane >> 5);
#pragma unroll
        for (int x = 0; x < TM; x++) {
            const int r = wi + x * 32 + (lane & 31);
#pragma unroll
            for (int h = 0; h < 2; h++) o.a[x][h] = *reinterpret_cast<const half8*>(at + h * kOpA + r * 64 + ((c ^ ((r >> 2) & 3)) << 4));
        }
#pragma unroll
        for (int y = 0; y < TN; y++) {
            const int r = wj + y * 32 + (lane & 31);
#pragma unroll
            for (int h = 0; h < 2; h++) o.b[y][h] = *reinterpret_cast<const half8*>(at + 2 * kOpA + h * kOpB + r * 64 + ((c ^ ((r >> 2) & 3)) << 4));
        }
    };
    auto multiply = [&](const Operands& o) {
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int y = 0; y < TN; y++) {
                f32x16 &first = kChains == 3 ? apart[0] : acc[x][y], &second = kChains == 3 ? apart[kChains / 2] : acc[x][y];
                first = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.a[x][1], o.b[y][0], first, 0, 0, 0);
                second = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.a[x][0], o.b[y][1], second, 0, 0, 0);
                acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.a[x][0], o.b[y][0], acc[x][y], 0, 0, 0);
            }
    };
    constexpr int kUnits = 2 * SUB;
    Operands o[2];
    // One stage, `now` its buffer: each unit's products run while the next one's operands are read; before the last unit
    // everybody has read this buffer and the next stage has arrived, so the one behind that is asked for.
    auto stage = [&](int step, unsigned char* now, unsigned char* next) {
#pragma unroll
        for (int unit = 0; unit < kUnits; unit++) {
            if (unit + 1 < kUnits) {
                read(now, unit + 1, o[(unit + 1) & 1]);
            } else {
                loads_arrived();
                load(step + 2 * SUB, now);
                read(next, 0, o[0]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (step + unit / 2 < end) multiply(o[unit & 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    load(begin, first_buffer);
    load(begin + SUB, second_buffer);
    loads_arrived();
    read(first_buffer, 0, o[0]);
    for (int step = begin; step < end; step += 2 * SUB) {
        stage(step, first_buffer, second_buffer);
        if (step + SUB >= end) break;
        stage(step + SUB, second_buffer, first_buffer);
    }
    loads_arrived();
    if (kChains == 3) acc[0][0] += apart[0] + apart[kChains / 2];

    if (!(KIND == kGram || KIND == kSquare) || g.splits == 1) {
        uint32_t* img = reinterpret_cast<uint32_t*>(first_buffer);
#pragma unroll 1
        for (int r0 = 0; r0 < BM; r0 += F::kRows) {
            if (r0) __syncthreads();
#pragma unroll
            for (int x = 0; x < TM; x++) {
                const int r = wi + x * 32 - r0;
                if (r < 0 || r >= F::kRows) continue;
#pragma unroll
                for (int y = 0; y < TN; y++) to_image<BN>(img, acc[x][y], r, wj + y * 32);
            }
            __syncthreads();
            emit<F::kRows, BN, kThreads, KIND>(s, args, g, grp, exponent, i0 + r0, j0, at_tile.diagonal, img);
        }
        return;
    }
    f32x4* mine = g.parts + ((int64_t)task * g.splits + split) * (BM * BN / 4) + tid;
#pragma unroll
    for (int x = 0; x < TM; x++)
#pragma unroll
        for (int y = 0; y < TN; y++)
#pragma unroll
            for (int q = 0; q < 4; q++)
                mine[((x * TN + y) * 4 + q) * kThreads] = f32x4{acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
}

// Adds the parts of 32 x 32 results, each of four waves every fourth part, and finishes them.
template <class F, Kind KIND>
__global__ __launch_bounds__(256) void k_add(Shape s, Args args, Product g) {
    constexpr int kBlocks = F::BM / 32 * (F::BN / 32), kEach = F::BM * F::BN / 4;
    __shared__ f32x4 sums[4][4][64];
    __shared__ __align__(16) uint32_t img[32 * 32];
    const int task = blockIdx.x / kBlocks, block = blockIdx.x - task * kBlocks, bi = block / (F::BN / 32), bj = block - bi * (F::BN / 32);
    const Tile at = tile_of<F::BM, F::BN, KIND>(g, task);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the block in the registers of the product's workgroup
    const int owner = bi / F::TM * F::WJ + bj / F::TN, x = bi % F::TM, y = bj % F::TN;
    const f32x4* from = g.parts + (int64_t)task * g.splits * kEach + (x * F::TN + y) * 4 * F::kThreads + owner * 64 + lane;
    f32x4 acc[4] = {};
#pragma unroll 4
    for (int part = wave; part < g.splits; part += 4)
#pragma unroll
        for (int q = 0; q < 4; q++) acc[q] += from[(int64_t)part * kEach + q * F::kThreads];
#pragma unroll
    for (int q = 0; q < 4; q++) sums[wave][q][lane] = acc[q];
    __syncthreads();
    const f32x4 v = sums[0][wave][lane] + sums[1][wave][lane] + sums[2][wave][lane] + sums[3][wave][lane];
#pragma unroll
    for (int e = 0; e < 4; e++) img[place<32>(wave * 8 + (lane >> 5) * 4 + e, lane & 31)] = __float_as_uint(v[e]);
    __syncthreads();
    emit<32, 32, 256, KIND>(s, args, g, at.grp, exponent_of<KIND>(g, at.grp), at.i0 + bi * 32, at.j0 + bj * 32, at.diagonal, img);
}

// Symmetric products of few rows: 32 x 32 results per workgroup, the sum over k shared out among its eight waves, which load their
// operands straight into registers, kAhead steps at a time, and add up through LDS.  A lane takes 32 bytes of a row per step (which
// k's a lane holds does not matter as long as both operands agree).
constexpr int kSlimWaves = 8, kAhead = 4;
template <Kind KIND>
__global__ __launch_bounds__(64 * kSlimWaves) void k_slim(Shape s, Args args, Product g) {
    __shared__ f32x4 sums[kSlimWaves][4][64];
    __shared__ __align__(16) uint32_t img[32 * 32];
    const Tile at = tile_of<32, 32, KIND>(g, (int)tile::xcd_sequence());
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ri = at.i0 + (lane & 31), rj = at.j0 + (lane & 31), k0 = (lane >> 5) * 16;
    const _Float16* pi = g.p.hi + at.grp * g.p.step + (int64_t)(ri < g.rows ? ri : g.rows - 1) * g.p.ld + k0;
    const _Float16* pj = g.q.hi + at.grp * g.q.step + (int64_t)(rj < g.cols ? rj : g.cols - 1) * g.q.ld + k0;
    const int all = g.depth / kDepth, begin = all * wave / kSlimWaves, end = all * (wave + 1) / kSlimWaves;
    f32x16 acc[3] = {};
    for (int step = begin; step < end; step += kAhead) {
        half8 a[kAhead][2][2], b[kAhead][2][2];
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            if (step + u >= end) break;
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int64_t o = (int64_t)(step + u) * kDepth + k * 8;
                a[u][k][0] = *reinterpret_cast<const half8*>(pi + o);
                a[u][k][1] = *reinterpret_cast<const half8*>(pi + o + g.p.plane);
                b[u][k][0] = *reinterpret_cast<const half8*>(pj + o);
                b[u][k][1] = *reinterpret_cast<const half8*>(pj + o + g.q.plane);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            if (step + u >= end) break;
#pragma unroll
            for (int k = 0; k < 2; k++) {
                acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[u][k][1], b[u][k][0], acc[0], 0, 0, 0);
                acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[u][k][0], b[u][k][1], acc[1], 0, 0, 0);
                acc[2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[u][k][0], b[u][k][0], acc[2], 0, 0, 0);
            }
        }
    }
    acc[2] += acc[0] + acc[1];
#pragma unroll
    for (int q = 0; q < 4; q++) sums[wave][q][lane] = f32x4{acc[2][4 * q], acc[2][4 * q + 1], acc[2][4 * q + 2], acc[2][4 * q + 3]};
    __syncthreads();
    if (wave < 4) {
        f32x4 v = sums[0][wave][lane];
#pragma unroll
        for (int w = 1; w < kSlimWaves; w++) v += sums[w][wave][lane];
#pragma unroll
        for (int e = 0; e < 4; e++) img[place<32>(wave * 8 + (lane >> 5) * 4 + e, lane & 31)] = __float_as_uint(v[e]);
    }
    __syncthreads();
    emit<32, 32, 64 * kSlimWaves, KIND>(s, args, g, at.grp, exponent_of<KIND>(g, at.grp), at.i0, at.j0, at.diagonal, img);
}

uint64_t up256(uint64_t v) { return (v + 255) & ~(uint64_t)255; }
// Whether two steps are taken at a time.  Measured, us of five steps one by one and so:
//   2048 x 8192   1766, 1437    1536 x 6144   999, 822    1024 x 4096   411, 377    512 x 4608   225, 200    256 x 2304   128, 122
//   2048 x 4096   1143, 1063    1536 x 3000   651, 603    1024 x 2048   297, 308    512 x 2048   160, 160    256 x 512    104, 108
//   two of 512 x 2048   206, 211    two of 420 x 4741   320, 262    eight of 256 x 2304   237, 203
bool by_twos(const Shape& s) { return s.n >= (s.m > 1024 ? 2 : s.m > 512 ? 4 : 5) * s.m; }
unsigned blocks(int64_t n, int64_t per) { return (unsigned)((n + per - 1) / per); }
int padded(int64_t n) { return (int)((n + kDepth - 1) / kDepth * kDepth); }

// How a product is cut.
struct Cut {
    int side = 0, tiles_i = 0, tiles_j = 0, tiles = 0;  // of the tiles; 32: k_slim
    int splits = 1;                                     // parts of the sum
};
// Measured with the ways forced, us of one product; "128 in 3" is a side and the parts of the sum:
//   rows x summands, symmetric:   512 x 512      32: 7, 64 in 4: 10          256 x 2304    64 in 12: 9, 128 in 8: 13, 32: 19
//                                 512 x 4608     64 in 7: 17, 128 in 8: 21   1024 x 4096   128 in 7: 28, 64 in 2: 31
//                                 1536 x 6144    128 in 3: 69, 64: 100       2048 x 8192   256 in 7: 118, 128 in 3: 133
//   rows x columns x summands:    512 x 4608 x 512     64: 20, 128: 21, 256: 43   1024 x 4096 x 1024   128: 38, 64: 42, 256: 71
//                                 1536 x 6144 x 1536   256: 115, 128: 130         2048 x 8192 x 2048   256: 190, 128: 233
Cut cut_of(bool symmetric, int64_t rows, int64_t cols, int64_t depth, int64_t G) {
    Cut c;
    auto tiles = [&](int side) {
        c.side = side;
        c.tiles_i = (int)((rows + side - 1) / side);
        c.tiles_j = (int)((cols + side - 1) / side);
        c.tiles = symmetric ? c.tiles_i * (c.tiles_i + 1) / 2 : c.tiles_i * c.tiles_j;
        return c.tiles * G;
    };
    // (a tile that mostly hangs over the edges is work for nothing)
    auto full = [&](double share) { return (double)rows * cols >= share * c.side * c.side * c.tiles_i * c.tiles_j; };
    const int64_t steps = depth / kDepth;
    if (!symmetric) {
        // the larger side as soon as it gives more than half of the compute units a tile
        if (!(tiles(256) >= 140 && full(0.75)) && !(tiles(128) >= 192 && full(0.6))) tiles(64);
        return c;
    }
    if (steps <= 24 && tiles(32) <= 256) return c;  // short sums: as many compute units as there are blocks of 32
    int64_t t = tiles(256);
    if (full(0.75) && (t >= 200 || (t >= 25 && steps >= 192))) {
        c.splits = t >= 128 ? 1 : (int)(256 / t);
        return c;
    }
    // Parts of a sum cost a launch and their way through memory (4 us and more): as many as give every compute unit one.
    t = tiles(128);
    if (full(0.6) && t * steps >= 3500) {
        c.splits = (int)std::max<int64_t>(1, std::min(t > 128 ? 512 / t : 256 / t, steps / 16));
        return c;
    }
    t = tiles(64);
    c.splits = (int)std::max<int64_t>(1, std::min<int64_t>(280 / t, steps / 6));
    return c;
}

template <class F, Kind KIND>
void launch(const Shape& s, const Args& a, const Product& g, hipStream_t stream) {
    CANVAS_LAUNCH((k_product<F, KIND>), dim3((unsigned)(g.tiles * g.splits * s.G)), dim3(F::kThreads), 0, stream, s, a, g);
    if constexpr (KIND == kGram || KIND == kSquare) {
        if (g.splits > 1) CANVAS_LAUNCH((k_add<F, KIND>), dim3((unsigned)(g.tiles * s.G) * (F::BM / 32 * (F::BN / 32))), dim3(256), 0, stream, s, a, g);
    }
}
template <Kind KIND>
void product(const Shape& s, const Args& a, Product g, hipStream_t stream) {
    constexpr bool kSymmetric = KIND == kGram || KIND == kSquare;
    const Cut c = cut_of(kSymmetric, g.rows, g.cols, g.depth, s.G);
    g.tiles_i = c.tiles_i;
    g.tiles_j = c.tiles_j;
    g.tiles = c.tiles;
    g.splits = c.splits;
    if constexpr (kSymmetric) {
        if (c.side == 32) {
            CANVAS_LAUNCH(k_slim<KIND>, dim3((unsigned)(g.tiles * s.G)), dim3(64 * kSlimWaves), 0, stream, s, a, g);
            return;
        }
    }
    if (c.side == 256)
        launch<Large, KIND>(s, a, g, stream);
    else if (c.side == 128)
        launch<Middle, KIND>(s, a, g, stream);
    else
        launch<Small, KIND>(s, a, g, stream);
}

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    if (small_plan(s).fits) {
        p.small = true;
        p.launches = 1;
        p.workspace_bytes = 256;  // (unused: callers of every plan pass one)
        return p;
    }
    p.parts = (int)((s.R * s.K + 16 * kThreads - 1) / (16 * kThreads));
    if (p.parts > 1024) p.parts = 1024;
    p.launches = 2;
    p.workspace_bytes = up256(8ull * s.G * p.parts);
    if (!s.steps) return p;
    // (256 x 256 results take 512 threads, less 256; symmetric products have few tiles where there are many matrices)
    auto longest = [&](const Cut& c) { p.workgroups = std::max(p.workgroups, (int64_t)c.tiles * s.G * (c.side == 256 ? 2 : 1)); };
    p.workgroups = (int64_t)blocks(s.K, 64) * blocks(s.R, 64);
    longest(cut_of(false, s.m, s.n, padded(s.m), s.G));
    if (s.tall) longest(cut_of(false, s.n, s.m, padded(s.m), s.G));
    const Cut gram = cut_of(true, s.m, s.m, padded(s.n), s.G), square = cut_of(true, s.m, s.m, padded(s.m), s.G);
    for (const Cut& c : {gram, square})
        if (c.splits > 1) p.part_bytes = std::max<uint64_t>(p.part_bytes, 4ull * c.side * c.side * c.tiles * c.splits * s.G);
    const int twos = by_twos(s) ? s.steps / 2 : 0, ones = s.steps - twos;
    p.launches += ones * (2 + (gram.splits > 1)) + (ones + 4 * twos) * (1 + (square.splits > 1));
    p.workspace_bytes += up256(4ull * s.G) + 2 * up256(4ull * s.G * s.m * padded(s.n)) + 2 * up256(4ull * s.G * s.n * padded(s.m)) + 3 * up256(4ull * s.G * s.m * padded(s.m)) + up256(p.part_bytes);
    return p;
}

void step(const Shape& s, const Plan& p, const Args& a, hipStream_t stream) {
    if (p.small) return step_small(s, a, stream);
    char* at = a.ws;
    auto take = [&](uint64_t bytes) {
        char* r = at;
        at += up256(bytes);
        return r;
    };
    auto pair = [&](int64_t rows, int64_t cols) {
        Pair q;
        q.ld = padded(cols);
        q.plane = rows * q.ld;
        q.step = 2 * q.plane;
        q.hi = (_Float16*)take(4ull * s.G * q.plane);
        return q;
    };
    double* sums = (double*)take(8ull * s.G * p.parts);
    f32x4* parts = (f32x4*)take(p.part_bytes);
    int* ups = s.steps ? (int*)take(4ull * s.G) : nullptr;
    const unsigned G = (unsigned)s.G;
    CANVAS_LAUNCH(k_mix, dim3(p.parts, G), dim3(kThreads), 0, stream, s, a, sums);
    if (!s.steps) {
        CANVAS_LAUNCH(k_normalised, dim3(blocks(s.R * s.K, kThreads), G), dim3(kThreads), 0, stream, s, a, sums, p.parts);
        return;
    }
    Pair x[2] = {pair(s.m, s.n), pair(s.m, s.n)}, xt[2] = {pair(s.n, s.m), pair(s.n, s.m)}, q = pair(s.m, s.m), b = pair(s.m, s.m), t = pair(s.m, s.m);
    CANVAS_LAUNCH(k_start, dim3(blocks(s.K, 64) * blocks(s.R, 64), G), dim3(kThreads), 0, stream, s, a, sums, p.parts, ups, x[0], xt[0]);
    const int m = (int)s.m, n = (int)s.n;
    // C = P Q of symmetric matrices that commute
    auto both = [&](const Pair& p, const Pair& q, const Pair& c) { product<kGram>(s, a, Product{p, q, m, m, p.ld, c, c, 0, 0, 0, 0, parts}, stream); };
    auto polynomial = [&](const Pair& q, const Pair& b) { product<kSquare>(s, a, Product{q, q, m, m, q.ld, b, b, 0, 0, 0, 0, parts}, stream); };
    for (int k = 0, at = 0; k < s.steps; k++, at ^= 1) {
        const Pair &from = x[at], &from_t = xt[at], &to = x[at ^ 1], &to_t = xt[at ^ 1];
        const int grown = grown_by(k);
        product<kGram>(s, a, Product{from, from, m, m, from.ld, q, q, 0, 0, 0, 0, parts, ups, grown}, stream);
        polynomial(q, b);
        Pair left = b;
        if (by_twos(s) && k + 1 < s.steps) {
            both(b, q, t);
            both(t, b, q);  // the second step's A
            polynomial(q, t);
            both(t, b, q);
            left = q;
            k++;
        }
        if (k + 1 < s.steps)
            product<kUpdate>(s, a, Product{left, from_t, m, n, left.ld, to, to_t, 0, 0, 0, 0, parts, ups, grown, grown_by(k + 1)}, stream);
        else if (s.tall)
            product<kLast>(s, a, Product{from_t, left, n, m, left.ld, to, to_t, 0, 0, 0, 0, parts, ups, grown}, stream);
        else
            product<kLast>(s, a, Product{left, from_t, m, n, left.ld, to, to_t, 0, 0, 0, 0, parts, ups, grown}, stream);
    }
}

}  // namespace ortho
}  // namespace canvas
