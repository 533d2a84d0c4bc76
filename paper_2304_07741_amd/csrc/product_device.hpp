// The inner part of a product: a tile of results in the registers of a workgroup, both operands through LDS.
//
// Operands are loaded straight into LDS, BUFFERS - 1 stages (of BK summands of all rows of the tile) ahead of their use.
// Rows along k: 16-byte pieces of eight summands; piece c of row r lies at place c ^ (r / rows per line of all banks), so that the
// pieces that 16 lanes read together fall on different banks.  Rows of k: the matrix units want eight summands of one index in a lane, so the
// rows are read by the transposing load, a block of 4 summands x 16 indexes by 16 lanes; the 32-byte units of row k lie at unit ^
// {0, 2, 5, 7}[k % 4] ({0, 0, 2, 2} where a line of all banks holds two rows), for the same reason.  What lies behind the end of the sum is not loaded: an offset outside the buffer gives zeros, which
// stages behind the last one load too, so that the number of loads in flight is always the same.
// By itself, results left in registers' order, 4096 x 4096 x 4096: 256 x 256 about 1350 TFLOP/s for rows along k and of k alike, at 1.65 to 1.75 GHz, which is what the chip holds under
// that load (a library's product 1412); fp32 by 128 x 128 191 to 247, by 128 x 256 247 to 255 (154).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "launch.hpp"
#include "product_kernels.hpp"
#include "tile_util.hpp"

namespace canvas {
namespace product {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
using tile::bf16x8_t;
using tile::u32x4;

enum Side { kRows, kCols };

// Tiles of BM x BN by WI x WJ waves, BK summands of PLANES planes at a time.
// (Kernels ask for two waves of each SIMD unit: the registers of one wave that takes more would keep a second workgroup of 128 x 128 in fp32 off its compute unit.)
template <int BM_, int BN_, int WI_, int WJ_, int PLANES_, int BK_, int BUFFERS_>
struct Form {
    static constexpr int BM = BM_, BN = BN_, WI = WI_, WJ = WJ_, PLANES = PLANES_, BK = BK_, BUFFERS = BUFFERS_;
    static constexpr int kThreads = 64 * WI * WJ, TM = BM / WI / 32, TN = BN / WJ / 32, kUnits = BK / 16;
    static constexpr int kBytesA = BM * BK * 2, kBytesB = BN * BK * 2;  // of a plane of a stage
    static constexpr int kStage = PLANES * (kBytesA + kBytesB), kLoadsA = PLANES * kBytesA / 16 / kThreads, kLoadsB = PLANES * kBytesB / 16 / kThreads, kLoads = kLoadsA + kLoadsB;  // of a thread
    static constexpr bool kApart = kUnits > 1;  // the two operands' loads go to different units of products
};
using Large = Form<256, 256, 2, 4, 1, 64, 2>;
using Middle = Form<128, 128, 2, 2, 1, 64, 2>;
using Small = Form<64, 64, 2, 2, 1, 64, 3>;
using Wide = Form<128, 256, 2, 4, 3, 32, 2>;
using Triple = Form<128, 128, 2, 2, 3, 16, 3>;
using SmallTriple = Form<64, 64, 2, 2, 3, 32, 3>;

// f with the form that a cut asks for
template <class F>
void with_form(bool f32, int side, F f) {
    if (f32 && side == 256)
        f(Wide());
    else if (f32 && side == 128)
        f(Triple());
    else if (f32)
        f(SmallTriple());
    else if (side == 256)
        f(Large());
    else if (side == 128)
        f(Middle());
    else
        f(Small());
}

// One array per stage in flight, not one for all: the compiler has to see that loads into the one do not concern reads of another.
template <class F>
struct Buffers {
    unsigned char* at[4];
    // (an array that is indexed by a variable would be kept in memory)
    __device__ __forceinline__ unsigned char* of(int n) const { return n == 0 ? at[0] : n == 1 ? at[1] : n == 2 ? at[2] : at[3]; }
};
#define PRODUCT_BUFFERS(F, name)                                                                                                                  \
    __shared__ __align__(16) unsigned char name##_0[F::kStage], name##_1[F::kStage], name##_2[F::BUFFERS > 2 ? F::kStage : 16], name##_3[F::BUFFERS > 3 ? F::kStage : 16]; \
    const ::canvas::product::Buffers<F> name{{name##_0, name##_1, name##_2, name##_3}}

constexpr uint32_t kOutside = 0x80000000u;  // an offset behind the end of every buffer
__device__ __forceinline__ tile::rsrc_t buffer_from(const void* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffff, 0x00020000); }
// 16 bytes per lane to LDS, lane after lane behind `to` (the same for the whole wave).
__device__ __forceinline__ void load_to_lds(tile::rsrc_t from, unsigned char* to, uint32_t offset) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 0);
}
// A barrier behind which everybody has read what it asked LDS for, and all but each thread's last N loads to LDS have arrived.
template <int N>
__device__ __forceinline__ void loads_arrived() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x70);  // vmcnt(N), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int ROW>
__device__ __forceinline__ int piece_of(int r, int c) { return c ^ ((r / (256 / ROW)) & (ROW / 16 - 1)); }
template <int ROW>
__device__ __forceinline__ int unit_of(int k, int unit) {
    static_assert(ROW >= 128, "four units in a row at least");
    return unit ^ (ROW == 128 ? k & 2 : ((k & 1) << 1) | ((k >> 1) & 1) * 5);
}

// What a thread loads of one operand.  PAIRS: indexes are taken 32 by 32 from the two matrices in turn.
template <class F, int BX, Side SIDE, bool PAIRS>
struct Loader {
    static constexpr int kRow = SIDE == kRows ? F::BK * 2 : BX * 2, kPieces = kRow / 16;
    static constexpr int kPlane = BX * F::BK * 2, kTimes = kPlane / 16 / F::kThreads;
    static_assert(kPlane % (16 * F::kThreads) == 0 && 256 % (SIDE == kRows ? kRow : 1) == 0, "whole pieces for every thread");
    uint32_t offset[kTimes];
    int behind;  // summands of a stage before this thread's, in its first piece; kApart more in each of the others
    static constexpr int kApart = SIDE == kRows ? 0 : F::kThreads / kPieces;
    static_assert(SIDE == kCols || kTimes == 1 || F::kThreads / kPieces % (256 / kRow * kPieces) == 0, "a thread's pieces are at the same place of their rows");
    const uint16_t *at, *other;  // what the next load begins with; in the second matrix of a pair

    static __device__ __forceinline__ int row_of(int tid, int q) { return (tid + q * F::kThreads) / kPieces; }
    static __device__ __forceinline__ int place_of(int tid, int q) { return (tid + q * F::kThreads) % kPieces; }

    static __device__ __forceinline__ uint32_t bytes_of(int piece) { return (uint32_t)column<F::PLANES>(piece * 8, 0) * 2u; }
    // The tile from index `first` on, the sum from k on.
    __device__ __forceinline__ void seek(const Factor& f, int which, int64_t first, int64_t k) {
        const int64_t from = SIDE == kRows ? first * f.ld + k * F::PLANES : first * F::PLANES + k * f.ld;  // (whole pieces of 16)
        at = (!PAIRS && which ? f.p[1] : f.p[0]) + from;
        if (PAIRS) other = f.p[1] + from;
    }
    __device__ __forceinline__ void begin(const Factor& f, int64_t first) {
        const int left = (int)(f.count - first < BX ? f.count - first : BX);  // indexes of the tile
        behind = SIDE == kRows ? piece_of<SIDE == kRows ? kRow : 256>(row_of(threadIdx.x, 0), place_of(threadIdx.x, 0)) * 8 : row_of(threadIdx.x, 0);
#pragma unroll
        for (int q = 0; q < kTimes; q++) {
            const int r = row_of(threadIdx.x, q), c = place_of(threadIdx.x, q);
            if (SIDE == kRows) {
                int row = PAIRS ? (r >> 6) * 32 + (r & 31) : r;
                row = row < left ? row : left - 1;  // (behind the last one: that one again, for results that nobody keeps)
                offset[q] = (uint32_t)row * (uint32_t)f.ld * 2u + bytes_of(piece_of<SIDE == kRows ? kRow : 256>(r, c));
            } else {
                const int piece = unit_of<SIDE == kRows ? 256 : kRow>(r, c >> 1) * 2 + (c & 1);
                offset[q] = piece * 8 < left ? (uint32_t)r * (uint32_t)f.ld * 2u + bytes_of(piece) : kOutside;
            }
        }
    }
    // The next BK summands, of which there are `left`.
    __device__ __forceinline__ void load(const Factor& f, int64_t left, unsigned char* to) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        to += wave * 1024;
        const int some = left < F::BK ? (int)left : F::BK;
#pragma unroll
        for (int h = 0; h < F::PLANES; h++)
#pragma unroll
            for (int q = 0; q < kTimes; q++) {
                const bool second = PAIRS && ((((wave * 64 + q * F::kThreads) / kPieces) >> 5) & 1);
                load_to_lds(buffer_from((second ? other : at) + h * 16), to + h * kPlane + q * (F::kThreads * 16), behind < some - q * kApart ? offset[q] : kOutside);
            }
        const int64_t step = SIDE == kRows ? F::BK * F::PLANES : F::BK * f.ld;
        at += step;
        if (PAIRS) other += step;
    }
};

// Where a lane reads its operands: of block x of 32 indexes, 16 summands from unit u on.  The exchange of places is an exclusive or of bits that
// the unit (rows along k) or the block (rows of k) has to itself, so that the other one is a constant added to the address.
template <class F, int BX, Side SIDE, int T>
struct Reader {
    static constexpr int kRow = SIDE == kRows ? F::BK * 2 : BX * 2, kPlane = BX * F::BK * 2, kKept = SIDE == kRows ? F::kUnits : T;
    int at[kKept];
    __device__ __forceinline__ void begin(int base) {  // base: the wave's first index, a multiple of 32 T
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int n = 0; n < kKept; n++) {
            if (SIDE == kRows) {
                const int r = base + (lane & 31);
                at[n] = r * kRow + piece_of<SIDE == kRows ? kRow : 256>(r, n * 2 + (lane >> 5)) * 16;
            } else {
                const int j = lane & 15, g = lane >> 4;
                at[n] = ((g >> 1) * 8 + (j >> 2)) * kRow + unit_of<SIDE == kRows ? 256 : kRow>(j >> 2, (base + n * 32) / 16 + (g & 1)) * 32 + (j & 3) * 8;
            }
        }
    }
    __device__ __forceinline__ bf16x8_t read(const unsigned char* plane, int x, int unit) const {
        bf16x8_t v;
        if (SIDE == kRows) {
            v = *reinterpret_cast<const bf16x8_t*>(plane + at[SIDE == kRows ? unit : 0] + x * (32 * kRow));
        } else {
            typedef __attribute__((address_space(3))) s16x4* Lds;
            const unsigned char* p = plane + at[SIDE == kRows ? 0 : x] + unit * (16 * kRow);
            const s16x4 two[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p), __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 4 * kRow))};
            __builtin_memcpy(&v, two, 16);
        }
        return v;
    }
};

template <int N, int END, class F>
__device__ __forceinline__ void turn(F&& f) {
    if constexpr (N < END) {
        f(std::integral_constant<int, N>());
        turn<N + 1, END>(f);
    }
}
template <int N, int END, class F>
__device__ __forceinline__ void rest(int left, F&& f) {  // N .. left - 1
    if constexpr (N + 1 < END) {
        if (N >= left) return;
        f(std::integral_constant<int, N>());
        rest<N + 1, END>(left, f);
    }
}

// The sum over steps begin .. end (BK summands each, `per` of them in each of `segments` halves) of a tile from (i0, j0) on.  acc[x][y]: 32 x 32
// results from (wave's row + 32 x, wave's column + 32 y) on; register k of a lane is row (k / 4) * 8 + (lane / 32) * 4 + k % 4, column lane % 32.
template <class F, Side SA, Side SB, bool PAIRS>
__device__ __forceinline__ void accumulate(const Factor& a, const Factor& b, int which, int64_t i0, int64_t j0, int64_t depth, int begin, int end, int per,
                                           int segments, const Buffers<F>& buffers, f32x16 (&acc)[F::TM][F::TN]) {
    constexpr int TM = F::TM, TN = F::TN, P = F::PLANES, N = F::BUFFERS;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Loader<F, F::BM, SA, false> la;
    Loader<F, F::BN, SB, PAIRS> lb;
    la.begin(a, i0);
    lb.begin(b, j0);
    Reader<F, F::BM, SA, TM> ra;
    Reader<F, F::BN, SB, TN> rb;
    ra.begin(wave / F::WJ * (TM * 32));
    rb.begin(wave % F::WJ * (TN * 32));
    const int half = segments == 2 && begin >= per, from = segments == 2 ? half : which;
    la.seek(a, from, i0, (int64_t)(begin - half * per) * F::BK);
    lb.seek(b, from, j0, (int64_t)(begin - half * per) * F::BK);
    // what is left of the sum, or of its half, from a step on
    auto left = [&](int step) { return step < end ? depth - (int64_t)(segments == 2 && step >= per ? step - per : step) * F::BK : 0; };
    auto load_a = [&](int step, unsigned char* to) {
        la.load(a, left(step), to);
        if (segments == 2 && step + 1 == per) la.seek(a, 1, i0, 0);
    };
    auto load_b = [&](int step, unsigned char* to) {
        lb.load(b, left(step), to + P * F::kBytesA);
        if (segments == 2 && step + 1 == per) lb.seek(b, 1, j0, 0);
    };
    struct Operands {
        bf16x8_t a[TM][P], b[TN][P];
    };
    auto read = [&](const unsigned char* buffer, int unit, Operands& o) {
#pragma unroll
        for (int h = 0; h < P; h++) {
#pragma unroll
            for (int x = 0; x < TM; x++) o.a[x][h] = ra.read(buffer + h * F::kBytesA, x, unit);
#pragma unroll
            for (int y = 0; y < TN; y++) o.b[y][h] = rb.read(buffer + P * F::kBytesA + h * F::kBytesB, y, unit);
        }
    };
    // Products of other planes than the first have a sum of their own: the large sum is rounded once for 16 summands, not six times.  Off in the mean, a gated
    // pair of 3320 summands: 5e-7 instead of 1.4e-6; gradients of a head of 16 x 1624 x 1023: 7e-7 instead of 1.7e-6; for half a percent of the time.
    f32x16 low[TM][TN] = {};
    auto multiply = [&](const Operands& o) {
        // pairings of planes, the smallest products first; what is left out is 2^-24 of a term at most (split)
        constexpr int kPairings = P == 1 ? 1 : 6, kOfA[6] = {2, 0, 1, 1, 0, 0}, kOfB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int h = 0; h < kPairings; h++)
#pragma unroll
            for (int x = 0; x < TM; x++)
#pragma unroll
                for (int y = 0; y < TN; y++) {
                    f32x16& sum = h + 1 < kPairings ? low[x][y] : acc[x][y];
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(o.a[x][P == 1 ? 0 : kOfA[h]], o.b[y][P == 1 ? 0 : kOfB[h]], sum, 0, 0, 0);
                }
    };
    constexpr int kPerProduct = 2;  // reads of LDS
    Operands o[2];
    // Stage n of a turn: each unit's products run while the next one's operands are read; before the last unit everybody has
    // read this buffer and the next stage has arrived, so this buffer takes the stage BUFFERS behind: its first
    // operand in that unit, its second one in the next.  (Loads are spread over the products: asked for together they keep the wave, and the matrix
    // units, waiting for their queue.)
    auto stage = [&](int step, auto number) {
        constexpr int n = decltype(number)::value, first = n * F::kUnits;
        unsigned char *now = buffers.at[n % N], *next = buffers.at[(n + 1) % N], *before = buffers.at[(n + N - 1) % N];
#pragma unroll
        for (int unit = 0; unit < F::kUnits; unit++) {
            Operands &mine = o[(first + unit) & 1], &then = o[(first + unit + 1) & 1];
            constexpr int kProducts = TM * TN * (P == 1 ? 1 : 6), kReads = P * (TM * (SA == kRows ? 1 : 2) + TN * (SB == kRows ? 1 : 2));
            const bool last = unit + 1 == F::kUnits;
            if (last) loads_arrived<(N - 2) * F::kLoads>();
            __builtin_amdgcn_sched_barrier(0);
            read(last ? next : now, last ? 0 : unit + 1, then);
            if (unit == 0 && F::kApart) load_b(step + n + N - 1, before);
            if (last) load_a(step + n + N, now);
            if (last && !F::kApart) load_b(step + n + N, now);
            multiply(mine);
            // products all the time, what is asked for between them
#pragma unroll
            for (int k = 0; k < kProducts; k++) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                if (k * kPerProduct < kReads) __builtin_amdgcn_sched_group_barrier(0x100, kPerProduct, 0);
                if (k < (last ? F::kLoadsA + (F::kApart ? 0 : F::kLoadsB) : unit == 0 ? F::kLoadsB : 0)) __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int n = 0; n < N; n++) {
        load_a(begin + n, buffers.at[n]);
        if (n + 1 < N || !F::kApart) load_b(begin + n, buffers.at[n]);
    }
    loads_arrived<(N - 1) * F::kLoads - (F::kApart ? F::kLoadsB : 0)>();
    read(buffers.at[0], 0, o[0]);
    constexpr int kTurn = (F::kUnits & 1) && (N & 1) ? 2 * N : N;  // stages until buffers and registers are the first ones again
    int step = begin;
    for (; step + kTurn <= end; step += kTurn) turn<0, kTurn>([&](auto n) { stage(step, n); });
    rest<0, kTurn>(end - step, [&](auto n) { stage(step, n); });
    loads_arrived<0>();
    if (P > 1) {
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int y = 0; y < TN; y++) acc[x][y] += low[x][y];
    }
}

// A value as the sum of three bf16 numbers: what is left of it rounded to nearest, twice, and the rest, which eight bits hold (but for what lies below the smallest
// of bf16's numbers).  The second is 2^-8 of the value at most and the third 2^-17, of either sign, so that what a product leaves out of the nine, 2^-24 of it at most, adds up to
// nothing.  Cut where rounding would make an infinity.  Not finite: the first alone.
__device__ __forceinline__ void split(float v, uint16_t (&part)[3]) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7f800000u) == 0x7f800000u) {
        part[0] = (uint16_t)(u >> 16);
        part[0] = (u & 0x7fffffu) ? (uint16_t)(part[0] | 0x40u) : part[0];
        part[1] = part[2] = 0;
        return;
    }
    const uint32_t near = (u + 0x8000u) & 0xffff0000u, top = (near & 0x7f800000u) == 0x7f800000u ? u & 0xffff0000u : near;
    const float r = v - __uint_as_float(top);
    const uint32_t mid = (__float_as_uint(r) + 0x8000u) & 0xffff0000u;
    part[0] = (uint16_t)(top >> 16);
    part[1] = (uint16_t)(mid >> 16);
    part[2] = (uint16_t)(__float_as_uint(r - __uint_as_float(mid)) >> 16);
}

// Columns col .. col + 7 of a row of a matrix, to the row of its copy (`to`): zeros behind the last column, and where the row is not kept.
template <bool F32>
__device__ __forceinline__ void copy8(const void* matrix, int64_t cols, int64_t row, int64_t col, bool keep, uint16_t* to) {
    constexpr int P = F32 ? 3 : 1;
    u32x4 w[P] = {};
    if (keep && col < cols) {
        const bool whole = (cols & 7) == 0;
        if (F32) {
            const float* x = static_cast<const float*>(matrix) + row * cols + col;
            float v[8];
            if (whole) {
                const f32x4 a = reinterpret_cast<const f32x4*>(x)[0], b = reinterpret_cast<const f32x4*>(x)[1];
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = a[e], v[4 + e] = b[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = col + e < cols ? x[e] : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                uint16_t lo[3], hi[3];
                split(v[2 * e], lo);
                split(v[2 * e + 1], hi);
#pragma unroll
                for (int h = 0; h < P; h++) w[h][e] = lo[h] | (uint32_t)hi[h] << 16;
            }
        } else {
            const uint16_t* x = static_cast<const uint16_t*>(matrix) + row * cols + col;
            if (whole) {
                w[0] = *reinterpret_cast<const u32x4*>(x);
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) w[0][e] = (col + 2 * e < cols ? x[2 * e] : 0) | (uint32_t)(col + 2 * e + 1 < cols ? x[2 * e + 1] : 0) << 16;
            }
        }
    }
#pragma unroll
    for (int h = 0; h < P; h++) *reinterpret_cast<u32x4*>(to + column<P>(col, h)) = w[h];
}

// Tile t of a launch's order: bands of kBand tiles of rows, down each column of a band, in the order of the XCDs, so that the tiles that an XCD works on at a
// time share their operands in its L2.
constexpr int kBand = 8;
struct Place {
    int64_t i, j;
    int which, split;
    bool inside;
};
__device__ __forceinline__ Place place_of(int64_t t, int64_t tiles_i, int64_t tiles_j, int splits, int results) {
    const int64_t tiles = tiles_i * tiles_j;
    Place p;
    p.inside = t < tiles * splits * results;
    p.split = (int)(t / (tiles * results));
    t -= p.split * (tiles * results);
    p.which = (int)(t / tiles);
    t -= p.which * tiles;
    const int64_t band = t / (kBand * tiles_j), rows = tiles_i - band * kBand < kBand ? tiles_i - band * kBand : kBand;
    t -= band * (kBand * tiles_j);
    p.j = t / rows;
    p.i = band * kBand + (t - p.j * rows);
    return p;
}

}  // namespace product
}  // namespace canvas
