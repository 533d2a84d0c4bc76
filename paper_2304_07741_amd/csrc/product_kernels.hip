// Products whose results are plain matrices, the ends of their sums, and copies of operands.
#include "product_kernels.hpp"

#include <algorithm>

#include "device_util.hpp"
#include "launch.hpp"
#include "product_device.hpp"
#include "tile_util.hpp"

namespace canvas {
namespace product {
namespace {

// What a kernel takes of a product.
struct Job {
    Factor a, b;
    int64_t depth, tiles_i, tiles_j, ld;
    int segments, results, splits;
    void* out[2];
    f32x4* parts;
    bool first;
};

// Where element (r, c) of an image of rows of BN results is: columns are exchanged in pieces of 16 by bits of the row, so that
// eight rows of a column, and the rows that the halves of a wave write at once, fall on different banks.
template <int BN>
__device__ __forceinline__ int place(int r, int c) {
    return r * BN + (c ^ (((((r >> 3) & 3) << 4) ^ (((r >> 2) & 1) << 5)) & (BN - 1)));
}
template <int BN>
__device__ __forceinline__ void to_image(float* img, const f32x16& acc, int r0, int c0) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < 16; k++) img[place<BN>(r0 + (k >> 2) * 8 + (lane >> 5) * 4 + (k & 3), c0 + (lane & 31))] = acc[k];
}

// Results (i, j ..) from an image of ROWS x BN of them to memory, rounded where they are bf16.
template <bool F32, int ROWS, int BN, int THREADS>
__device__ __forceinline__ void emit(const Job& g, int which, int64_t i0, int64_t j0, const float* img) {
    const bool whole = (g.ld & 7) == 0;
#pragma unroll 2
    for (int e = threadIdx.x; e < ROWS * (BN / 8); e += THREADS) {
        const int r = e / (BN / 8), c = (e - r * (BN / 8)) * 8;
        const int64_t i = i0 + r, j = j0 + c;
        if (i >= g.a.count || j >= g.b.count) continue;
        const f32x4* from = reinterpret_cast<const f32x4*>(img + place<BN>(r, c));  // (pieces of 16 columns stay together)
        const f32x4 v[2] = {from[0], from[1]};
        const int64_t at = i * g.ld + j;
        if (F32) {
            float* to = static_cast<float*>(g.out[which]) + at;
            if (whole && j + 8 <= g.b.count) {
                reinterpret_cast<f32x4*>(to)[0] = v[0];
                reinterpret_cast<f32x4*>(to)[1] = v[1];
            } else {
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (j + k < g.b.count) to[k] = v[k >> 2][k & 3];
            }
        } else {
            uint16_t* to = static_cast<uint16_t*>(g.out[which]) + at;
            if (whole && j + 8 <= g.b.count) {
                *reinterpret_cast<u32x4*>(to) = u32x4{tile::pack_bf16(v[0][0], v[0][1]), tile::pack_bf16(v[0][2], v[0][3]), tile::pack_bf16(v[1][0], v[1][1]), tile::pack_bf16(v[1][2], v[1][3])};
            } else {
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (j + k < g.b.count) to[k] = f32_to_bf16(v[k >> 2][k & 3]);
            }
        }
    }
}

template <class F, Side SA>
__device__ __forceinline__ void run(const Job& g, int64_t number, const Buffers<F>& buffers) {
    constexpr int TM = F::TM, TN = F::TN, BM = F::BM, BN = F::BN;
    const Place at = place_of(number, g.tiles_i, g.tiles_j, g.splits, g.results);
    if (!at.inside) return;
    const int64_t i0 = at.i * BM, j0 = at.j * BN;
    const int per = (int)((g.depth + F::BK - 1) / F::BK), all = per * g.segments;
    const int begin = (int)((int64_t)all * at.split / g.splits), end = (int)((int64_t)all * (at.split + 1) / g.splits);
    f32x16 acc[TM][TN] = {};
    accumulate<F, SA, kCols, false>(g.a, g.b, at.which, i0, j0, g.depth, begin, end, per, g.segments, buffers, acc);
    if (g.parts) {
        f32x4* mine = g.parts + (((at.which * g.tiles_i + at.i) * g.tiles_j + at.j) * g.splits + at.split) * (BM * BN / 4) + threadIdx.x;
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int y = 0; y < TN; y++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    f32x4 v = {acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
                    f32x4* to = mine + ((x * TN + y) * 4 + q) * F::kThreads;
                    if (!g.first) v += *to;
                    *to = v;
                }
        return;
    }
    // through LDS, kRows rows of results to a buffer
    constexpr int kFit = F::kStage / (BN * 4) / 32 * 32, kRows = kFit < BM / 2 ? kFit : BM / 2, kRound = 2 * kRows;
    static_assert(BM % kRound == 0, "rows of results in the buffers");
    const int wave = threadIdx.x >> 6, wi = wave / F::WJ * (TM * 32), wj = wave % F::WJ * (TN * 32);
#pragma unroll 1
    for (int r0 = 0; r0 < BM; r0 += kRound) {
        if (r0) tile::lds_barrier();
#pragma unroll
        for (int x = 0; x < TM; x++) {
            const int r = wi + x * 32 - r0;
            if (r < 0 || r >= kRound) continue;
#pragma unroll
            for (int y = 0; y < TN; y++) to_image<BN>(reinterpret_cast<float*>(buffers.of(r / kRows)), acc[x][y], r % kRows, wj + y * 32);
        }
        tile::lds_barrier();
#pragma unroll
        for (int n = 0; n < 2; n++) emit<F::PLANES == 3, kRows, BN, F::kThreads>(g, at.which, i0 + r0 + n * kRows, j0, reinterpret_cast<const float*>(buffers.at[n]));
    }
}

// Two products in one launch, the first with rows of the summed index along it.  (Neither waits for the other, and small ones do not fill the chip.)
// Bound by the matrix units: the gradients of 4096 x 2048 x 2 * 8192 bf16 in 500 us (1.1 PFLOP/s), of 1500 x 1000 x 2 * 2731 fp32 in 192 (171 TFLOP/s of fp32 results).
template <class F>
__global__ __launch_bounds__(F::kThreads, 2) void k_products(Job first, Job second, int64_t firsts) {
    PRODUCT_BUFFERS(F, buffers);
    // each XCD takes its eighth of the first product's tiles, then its share of the second's (they may take twice as long as the others)
    const unsigned total = gridDim.x * gridDim.y, lin = blockIdx.y * gridDim.x + blockIdx.x, xcd = lin & 7u, n = (unsigned)firsts;
    auto before = [&](unsigned all) { return xcd * (all >> 3) + (xcd < (all & 7u) ? xcd : (all & 7u)); };
    const unsigned mine = (n >> 3) + (xcd < (n & 7u)), at = lin >> 3;
    if (at < mine)
        run<F, kRows>(first, before(n) + at, buffers);
    else
        run<F, kCols>(second, before(total) - before(n) + at - mine, buffers);
}
template <class F, Side SA>
__global__ __launch_bounds__(F::kThreads, 2) void k_product(Job g) {
    PRODUCT_BUFFERS(F, buffers);
    run<F, SA>(g, tile::xcd_sequence(), buffers);
}

// Adds the parts of 32 x 32 results, each of four waves every fourth part, and finishes them.  Bound by memory, mostly the last-level cache: four parts of 4096 x 2048, 151 MB in 20 us.
template <class F>
__device__ __forceinline__ void join(const Job& g, int64_t number, f32x4 (&sums)[4][4][64], float* img) {
    constexpr int kBlocks = F::BM / 32 * (F::BN / 32), kEach = F::BM * F::BN / 4;
    const int64_t tile = number / kBlocks, tiles = g.tiles_i * g.tiles_j;
    if (tile >= tiles * g.results) return;
    const int block = (int)(number - tile * kBlocks), bi = block / (F::BN / 32), bj = block - bi * (F::BN / 32);
    const int which = (int)(tile / tiles);
    const int64_t ti = (tile - which * tiles) / g.tiles_j, tj = tile - which * tiles - ti * g.tiles_j;
    const int64_t i0 = ti * F::BM + bi * 32, j0 = tj * F::BN + bj * 32;
    if (i0 >= g.a.count || j0 >= g.b.count) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the block in the registers of the product's workgroup
    const int owner = bi / F::TM * F::WJ + bj / F::TN, x = bi % F::TM, y = bj % F::TN;
    const f32x4* from = g.parts + tile * g.splits * kEach + (x * F::TN + y) * 4 * F::kThreads + owner * 64 + lane;
    f32x4 acc[4] = {};
#pragma unroll 4
    for (int part = wave; part < g.splits; part += 4)
#pragma unroll
        for (int q = 0; q < 4; q++) acc[q] += from[(int64_t)part * kEach + q * F::kThreads];
#pragma unroll
    for (int q = 0; q < 4; q++) sums[wave][q][lane] = acc[q];
    __syncthreads();
    const f32x4 v = (sums[0][wave][lane] + sums[1][wave][lane]) + (sums[2][wave][lane] + sums[3][wave][lane]);
#pragma unroll
    for (int e = 0; e < 4; e++) img[place<32>(wave * 8 + (lane >> 5) * 4 + e, lane & 31)] = v[e];
    __syncthreads();
    emit<F::PLANES == 3, 32, 32, 256>(g, which, i0, j0, img);
}
template <class F>
__global__ __launch_bounds__(256) void k_join(Job first, Job second, int64_t firsts) {
    __shared__ f32x4 sums[4][4][64];
    __shared__ __align__(16) float img[32 * 32];
    const int64_t number = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (number < firsts)
        join<F>(first, number, sums, img);
    else
        join<F>(second, number - firsts, sums, img);
}

struct Copies {
    Copy c[3];
};
// Eight columns per thread and turn; bound by memory: fp32 to planes, 70 MB in 18 us.
template <bool F32>
__global__ __launch_bounds__(256) void k_copy(Copies all) {
    const Copy& c = all.c[blockIdx.y];
    const int64_t wide = padded(F32, c.cols) / 8, n = c.rows * wide, ld = pitch(F32, c.cols);
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < n; k += (int64_t)gridDim.x * 256) {
        const int64_t row = k / wide, col = (k - row * wide) * 8;
        copy8<F32>(c.from, c.cols, row, col, !c.live || c.live[row], c.to + row * ld);
    }
}

Job job_of(const Product& p) {
    return Job{p.a, p.b, p.depth, p.cut.tiles_i, p.cut.tiles_j, p.ld, p.segments, p.results, p.cut.splits, {p.out[0], p.out[1]}, reinterpret_cast<f32x4*>(p.parts), p.first};
}
int64_t workgroups(const Product& p) { return p.cut.tiles() * p.cut.splits * p.results; }
// Of the launch that adds the parts of a product; none if it leaves none, or others add to them.
template <class F>
int64_t joins(const Product& p) { return p.parts && p.last ? p.cut.tiles() * p.results * (F::BM / 32 * (F::BN / 32)) : 0; }

}  // namespace

// What a form costs, in us: a stage of a workgroup where a few compute units have one, where each has one, and where each has two or three (`slots`), and
// the beginning and the end of a tile.  Measured, us of rows x columns x summands without parts, for tiles of 256, 128, 64, and in fp32 of 128, 64:
//   256 x 256 x 4096      77   33   23    130   51      1024 x 1024 x 4096    80   48   26    136   63      2048 x 2048 x 4096    80   56   60    158  217
//   2048 x 4096 x 4096    86   66  109    290  483      4096 x 4096 x 4096   106  136  222    551  701      4096 x 4096 x 256     18   20   29     48   61
// in four parts: 1024 x 1024 x 4096    33   27   26     52   60
// fp32's 128 x 256 are for long sums over many tiles (4096^3: 247 TFLOP/s, 128 x 128 reach 191; 512 summands: 212 and 188).  Where they are taken by this rule, us
// with and without them: 4096 x 1024 x 2 * 4096 forward 353 and 380, 3000 x 1500 x 2 * 3900 both ways 1207 and 1237, a head of 256 x 1024 x 32000 475 and 490.
struct Speed {
    int side, high, depth, slots;
    double few, one, two, three, ends;
};
constexpr Speed kSpeeds[2][3] = {{{256, 256, 64, 1, 1.15, 1.6, 0, 0, 8.0}, {128, 128, 64, 2, 0.55, 0.80, 0.95, 0, 4.8}, {64, 64, 64, 3, 0.34, 0.36, 0.43, 0.51, 2.6}},
                                 {{256, 128, 32, 1, 1.5, 2.05, 0, 0, 8.0}, {128, 128, 16, 2, 0.51, 0.60, 1.10, 0, 4.8}, {64, 64, 32, 2, 0.39, 0.46, 0.82, 0, 1.0}}};

// The best way of a form, and what it takes.
Cut cut_with(const Speed& v, int64_t rows, int64_t cols, int64_t depth, int results, bool may_split, double& least) {
    Cut c;
    c.side = v.side;
    c.high = v.high;
    c.tiles_i = (rows + v.high - 1) / v.high;
    c.tiles_j = (cols + v.side - 1) / v.side;
    const int64_t tiles = c.tiles() * results, steps = (depth + v.depth - 1) / v.depth;
    // `n` workgroups at a time
    auto turn = [&](int64_t n, double stages) {
        const double at[4] = {v.few, v.one, v.two, v.three};
        const int k = (int)((n - 1) / 256);
        const double share = (double)(n - k * 256) / 256;
        return stages * (at[k] + (at[k + 1] - at[k]) * share) + v.ends * (0.4 + 0.6 * n / (256.0 * v.slots));
    };
    least = 0;
    Cut best = c;
    for (int splits = 1; splits <= 32; splits += splits < 4 ? 1 : splits < 8 ? 2 : splits / 4) {
        if (splits > 1 && (!may_split || tiles * splits > 1024 || steps / splits < 2)) break;
        const double each = (double)((steps + splits - 1) / splits);
        const int64_t all = tiles * splits, slots = 256 * v.slots, rest = all % slots;
        double t = (double)(all / slots) * turn(slots, each) + (rest ? turn(rest, each) : 0);
        // parts of a sum: a launch, and their way to memory and back
        if (splits > 1) t += 4 + 0.15e-6 * 4 * v.high * v.side * (double)all;
        if (!least || t < least) {
            least = t;
            best.splits = splits;
        }
    }
    return best;
}

Cut cut_of(bool f32, int64_t rows, int64_t cols, int64_t depth, int results, bool may_split, double* us) {
    Cut best;
    double least = 0, t;
    for (const Speed& v : kSpeeds[f32]) {
        const Cut c = cut_with(v, rows, cols, depth, results, may_split, t);
        if (!least || t < least) {
            least = t;
            best = c;
        }
    }
    if (us) *us = least;
    return best;
}

void cuts_of(bool f32, const Size& x, const Size& y, Cut& cx, Cut& cy) {
    double least = 0;
    for (const Speed& v : kSpeeds[f32])
        for (const Speed& w : kSpeeds[f32]) {
            double tx, ty;
            const Cut a = cut_with(v, x.rows, x.cols, x.depth, x.results, true, tx), b = cut_with(w, y.rows, y.cols, y.depth, y.results, true, ty);
            const double t = tx + ty + (v.side == w.side ? 0 : 4);  // (a launch more)
            if (!least || t < least) {
                least = t;
                cx = a;
                cy = b;
            }
        }
}

uint64_t parts_bytes(const Cut& c, int results, bool several) {
    return c.splits > 1 || several ? 4ull * c.high * c.side * c.tiles() * c.splits * results : 0;
}
bool together(const Product& x, const Product& y) { return x.cut.side == y.cut.side && x.a_rows && !y.a_rows; }
int launches_of(const Cut& x, const Cut& y, bool several) {
    const bool jx = x.splits > 1 || several, jy = y.splits > 1;
    return x.side == y.side ? 1 + (jx || jy) : 2 + jx + jy;
}

void multiply(const Product& p, hipStream_t stream) {
    with_form(p.f32, p.cut.side, [&](auto form) {
        using F = decltype(form);
        const Job t = job_of(p);
        const dim3 grid = rows_of_workgroups(workgroups(p), F::kThreads);
        if (p.a_rows)
            CANVAS_LAUNCH((k_product<F, kRows>), grid, dim3(F::kThreads), 0, stream, t);
        else
            CANVAS_LAUNCH((k_product<F, kCols>), grid, dim3(F::kThreads), 0, stream, t);
        if (const int64_t n = joins<F>(p)) CANVAS_LAUNCH((k_join<F>), rows_of_workgroups(n, 256), dim3(256), 0, stream, t, t, n);
    });
}
void multiply(const Product& x, const Product& y, hipStream_t stream) {
    if (!together(x, y)) {
        multiply(x, stream);
        multiply(y, stream);
        return;
    }
    with_form(x.f32, x.cut.side, [&](auto form) {
        using F = decltype(form);
        const Job t = job_of(x), u = job_of(y);
        CANVAS_LAUNCH((k_products<F>), rows_of_workgroups(workgroups(x) + workgroups(y), F::kThreads), dim3(F::kThreads), 0, stream, t, u, workgroups(x));
        const int64_t nx = joins<F>(x), ny = joins<F>(y);
        if (nx + ny) CANVAS_LAUNCH((k_join<F>), rows_of_workgroups(nx + ny, 256), dim3(256), 0, stream, t, u, nx);
    });
}

void copy(bool f32, const Copy* copies, int n, hipStream_t stream) {
    Copies all{};
    int64_t most = 0;
    for (int i = 0; i < n; i++) {
        all.c[i] = copies[i];
        most = std::max(most, copies[i].rows * padded(f32, copies[i].cols) / 8);
    }
    const dim3 grid((unsigned)std::min<int64_t>((most + 255) / 256, 4096), (unsigned)n);
    if (f32)
        CANVAS_LAUNCH(k_copy<true>, grid, dim3(256), 0, stream, all);
    else
        CANVAS_LAUNCH(k_copy<false>, grid, dim3(256), 0, stream, all);
}

}  // namespace product
}  // namespace canvas
