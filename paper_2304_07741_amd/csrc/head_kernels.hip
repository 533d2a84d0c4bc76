// Log probabilities of given tokens from features and the head's weight.
//
// Forward: tiles of logits that never leave the registers.  Classes are the rows of a tile and the rows of x its columns, so that a lane
// has the classes of its tile for one or two rows of x; it takes their largest logit m, S = sum exp(z - z_m) and sum exp(z - z_m) (z - z_m), joins them with the
// other half of the wave, and leaves them to a second launch that joins the segments of all classes in a fixed order.
// Backward: a piece of the classes at a time, a tile of logits is read, or computed again by the same sums in the same order as in forward, and becomes their gradients in bf16 (three planes of them in fp32
// plans), rows of x by classes; dx is the sum over all pieces' products with W, dW of the piece one product with x.
#include "head_kernels.hpp"

#include <algorithm>

#include "../../include/canvas_head.h"
#include "device_util.hpp"
#include "exp_util.hpp"
#include "few_device.hpp"
#include "launch.hpp"
#include "product_device.hpp"
#include "tile_util.hpp"
#include "wave_util.hpp"

namespace canvas {
namespace head {
namespace {

using product::f32x16;
using product::f32x4;
using product::Factor;
using product::Form;
using tile::u32x4;

constexpr float kInf = __builtin_inff(), kLowest = -3.402823466e38f;

// e^x of one logit's x = (logit - most) * it, at most 0, and x itself in the unit that the exponential is taken in, not below -300 of it (NaN stays in the
// former).  bf16 plans: powers of two by one multiplication, whose argument is rounded by up to 2^-24 of itself; fp32 plans to about a unit of the last place.
template <bool F32>
struct Exp {
    float scale;
    // (the largest number in the place of a temperature that log2(e) takes past it)
    __device__ __forceinline__ explicit Exp(float it) : scale(F32 ? it : fminf(it * kLog2e, 3.402823466e38f)) {}
    __device__ __forceinline__ float of(float logit, float most, float& x) const {
        const float d = (logit - most) * scale;
        x = fmaxf(d, -300.f);
        return F32 ? exp_finite(d < -300.f ? -300.f : d) : __builtin_amdgcn_exp2f(d);
    }
    static constexpr float kUnit = F32 ? 1.f : kLn2;
};

// The sums of some logits of one row, x = (logit - most) * it: e^x added up, and e^x x.
struct Sums {
    float most, s, t;
};
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float it) {
    const Exp<true> power(it);
    Sums r;
    r.most = fmaxf(a.most, b.most);
    float xa, xb;
    const float ea = power.of(a.most, r.most, xa), eb = power.of(b.most, r.most, xb);
    r.s = fmaf(a.s, ea, b.s * eb);
    r.t = fmaf(ea, fmaf(a.s, xa, a.t), eb * fmaf(b.s, xb, b.t));
    return r;
}
template <int O>
__device__ __forceinline__ float from_lane(float v) { return __shfl_xor(v, O); }

// Bytes that are not zero for those of four classes from c on (a multiple of four) that are classes and that the mask allows.
__device__ __forceinline__ uint32_t allowed4(const uint8_t* mask, int64_t c, int64_t classes) {
    if (c + 4 <= classes) return mask ? *reinterpret_cast<const uint32_t*>(mask + c) : 0x01010101u;
    uint32_t w = 0;
#pragma unroll 1
    for (int e = 3; e >= 0; e--) w = w << 8 | (c + e < classes ? mask ? mask[c + e] : 1u : 0u);
    return w;
}

struct FwdArgs {
    Factor w, x;
    int64_t rows, features, classes, tiles_i, tiles_j;
    float it;
    const uint8_t* mask;
    const int64_t* tokens;
    Sums* sums;    // [segments][rows]
    float* token;  // [rows]: the token's logit
    f32x4* kept;   // for backward, those of the first classes, as the tiles' workgroups hold them
    int64_t kept_classes;
};
// A tile's logits, or where they are.
template <class F>
__device__ __forceinline__ f32x4* kept_of(f32x4* kept, int64_t tile) { return kept + tile * (F::BM * F::BN / 4) + threadIdx.x; }

// N logits of one row of x in a lane, the sums of those and of what the lanes LOW, 2 LOW, .. 32 apart hold.
template <int N, int LOW, bool F32>
__device__ __forceinline__ Sums sums_of(const float (&z)[N], float it) {
    const Exp<F32> power(it);
    Sums r{kLowest, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < N; k++) r.most = fmaxf(r.most, z[k]);
    if (LOW <= 16) r.most = fmaxf(r.most, from_lane<16>(r.most));
    r.most = fmaxf(r.most, from_lane<32>(r.most));
#pragma unroll
    for (int k = 0; k < N; k++) {
        float x;
        const float e = power.of(z[k], r.most, x);  // (NaN and +inf make both sums NaN)
        r.s += e;
        r.t = fmaf(e, x, r.t);
    }
    r.t *= power.kUnit;
    if (LOW <= 16) {
        r.s += from_lane<16>(r.s);
        r.t += from_lane<16>(r.t);
    }
    r.s += from_lane<32>(r.s);
    r.t += from_lane<32>(r.t);
    return r;
}

// Bound by the matrix units; a tile's exponentials, and the logits that are kept, are not hidden by another tile where one fills its compute unit.
// 4096 x 1024 x 32768 bf16: 272 us (1.01 PFLOP/s), 315 with 537 MB of logits kept; 4096 x 4096 x 32768, which keeps them, 914 (1.2); 1500 x 1000 x 50021 170 us, 4.6 rounds of tiles of 256.  (With a branch
// per register for the token's logit instead of selections 345.)
template <class F>
__global__ __launch_bounds__(F::kThreads, 2) void k_logits(FwdArgs a) {
    constexpr int TM = F::TM, TN = F::TN;
    PRODUCT_BUFFERS(F, buffers);
    const product::Place at = product::place_of(tile::xcd_sequence(), a.tiles_i, a.tiles_j, 1, 1);
    if (!at.inside) return;
    const int64_t i0 = at.i * F::BM, j0 = at.j * F::BN;
    const int steps = (int)((a.features + F::BK - 1) / F::BK);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c0 = i0 + wave / F::WJ * (TM * 32) + (lane >> 5) * 4, t0 = j0 + wave % F::WJ * (TN * 32) + (lane & 31);
    int token[TN];  // the row's token among this lane's classes, -1 if it is not
#pragma unroll
    for (int y = 0; y < TN; y++) {
        token[y] = -1;
        if (a.token && t0 + y * 32 < a.rows) {
            const int64_t c = a.tokens[t0 + y * 32] - c0;
            if (c >= 0 && c < TM * 32 && !(c & 4)) token[y] = (int)c;
        }
    }
    f32x16 acc[TM][TN] = {};
    product::accumulate<F, product::kRows, product::kRows, false>(a.w, a.x, 0, i0, j0, a.features, 0, steps, steps, 1, buffers, acc);
    if (i0 < a.kept_classes) {
        f32x4* to = kept_of<F>(a.kept, at.i * a.tiles_j + at.j);
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int y = 0; y < TN; y++)
#pragma unroll
                for (int q = 0; q < 4; q++) to[((x * TN + y) * 4 + q) * F::kThreads] = f32x4{acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
    }
    if (a.mask || i0 + F::BM > a.classes) {
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const uint32_t in = allowed4(a.mask, c0 + x * 32 + q * 8, a.classes);
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (!(in >> (8 * e) & 0xffu)) {
#pragma unroll
                        for (int y = 0; y < TN; y++) acc[x][y][q * 4 + e] = -kInf;
                    }
            }
    }
#pragma unroll
    for (int y = 0; y < TN; y++) {
        const int64_t t = t0 + y * 32;
        if (__any(token[y] >= 0)) {
            float v = 0.f;
#pragma unroll
            for (int x = 0; x < TM; x++)
#pragma unroll
                for (int k = 0; k < 16; k++) v = token[y] == x * 32 + (k >> 2) * 8 + (k & 3) ? acc[x][y][k] : v;
            if (token[y] >= 0) a.token[t] = v;
        }
        float z[TM * 16];
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int k = 0; k < 16; k++) z[x * 16 + k] = acc[x][y][k];
        const Sums r = sums_of<TM * 16, 32, F::PLANES == 3>(z, a.it);
        if (lane < 32 && t < a.rows) a.sums[(at.i * F::WI + wave / F::WJ) * a.rows + t] = r;
    }
}

struct FewArgs {
    const void *x, *weight;
    int64_t rows, features, classes;
    float it;
    const uint8_t* mask;
    const int64_t* tokens;
    Sums* sums;
    float* token;
    float* logits;  // for backward, [rows][classes to the next multiple of 8]
};
// Blocks of 16 classes of a workgroup.  With 17 rows or more x is as much to read from the L2 as two blocks' weights from memory: four where there are enough of them (32 x 2048 x 131072,
// without LDS between: 122 us instead of 135; 20 x 1000 x 50021 38 and 44; fp32 32 x 1024 x 50000 66 and 70; but 17 x 333 x 3000 12 instead of 10; 24 x 256 x 10000 the same).
constexpr int64_t kManyClasses = 16384;
int few_blocks(int64_t rows, int64_t classes) { return rows > 16 && rows <= few::kRows && classes > kManyClasses ? 4 : 2; }
// Bound by the weight's bytes: 4 x 2048 x 131072 bf16, 537 MB in 95 us, 5.7 TB/s.
template <class T, int NT, int R, bool STAGED>
__global__ __launch_bounds__(few::kThreads) void k_few(FewArgs a) {
    __shared__ f32x4 shared[few::kShared<STAGED, R, NT>];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * (16 * R), mine = few::Lanes<STAGED>::row();
    const T *w[R], *x[NT];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t c = first + r * 16 + mine;
        w[r] = static_cast<const T*>(a.weight) + (c < a.classes ? c : a.classes - 1) * a.features;
    }
#pragma unroll
    for (int n = 0; n < NT; n++) {
        const int64_t t = blockIdx.y * (16 * NT) + n * 16 + mine;
        x[n] = static_cast<const T*>(a.x) + (t < a.rows ? t : a.rows - 1) * a.features;
    }
    // (asked for ahead of the weights: a workgroup's end is short then)
    const int64_t t = blockIdx.y * (16 * NT) + wave * 16 + (lane & 15), c0 = first + (lane >> 4) * 4;
    const bool known = a.token && wave < NT && t < a.rows;
    const int64_t c = known ? a.tokens[t] - c0 : -1;
    uint32_t in[R];
#pragma unroll
    for (int r = 0; r < R; r++) in[r] = wave < NT ? allowed4(a.mask, c0 + r * 16, a.classes) : 0u;
    f32x4 sums[R];
    few::accumulate<STAGED, T, R, NT, few::ahead(R, NT)>(w, x, a.features, sums, shared);
    if (wave >= NT) return;
    float z[R * 4];
#pragma unroll
    for (int r = 0; r < R; r++) {
#pragma unroll
        for (int e = 0; e < 4; e++) z[r * 4 + e] = in[r] >> (8 * e) & 0xffu ? sums[r][e] : -kInf;
    }
    if (a.logits && t < a.rows) {
        float* to = a.logits + t * ((a.classes + 7) & ~(int64_t)7) + c0;
#pragma unroll
        for (int r = 0; r < R; r++)
            if (c0 + r * 16 < a.classes) *reinterpret_cast<f32x4*>(to + r * 16) = f32x4{z[r * 4], z[r * 4 + 1], z[r * 4 + 2], z[r * 4 + 3]};
    }
    if (known) {
#pragma unroll
        for (int k = 0; k < R * 4; k++)
            if (c == (k >> 2) * 16 + (k & 3)) a.token[t] = z[k];
    }
    const Sums r = sums_of<R * 4, 16, sizeof(T) == 4>(z, a.it);
    if (lane < 16 && t < a.rows) a.sums[blockIdx.x * a.rows + t] = r;
}

struct RowArgs {
    int64_t rows, classes;
    int segments, across;  // rows of x by a workgroup: a power of two
    float it;
    const uint8_t* mask;
    const int64_t* tokens;
    const Sums* sums;
    const float* token;
    float *logprob, *entropy;
    Row* row;
};
// Joins the segments of each row: latency of a few dependent loads and lane exchanges; 4 rows of 4096 segments 7.6 us, 4096 of 256 12 us.
__global__ __launch_bounds__(256) void k_rows(RowArgs a) {
    __shared__ Sums part[256];
    const int mine = threadIdx.x & (a.across - 1), turn = threadIdx.x / a.across, turns = 256 / a.across;
    const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.across + mine;
    Sums r{kLowest, 0.f, 0.f};
    if (t < a.rows) {
        constexpr int kAhead = 4;
        for (int k = turn; k < a.segments; k += turns * kAhead) {
            Sums s[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; u++) s[u] = k + u * turns < a.segments ? a.sums[(int64_t)(k + u * turns) * a.rows + t] : Sums{kLowest, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < kAhead; u++) r = join(r, s[u], a.it);
        }
    }
    part[threadIdx.x] = r;
    __syncthreads();
    for (int o = turns / 2; o; o >>= 1) {
        if (turn < o) part[threadIdx.x] = join(part[threadIdx.x], part[threadIdx.x + o * a.across], a.it);
        __syncthreads();
    }
    if (turn || t >= a.rows) return;
    r = part[threadIdx.x];
    const bool empty = r.s == 0.f;  // (the largest of what is left counts one)
    const float log_sum = empty ? -kInf : logf(r.s), entropy = empty ? 0.f : log_sum - r.t / r.s;
    if (a.entropy) a.entropy[t] = entropy;
    if (a.logprob) {
        const int64_t c = a.tokens[t];
        const bool given = c >= 0 && c < a.classes;
        float v = 0.f;
        if (given) {
            // (a row with nothing left, and a masked token in a row of NaN, too)
            const bool hidden = a.mask && !a.mask[c];
            v = empty || hidden ? -kInf : (a.token[t] - r.most) * a.it - log_sum;
        }
        a.logprob[t] = v;
    }
    if (a.row) a.row[t] = Row{r.most, log_sum, entropy, empty ? 0.f : 1.f / r.s};
}

struct SlopeArgs {
    int64_t rows, classes, features;
    float it;
    const int64_t* tokens;
    const float *dlogprob, *dentropy;
    const Row* row;
    Slope* slope;
    const void* x;
    uint16_t* copy;
};
// Slopes of the rows, and x as products read it: with zeros for the rows without a gradient, whose products by the zeros of their logits' gradients are
// zero then, whatever they hold.  A few us: 4096 x 1024 bf16 6.2.
template <bool F32>
__global__ __launch_bounds__(256) void k_slopes(SlopeArgs a) {
    const int64_t wide = product::padded(F32, a.features) / 8, n = a.rows * wide, ld = product::pitch(F32, a.features);
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < n; k += (int64_t)gridDim.x * 256) {
        const int64_t t = k / wide, col = (k - t * wide) * 8;
        const Row r = a.row[t];
        const int64_t c = a.tokens ? a.tokens[t] : -1;
        const bool given = c >= 0 && c < a.classes && a.dlogprob;
        const float g = given ? a.dlogprob[t] * a.it : 0.f, h = a.dentropy ? a.dentropy[t] * a.it : 0.f;
        // p (-g - h (log p + entropy)) with p = e^x / sum, log p = x - log sum
        const bool keep = r.log_sum != -kInf && (g != 0.f || h != 0.f);
        if (col == 0)
            a.slope[t] = Slope{r.most, -r.inverse * (g + h * (r.entropy - r.log_sum)), -r.inverse * h * Exp<F32>::kUnit, g, given ? (int32_t)c : -1, keep ? 0xffffffffu : 0u, {0, 0}};
        product::copy8<F32>(a.x, a.features, t, col, keep, a.copy + t * ld);
    }
}

struct GradArgs {
    Factor w, x;                   // of this piece
    int64_t rows, features, classes, tiles_i, tiles_j;
    int64_t first;                 // class of the piece
    float it;
    const uint8_t* mask;           // of this piece
    const Slope* slope;
    uint16_t* to;                  // [rows][ld], `wide` columns
    int64_t ld, wide;
    f32x4* kept;                   // the piece's logits, where forward has left them
};
// The gradients of a tile of logits.  4096 x 32768 of them in bf16 plans: 172 us from kept logits (805 MB, 4.7 TB/s: one workgroup to a compute unit reads, computes and writes in turn), 289 with their
// product over 1024 features, of which the matrix units are the bound.
template <class F, bool KEPT>
__global__ __launch_bounds__(F::kThreads, 2) void k_grads(GradArgs a) {
    constexpr int TM = F::TM, TN = F::TN, P = F::PLANES, kHalf = F::BN / 2;
    PRODUCT_BUFFERS(F, buffers);
    const product::Place at = product::place_of(tile::xcd_sequence(), a.tiles_i, a.tiles_j, 1, 1);
    if (!at.inside) return;
    const int64_t i0 = at.i * F::BM, j0 = at.j * F::BN;
    const int steps = (int)((a.features + F::BK - 1) / F::BK);
    f32x16 acc[TM][TN] = {};
    if (KEPT) {
        const f32x4* from = kept_of<F>(a.kept, at.i * a.tiles_j + at.j);
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int y = 0; y < TN; y++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const f32x4 v = from[((x * TN + y) * 4 + q) * F::kThreads];
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[x][y][4 * q + e] = v[e];
                }
    } else {
        product::accumulate<F, product::kRows, product::kRows, false>(a.w, a.x, 0, i0, j0, a.features, 0, steps, steps, 1, buffers, acc);
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / F::WJ * (TM * 32) + (lane >> 5) * 4, wj = wave % F::WJ * (TN * 32) + (lane & 31);
    const Exp<P == 3> power(a.it);
#pragma unroll
    for (int y = 0; y < TN; y++) {
        const int64_t t = j0 + wj + y * 32;
        Slope s{};
        s.at = -1;
        if (t < a.rows) s = a.slope[t];
        const int64_t token = s.at - a.first - i0 - wi;
        const int here = s.at >= 0 && token >= 0 && token < TM * 32 && !(token & 4) ? (int)token : -1;
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int k = 0; k < 16; k++) {
                float d;
                const float e = power.of(acc[x][y][k], s.most, d);
                acc[x][y][k] = e * fmaf(s.second, d, s.first);
            }
        if (__any(here >= 0)) {
#pragma unroll
            for (int x = 0; x < TM; x++)
#pragma unroll
                for (int k = 0; k < 16; k++) acc[x][y][k] += here == x * 32 + (k >> 2) * 8 + (k & 3) ? s.token : 0.f;
        }
        if (__any(!s.keep)) {
#pragma unroll
            for (int x = 0; x < TM; x++)
#pragma unroll
                for (int k = 0; k < 16; k++) acc[x][y][k] = s.keep ? acc[x][y][k] : 0.f;
        }
    }
    if (a.mask || i0 + F::BM > a.classes) {
#pragma unroll
        for (int x = 0; x < TM; x++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const uint32_t in = allowed4(a.mask, i0 + wi + x * 32 + q * 8, a.classes);
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (!(in >> (8 * e) & 0xffu)) {
#pragma unroll
                        for (int y = 0; y < TN; y++) acc[x][y][q * 4 + e] = 0.f;
                    }
            }
    }
    // Plane by plane through LDS, rows of x by classes: half of the rows in a buffer.  16-byte pieces
    // of row r are exchanged by the bits of r, so that the lanes of a wave, a row each, write to different banks.
    static_assert(kHalf * F::BM * 2 <= F::kStage, "half a tile in a buffer");
    constexpr int kPieces = F::BM / 8;
#pragma unroll
    for (int h = 0; h < P; h++) {
        if (h) tile::lds_barrier();
        unsigned char* img = buffers.of(wave % F::WJ * (TN * 32) / kHalf);
#pragma unroll
        for (int y = 0; y < TN; y++) {
            const int r = (wj + y * 32) & (kHalf - 1);
#pragma unroll
            for (int x = 0; x < TM; x++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    uint32_t w[2];
                    if (P == 1) {
                        w[0] = tile::pack_bf16(acc[x][y][4 * q], acc[x][y][4 * q + 1]);
                        w[1] = tile::pack_bf16(acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]);
                    } else {
                        uint16_t part[4][3];
#pragma unroll
                        for (int e = 0; e < 4; e++) product::split(acc[x][y][4 * q + e], part[e]);
                        w[0] = part[0][h] | (uint32_t)part[1][h] << 16;
                        w[1] = part[2][h] | (uint32_t)part[3][h] << 16;
                    }
                    const int c = wi + x * 32 + q * 8;  // of the tile, a multiple of 4
                    __builtin_memcpy(img + r * (F::BM * 2) + ((((c >> 3) ^ r) & (kPieces - 1)) << 4) + (c & 4) * 2, w, 8);
                }
        }
        tile::lds_barrier();
#pragma unroll 4
        for (int e = threadIdx.x; e < F::BN * kPieces; e += F::kThreads) {
            const int r = e / kPieces, c = e % kPieces;
            const int64_t t = j0 + r, col = i0 + c * 8;
            if (t >= a.rows || col >= a.wide) continue;
            const u32x4 v = *reinterpret_cast<const u32x4*>(buffers.of(r / kHalf) + (r & (kHalf - 1)) * (F::BM * 2) + (((c ^ r) & (kPieces - 1)) << 4));
            *reinterpret_cast<u32x4*>(a.to + t * a.ld + product::column<P>(col, h)) = v;
        }
    }
}

// The gradients of the logits that forward has kept of few rows, eight per thread.  A tile would compute them by sums in another order than forward's, and a cold distribution
// multiplies what they differ by.  16 x 1024 x 50000 both ways: 112 us (127 with a tile's sums, which read W once more), 32 x 2048 x 131072 488 (568); fp32 16 x 1024 x 50000 320 (386).
struct FewGradArgs {
    const float* logits;
    int64_t rows, classes, all;  // of the piece; of all pieces
    int64_t first;
    float it;
    const uint8_t* mask;         // of this piece
    const Slope* slope;
    uint16_t* to;
    int64_t ld, wide;
};
template <bool F32>
__global__ __launch_bounds__(256) void k_few_grads(FewGradArgs a) {
    constexpr int P = F32 ? 3 : 1;
    const int64_t t = blockIdx.y, col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= a.wide) return;
    const Slope s = a.slope[t];
    u32x4 w[P] = {};
    if (s.keep && col < a.classes) {
        const f32x4* from = reinterpret_cast<const f32x4*>(a.logits + t * ((a.all + 7) & ~(int64_t)7) + a.first + col);
        const f32x4 z[2] = {from[0], from[1]};
        const uint32_t in[2] = {allowed4(a.mask, col, a.classes), allowed4(a.mask, col + 4, a.classes)};
        const int64_t token = s.at >= 0 ? s.at - a.first - col : -1;
        const Exp<F32> power(a.it);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; k++) {
            float d;
            const float e = power.of(z[k >> 2][k & 3], s.most, d);
            const float slope = fmaf(e, fmaf(s.second, d, s.first), token == k ? s.token : 0.f);
            v[k] = in[k >> 2] >> (8 * (k & 3)) & 0xffu ? slope : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 4; k++) {
            if (F32) {
                uint16_t lo[3], hi[3];
                product::split(v[2 * k], lo);
                product::split(v[2 * k + 1], hi);
#pragma unroll
                for (int h = 0; h < P; h++) w[h][k] = lo[h] | (uint32_t)hi[h] << 16;
            } else {
                w[0][k] = tile::pack_bf16(v[2 * k], v[2 * k + 1]);
            }
        }
    }
#pragma unroll
    for (int h = 0; h < P; h++) *reinterpret_cast<u32x4*>(a.to + t * a.ld + product::column<P>(col, h)) = w[h];
}

// Gradients of a piece's logits.  Every piece more adds to dx in memory once more; a longer one leaves the last-level cache (256 MB) before it is read.  Measured with pieces of
// 64, 128, 300, 600 MB, us: 4096 x 1024 x 32768 (268 MB in all) 1138, 1029, 1014, 1014; 8192 x 512 x 16000 (262) 729, 678, 624, 624;
// 8192 x 1024 x 32768 (537) -, 2114, 1982, 2021; 4096 x 2048 x 65536 (537) -, 3610, 3672, 3704.
constexpr uint64_t kPieceBytes = 288u << 20;
// Logits that forward leaves for backward, a tile as its workgroup holds it: those of the first pieces, up to a GiB, where to compute them again takes about an eighth longer and more.  To write and
// read them is memory's work, to compute them again the matrix units', which is more with many features, and in fp32.  Both ways with the logits and with their computing again, us:
// 4096 x 4096 x 32768 2885 and 3640; 4096 x 2048 x 65536 3249 and 3711; 1000 x 2048 x 10000 197 and 225; fp32 4000 x 1000 x 30000 4350 and 5295; 2000 x 512 x 20000 862 and 1015.  Less is not worth their
// memory: 4096 x 1536 x 32768 1432 and 1559; 4096 x 1024 x 32768 997 and 1025, with 961 MB of workspace and 424; fp32 8000 x 300 x 16000 2050 and 2274; 4000 x 256 x 16000 860 and 919.
// In the L2s: 256 x 512 x 1000 26 and 28; 250 x 256 x 2000 28 and 29; fp32 256 x 512 x 1000 42 and 48; 1000 x 100 x 2000 48 and 50.
constexpr uint64_t kKeptBytes = 1u << 30, kNearBytes = 16u << 20;
int64_t kept_from(bool f32, uint64_t bytes) { return bytes <= kNearBytes ? (f32 ? 1 : 256) : f32 ? 512 : 2048; }
uint64_t up256(uint64_t v) { return (v + 255) & ~(uint64_t)255; }

template <class T>
void launch_few(const FewArgs& a, hipStream_t stream) {
    const int blocks = few_blocks(a.rows, a.classes);
    const dim3 grid((unsigned)((a.classes + 16 * blocks - 1) / (16 * blocks)), (unsigned)((a.rows + 63) / 64));
    constexpr bool kStaged = sizeof(T) == 2;
    if (a.rows <= 16 && kStaged && a.features % 8)
        CANVAS_LAUNCH((k_few<T, 1, 2, kStaged>), grid, dim3(few::kThreads), 0, stream, a);
    else if (a.rows <= 16)
        CANVAS_LAUNCH((k_few<T, 1, 2, false>), grid, dim3(few::kThreads), 0, stream, a);
    else if (a.rows <= few::kRows && blocks == 2)
        CANVAS_LAUNCH((k_few<T, 2, 2, kStaged>), grid, dim3(few::kThreads), 0, stream, a);
    else if (a.rows <= few::kRows)
        CANVAS_LAUNCH((k_few<T, 2, 4, kStaged>), grid, dim3(few::kThreads), 0, stream, a);
    else if constexpr (sizeof(T) == 4)
        CANVAS_LAUNCH((k_few<T, 4, 2, kStaged>), grid, dim3(few::kThreads), 0, stream, a);
}
template <class F>
void launch_logits(const FwdArgs& a, hipStream_t stream) {
    CANVAS_LAUNCH(k_logits<F>, rows_of_workgroups(a.tiles_i * a.tiles_j, F::kThreads), dim3(F::kThreads), 0, stream, a);
}
template <class F>
void launch_grads(const GradArgs& a, hipStream_t stream) {
    const dim3 grid = rows_of_workgroups(a.tiles_i * a.tiles_j, F::kThreads);
    if (a.kept)
        CANVAS_LAUNCH((k_grads<F, true>), grid, dim3(F::kThreads), 0, stream, a);
    else
        CANVAS_LAUNCH((k_grads<F, false>), grid, dim3(F::kThreads), 0, stream, a);
}

Factor factor_of(const uint16_t* at, int64_t rows, int64_t ld) { return Factor{{at, at}, ld, rows}; }

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    const int64_t ld = product::pitch(s.f32, s.features), planes = s.f32 ? 3 : 1;
    double tiles;
    p.logits = product::cut_of(s.f32, s.classes, s.rows, s.features, 1, false, &tiles);
    p.few = few::fits(s.f32, s.rows, s.classes, s.features, tiles);
    p.copies = (s.f32 || s.features % 8) && !(p.few && s.inference);
    const int segment = 16 * few_blocks(s.rows, s.classes);
    p.segments = (int)(p.few ? (s.classes + segment - 1) / segment : p.logits.tiles_i * 2);
    p.launches_fwd = 2 + (p.copies && !p.few);
    p.most_tiles = p.few ? p.segments : p.logits.tiles();
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t r = at;
        at += up256(bytes);
        return r;
    };
    p.sums_at = take(sizeof(Sums) * (uint64_t)s.rows * p.segments);
    p.token_at = take(4ull * s.rows);
    if (p.copies || !s.inference) p.copy_at[0] = take(2ull * s.rows * ld);
    if (p.copies) p.copy_at[1] = take(2ull * s.classes * ld);
    if (!s.inference) {
        p.rows_at = take(sizeof(Row) * (uint64_t)s.rows);
        p.slope_at = take(sizeof(Slope) * (uint64_t)s.rows);
        const int64_t fit = std::max<int64_t>(1, (int64_t)(kPieceBytes / (2ull * planes * s.rows)) / 256) * 256;
        p.pieces = (int)((s.classes + fit - 1) / fit);
        p.length = std::min<int64_t>(((s.classes + p.pieces - 1) / p.pieces + 255) / 256 * 256, s.classes);
        p.pieces = (int)((s.classes + p.length - 1) / p.length);
        p.piece = p.logits;
        p.piece.tiles_i = (p.length + p.piece.high - 1) / p.piece.high;
        if (p.few) {
            p.logits_at = take(4ull * s.rows * ((s.classes + 7) / 8 * 8));
        } else {
            const uint64_t each = 4ull * p.piece.tiles() * p.piece.high * p.piece.side;
            if (s.features >= kept_from(s.f32, each * p.pieces)) p.kept = (int)std::min<uint64_t>(p.pieces, kKeptBytes / each);
            p.logits_at = take(each * p.kept);
        }
        product::cuts_of(s.f32, {s.rows, s.features, p.length, 1}, {p.length, s.features, s.rows, 1}, p.dx, p.dw);
        if (!p.copies) p.copy_at[1] = take(2ull * p.length * ld);
        p.launches_bwd = 1 + (p.copies && p.few) + p.pieces + (p.pieces - 1) * product::launches_of(product::Cut{p.dx.side}, p.dw, false) + product::launches_of(p.dx, p.dw, p.pieces > 1);
        p.launches_mask = p.copies ? 0 : p.pieces;
        p.again = p.few ? 0 : s.classes - std::min(s.classes, p.kept * p.length);
        p.most_tiles = std::max({p.most_tiles, p.piece.tiles(), p.dx.tiles() * p.dx.splits + p.dw.tiles() * p.dw.splits});
        p.grad_at = take(2ull * s.rows * product::pitch(s.f32, p.length));
        p.parts_dx_at = take(product::parts_bytes(p.dx, 1, p.pieces > 1));
        p.parts_dw_at = take(product::parts_bytes(p.dw, 1, false));
    }
    p.workspace_bytes = at;
    return p;
}

void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    Sums* sums = reinterpret_cast<Sums*>(a.ws + p.sums_at);
    float* token = a.logprob ? reinterpret_cast<float*>(a.ws + p.token_at) : nullptr;
    if (p.few) {
        const FewArgs f{a.x, a.weight, s.rows, s.features, s.classes, a.it, a.mask, a.tokens, sums, token, s.inference ? nullptr : reinterpret_cast<float*>(a.ws + p.logits_at)};
        if (s.f32)
            launch_few<float>(f, stream);
        else
            launch_few<uint16_t>(f, stream);
    } else {
        const uint16_t *x = static_cast<const uint16_t*>(a.x), *w = static_cast<const uint16_t*>(a.weight);
        if (p.copies) {
            uint16_t *cx = reinterpret_cast<uint16_t*>(a.ws + p.copy_at[0]), *cw = reinterpret_cast<uint16_t*>(a.ws + p.copy_at[1]);
            const product::Copy c[2] = {{x, cx, s.rows, s.features, nullptr}, {w, cw, s.classes, s.features, a.mask}};
            product::copy(s.f32, c, 2, stream);
            x = cx;
            w = cw;
        }
        const int64_t ld = product::pitch(s.f32, s.features);
        const FwdArgs f{factor_of(w, s.classes, ld), factor_of(x, s.rows, ld), s.rows, s.features, s.classes, p.logits.tiles_i, p.logits.tiles_j, a.it, a.mask, a.tokens, sums, token, reinterpret_cast<f32x4*>(a.ws + p.logits_at), p.kept * p.length};
        product::with_form(s.f32, p.logits.side, [&](auto form) { launch_logits<decltype(form)>(f, stream); });
    }
    // as many threads to a row as give each a few segments (16 rows of 1563: 8 us with 256 threads each, 20 with 16)
    int turns = 16;
    while (turns < 256 && turns * 6 < p.segments) turns *= 2;
    const int across = 256 / turns;
    const RowArgs r{s.rows, s.classes, p.segments, across, a.it, a.mask, a.tokens, sums, token, a.logprob, a.entropy, s.inference ? nullptr : reinterpret_cast<Row*>(a.ws + p.rows_at)};
    CANVAS_LAUNCH(k_rows, rows_of_workgroups((s.rows + across - 1) / across, 256), dim3(256), 0, stream, r);
}

void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    Slope* slope = reinterpret_cast<Slope*>(a.ws + p.slope_at);
    uint16_t* grads = reinterpret_cast<uint16_t*>(a.ws + p.grad_at);
    // W, where it is not a copy that forward has left, has zeros for masked classes too, whole or piece by piece
    uint16_t *cx = reinterpret_cast<uint16_t*>(a.ws + p.copy_at[0]), *cw = reinterpret_cast<uint16_t*>(a.ws + p.copy_at[1]);
    const SlopeArgs l{s.rows, s.classes, s.features, a.it, a.tokens, a.dlogprob, a.dentropy, reinterpret_cast<const Row*>(a.ws + p.rows_at), slope, a.x, cx};
    const dim3 grid((unsigned)std::min<int64_t>((s.rows * product::padded(s.f32, s.features) / 8 + 255) / 256, 4096));
    if (s.f32)
        CANVAS_LAUNCH(k_slopes<true>, grid, dim3(256), 0, stream, l);
    else
        CANVAS_LAUNCH(k_slopes<false>, grid, dim3(256), 0, stream, l);
    if (p.copies && p.few) {
        const product::Copy c{a.weight, cw, s.classes, s.features, a.mask};
        product::copy(s.f32, &c, 1, stream);
    }
    const int64_t lx = product::pitch(s.f32, s.features);
    const Factor x = factor_of(cx, s.rows, lx), all = factor_of(p.copies ? cw : static_cast<const uint16_t*>(a.weight), s.classes, lx);
    const int64_t ld = product::pitch(s.f32, p.length), wide = product::padded(s.f32, p.length);
    for (int n = 0; n < p.pieces; n++) {
        const int64_t first = n * p.length, length = std::min(p.length, s.classes - first);
        Factor w = all;
        w.p[0] = w.p[1] = all.p[0] + first * lx;
        w.count = length;
        const uint8_t* mask = a.mask ? a.mask + first : nullptr;
        if (p.few) {
            const FewGradArgs g{reinterpret_cast<const float*>(a.ws + p.logits_at), s.rows, length, s.classes, first, a.it, mask, slope, grads, ld, wide};
            const dim3 grid((unsigned)((wide / 8 + 255) / 256), (unsigned)s.rows);
            if (s.f32)
                CANVAS_LAUNCH(k_few_grads<true>, grid, dim3(256), 0, stream, g);
            else
                CANVAS_LAUNCH(k_few_grads<false>, grid, dim3(256), 0, stream, g);
        } else {
            const GradArgs g{w, x, s.rows, s.features, length, (length + p.piece.high - 1) / p.piece.high, p.piece.tiles_j, first, a.it, mask, slope, grads, ld, wide,
                             n < p.kept ? reinterpret_cast<f32x4*>(a.ws + p.logits_at) + first * p.piece.tiles_j * p.piece.side / 4 : nullptr};
            product::with_form(s.f32, p.piece.side, [&](auto form) { launch_grads<decltype(form)>(g, stream); });
        }
        if (mask && !p.copies) {
            const product::Copy m{w.p[0], cw, length, s.features, mask};
            product::copy(false, &m, 1, stream);
            w.p[0] = w.p[1] = cw;
        }
        product::Product d;
        d.f32 = s.f32;
        d.a = Factor{{grads, grads}, ld, s.rows};
        d.a_rows = true;
        d.b = w;
        d.b.count = s.features;
        d.depth = length;
        d.out[0] = a.dx;
        d.ld = s.features;
        d.cut = p.dx;
        d.parts = p.dx.splits > 1 || p.pieces > 1 ? reinterpret_cast<float*>(a.ws + p.parts_dx_at) : nullptr;
        d.first = n == 0;
        d.last = n + 1 == p.pieces;
        product::Product e = d;
        e.a.count = length;
        e.a_rows = false;
        e.b = x;
        e.b.count = s.features;
        e.depth = s.rows;
        e.out[0] = static_cast<char*>(a.dweight) + first * s.features * (s.f32 ? 4 : 2);
        e.cut = p.dw;
        e.cut.tiles_i = (length + p.dw.high - 1) / p.dw.high;
        e.parts = p.dw.splits > 1 ? reinterpret_cast<float*>(a.ws + p.parts_dw_at) : nullptr;
        e.first = e.last = true;
        product::multiply(d, e, stream);
    }
}

}  // namespace head
}  // namespace canvas
