// The gated pair of FCs: y = act(x Wg^T) (x Wu^T).
//
// Forward: one product whose columns are those of both weights, 32 of the gate and 32 of the other in turn, so that a wave holds g and u of
// the same results in the same places of its registers and y is theirs.  Training keeps g and u (Kept).
// Backward: dg and du element by element from g, u and dy; then dx as one sum over the columns of both, and dWg and dWu as one launch.
#include "gated_kernels.hpp"

#include <algorithm>
#include <type_traits>

#include "../../include/canvas_gated.h"
#include "device_util.hpp"
#include "exp_util.hpp"
#include "few_device.hpp"
#include "launch.hpp"
#include "product_device.hpp"
#include "row_util.hpp"
#include "tile_util.hpp"

namespace canvas {
namespace gated {
namespace {

using product::f32x16;
using product::f32x4;
using product::Factor;
using product::Form;
using tile::u32x4;

// act(g); with SLOPE its derivative too.  e^-|g| serves both signs; NaN stays (comparisons, not maxima).
template <int ACT, bool SLOPE>
__device__ __forceinline__ float act_of(float g, float& slope) {
    if (ACT == CANVAS_GATED_GELU) {
        const float cdf = 0.5f * erfcf(g * -0.70710678118654752f);
        if (SLOPE) {
            const float half = -0.5f * g * g;
            slope = fmaf(g * 0.39894228040143268f, exp_finite(half < -300.f ? -300.f : half), cdf);
        }
        return g * cdf;
    }
    const float m = -fabsf(g), e = exp_finite(m < -300.f ? -300.f : m), r = __builtin_amdgcn_rcpf(1.f + e);
    const float sig = g < 0.f ? e * r : r, other = g < 0.f ? r : e * r;  // other = 1 - sig without a difference
    if (ACT == CANVAS_GATED_SIGMOID) {
        if (SLOPE) slope = sig * other;
        return sig;
    }
    if (SLOPE) slope = sig * fmaf(g, other, 1.f);
    return g * sig;
}

// What backward needs of g and u: both as they are, in fp32.  (20 bits of each in bf16 plans would be 5 bytes an element to write and to read again instead of 8:
// 4096 x 2048 x 8192 forward and backward 801 us instead of 832, with gradients that are no longer those of g and u.)
struct Kept {
    float* at;      // g, then u
    int64_t plane;  // elements
    static constexpr int kBytes = 8;  // of an element

    __device__ __forceinline__ void put1(int64_t i, float g, float u) const {
        at[i] = g;
        at[plane + i] = u;
    }
    // eight elements from i on, a multiple of 8
    __device__ __forceinline__ void put8(int64_t i, const f32x4 (&g)[2], const f32x4 (&u)[2]) const {
        f32x4 *to = reinterpret_cast<f32x4*>(at) + i / 4, *to_u = to + plane / 4;
        to[0] = g[0];
        to[1] = g[1];
        to_u[0] = u[0];
        to_u[1] = u[1];
    }
    __device__ __forceinline__ void get8(int64_t i, float (&g)[8], float (&u)[8]) const {
        const f32x4 *from = reinterpret_cast<const f32x4*>(at) + i / 4, *from_u = from + plane / 4;
        const f32x4 v[4] = {from[0], from[1], from_u[0], from_u[1]};
#pragma unroll
        for (int k = 0; k < 8; k++) g[k] = v[k >> 2][k & 3], u[k] = v[2 + (k >> 2)][k & 3];
    }
};

struct FwdArgs {
    Factor x, w;
    int64_t rows, features, width, tiles_i, tiles_j, ld;
    void* y;
    float* kept;
    int64_t plane;
};

// Tiles whose columns are those of both matrices.
using SmallPair = Form<64, 128, 2, 2, 1, 64, 3>;
using SmallTriplePair = Form<64, 128, 2, 2, 3, 32, 2>;
template <class F>
struct Paired {
    using Type = F;
};
template <>
struct Paired<product::Small> {
    using Type = SmallPair;
};
template <>
struct Paired<product::SmallTriple> {
    using Type = SmallTriplePair;
};

// Bound by the matrix units, and at a tile's end by memory (10 bytes of results in bf16 training), which nothing hides where the tile fills its compute unit: 4096 x 2048 x 2 * 8192
// bf16 301 us with g and u kept (0.91 PFLOP/s), fp32 4096 x 1024 x 2 * 4096 353 us with the operands' copies (195 TFLOP/s of fp32 results).  Tiles of 128 x 128, two workgroups to a
// compute unit, hide it and read more: 918 us forward and backward instead of 879 at the time.
template <class F, int ACT>
__global__ __launch_bounds__(F::kThreads, 2) void k_forward(FwdArgs a) {
    constexpr int TM = F::TM, TN = F::TN, kCols = F::BN / 2;
    constexpr bool kF32 = F::PLANES == 3;
    static_assert(TN == 2, "a wave holds one block of each matrix");
    PRODUCT_BUFFERS(F, buffers);
    const product::Place at = product::place_of(tile::xcd_sequence(), a.tiles_i, a.tiles_j, 1, 1);
    if (!at.inside) return;
    const int64_t i0 = at.i * F::BM, j0 = at.j * kCols;
    const int steps = (int)((a.features + F::BK - 1) / F::BK);
    f32x16 acc[TM][TN] = {};
    product::accumulate<F, product::kRows, product::kRows, true>(a.x, a.w, 0, i0, j0, a.features, 0, steps, steps, 1, buffers, acc);
    // g and u through LDS, kRows rows of the tile at a time: a few lines of code for all elements (64 copies of the activation, one for each
    // register, take longer to fetch than to run where there is little else to do), and whole vectors to memory.  Elements change places by bits of the row, so that what
    // the halves of a wave write at once falls on different banks.
    constexpr int kFit = F::kStage / (kCols * 4), kTwos = kFit >= 128 ? 128 : kFit >= 64 ? 64 : 32, kRows = kTwos < F::BM ? kTwos : F::BM;
    static_assert(kRows <= kFit && F::BM % kRows == 0, "rows of the tile in a buffer");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / F::WJ * (TM * 32), wj = wave % F::WJ * 32;
    float *img_g = reinterpret_cast<float*>(buffers.at[0]), *img_u = reinterpret_cast<float*>(buffers.at[1]);
    const bool whole = (a.width & 7) == 0;
#pragma unroll 1
    for (int r0 = 0; r0 < F::BM; r0 += kRows) {
        if (r0) tile::lds_barrier();
#pragma unroll
        for (int x = 0; x < TM; x++) {
            if (wi + x * 32 < r0 || wi + x * 32 >= r0 + kRows) continue;
#pragma unroll
            for (int k = 0; k < 16; k++) {
                const int r = wi + x * 32 - r0 + (k >> 2) * 8 + (lane >> 5) * 4 + (k & 3), c = (wj + (lane & 31)) ^ ((r >> 2 & 1) << 5);
                img_g[r * kCols + c] = acc[x][0][k];
                img_u[r * kCols + c] = acc[x][1][k];
            }
        }
        tile::lds_barrier();
#pragma unroll 1
        for (int e = threadIdx.x; e < kRows * (kCols / 8); e += F::kThreads) {
            const int r = e / (kCols / 8), c = (e - r * (kCols / 8)) * 8, from = r * kCols + (c ^ ((r >> 2 & 1) << 5));
            const int64_t i = i0 + r0 + r, j = j0 + c;
            if (i >= a.rows || j >= a.width) continue;
            const f32x4 g[2] = {*reinterpret_cast<const f32x4*>(img_g + from), *reinterpret_cast<const f32x4*>(img_g + from + 4)};
            const f32x4 u[2] = {*reinterpret_cast<const f32x4*>(img_u + from), *reinterpret_cast<const f32x4*>(img_u + from + 4)};
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; k++) {
                float unused;
                y[k] = act_of<ACT, false>(g[k >> 2][k & 3], unused) * u[k >> 2][k & 3];
            }
            if (a.kept) Kept{a.kept, a.plane}.put8(i * a.ld + j, g, u);  // (rows of a multiple of 8)
            if (kF32) {
                float* to = static_cast<float*>(a.y) + i * a.width + j;
                if (whole) {
                    reinterpret_cast<f32x4*>(to)[0] = f32x4{y[0], y[1], y[2], y[3]};
                    reinterpret_cast<f32x4*>(to)[1] = f32x4{y[4], y[5], y[6], y[7]};
                } else {
#pragma unroll
                    for (int k = 0; k < 8; k++)
                        if (j + k < a.width) to[k] = y[k];
                }
            } else {
                uint16_t* to = static_cast<uint16_t*>(a.y) + i * a.width + j;
                if (whole) {
                    *reinterpret_cast<u32x4*>(to) = u32x4{tile::pack_bf16(y[0], y[1]), tile::pack_bf16(y[2], y[3]), tile::pack_bf16(y[4], y[5]), tile::pack_bf16(y[6], y[7])};
                } else {
#pragma unroll
                    for (int k = 0; k < 8; k++)
                        if (j + k < a.width) to[k] = f32_to_bf16(y[k]);
                }
            }
        }
    }
}

struct FewArgs {
    const void *x, *w_gate, *w_up;
    int64_t rows, features, width, ld;
    void* y;
    float* kept;
    int64_t plane;
};
// 16 results of y for all rows of x by a workgroup; bound by the weights' bytes: 4 x 2048 x 2 * 8192 bf16, 67 MB in 12.2 us, 5.5 TB/s; fp32 134 MB in 26.3, 5.1.
template <class T, int NT, int ACT>
__global__ __launch_bounds__(few::kThreads) void k_few(FewArgs a) {
    constexpr bool kStaged = sizeof(T) == 2;
    __shared__ f32x4 shared[few::kShared<kStaged, 2, NT>];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t f0 = (int64_t)blockIdx.x * 16, mine = few::Lanes<kStaged>::row(), row = f0 + mine < a.width ? f0 + mine : a.width - 1;
    const T* const w[2] = {static_cast<const T*>(a.w_gate) + row * a.features, static_cast<const T*>(a.w_up) + row * a.features};
    const T* x[NT];
#pragma unroll
    for (int n = 0; n < NT; n++) {
        const int64_t t = blockIdx.y * (16 * NT) + n * 16 + mine;
        x[n] = static_cast<const T*>(a.x) + (t < a.rows ? t : a.rows - 1) * a.features;
    }
    f32x4 sums[2];
    few::accumulate<kStaged, T, 2, NT, few::ahead(2, NT)>(w, x, a.features, sums, shared);
    const int64_t t = blockIdx.y * (16 * NT) + wave * 16 + (lane & 15), f = f0 + (lane >> 4) * 4;
    if (wave >= NT || t >= a.rows) return;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        if (f + e >= a.width) break;
        float unused;
        const float y = act_of<ACT, false>(sums[0][e], unused) * sums[1][e];
        const int64_t to = t * a.width + f + e;
        if (sizeof(T) == 4)
            static_cast<float*>(a.y)[to] = y;
        else
            static_cast<uint16_t*>(a.y)[to] = f32_to_bf16(y);
        if (a.kept) Kept{a.kept, a.plane}.put1(t * a.ld + f + e, sums[0][e], sums[1][e]);
    }
}

struct GradArgs {
    float* kept;
    int64_t plane, rows, width, ld;
    const void* dy;
    uint16_t *dg, *du;
    int64_t pitch;
};
// dg = dy u act'(g) and du = dy act(g), eight elements per thread and turn; zeros behind the columns.  Rounded to bf16 once in bf16 plans, as the products' operands.
// Bound by memory: 4096 x 8192 bf16, 470 MB in 100 us, 4.7 TB/s.
template <bool F32, int ACT>
__global__ __launch_bounds__(256) void k_grads(GradArgs a) {
    constexpr int P = F32 ? 3 : 1;
    const int64_t wide = a.ld / 8, n = a.rows * wide;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < n; k += (int64_t)gridDim.x * 256) {
        const int64_t row = k / wide, col = (k - row * wide) * 8;
        float g[8], u[8];
        Kept{a.kept, a.plane}.get8(k * 8, g, u);
        using T = std::conditional_t<F32, float, uint16_t>;
        T given[8];
        rows::load8(static_cast<const T*>(a.dy) + row * a.width, col, a.width, given);
        float dy[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            if constexpr (F32)
                dy[e] = given[e];
            else
                dy[e] = bf16_to_f32(given[e]);
        }
        float dg[8], du[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            float slope;
            const float act = act_of<ACT, true>(g[e], slope);
            const bool in = col + e < a.width;  // (behind the columns nothing was written)
            du[e] = in ? dy[e] * act : 0.f;
            dg[e] = in ? dy[e] * u[e] * slope : 0.f;
        }
#pragma unroll
        for (int which = 0; which < 2; which++) {
            const float* v = which ? du : dg;
            uint16_t* to = (which ? a.du : a.dg) + row * a.pitch;
            u32x4 w[P];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (F32) {
                    uint16_t lo[3], hi[3];
                    product::split(v[2 * e], lo);
                    product::split(v[2 * e + 1], hi);
#pragma unroll
                    for (int h = 0; h < P; h++) w[h][e] = lo[h] | (uint32_t)hi[h] << 16;
                } else {
                    w[0][e] = tile::pack_bf16(v[2 * e], v[2 * e + 1]);
                }
            }
#pragma unroll
            for (int h = 0; h < P; h++) *reinterpret_cast<u32x4*>(to + product::column<P>(col, h)) = w[h];
        }
    }
}

uint64_t up256(uint64_t v) { return (v + 255) & ~(uint64_t)255; }

// f with the activation as a constant
template <class F>
void with_act(int act, F f) {
    if (act == CANVAS_GATED_SIGMOID)
        f(std::integral_constant<int, CANVAS_GATED_SIGMOID>());
    else if (act == CANVAS_GATED_SILU)
        f(std::integral_constant<int, CANVAS_GATED_SILU>());
    else
        f(std::integral_constant<int, CANVAS_GATED_GELU>());
}
template <class T>
void launch_few(int act, const FewArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.width + 15) / 16), (unsigned)((a.rows + 63) / 64));
    with_act(act, [&](auto kind) {
        if (a.rows <= 16)
            CANVAS_LAUNCH((k_few<T, 1, decltype(kind)::value>), grid, dim3(few::kThreads), 0, stream, a);
        else if (a.rows <= few::kRows)
            CANVAS_LAUNCH((k_few<T, 2, decltype(kind)::value>), grid, dim3(few::kThreads), 0, stream, a);
        else if constexpr (sizeof(T) == 4)
            CANVAS_LAUNCH((k_few<T, 4, decltype(kind)::value>), grid, dim3(few::kThreads), 0, stream, a);
    });
}
template <class F>
void launch_forward(int act, const FwdArgs& a, hipStream_t stream) {
    with_act(act, [&](auto kind) {
        CANVAS_LAUNCH((k_forward<F, decltype(kind)::value>), rows_of_workgroups(a.tiles_i * a.tiles_j, F::kThreads), dim3(F::kThreads), 0, stream, a);
    });
}

// The three tensors that products read, as they read them.
struct Operands {
    Factor x, w;
};
Operands operands_of(const Shape& s, const Plan& p, const void* x, const void* w_gate, const void* w_up, char* ws) {
    Operands o;
    const void* given[3] = {x, w_gate, w_up};
    const uint16_t* at[3];
    for (int i = 0; i < 3; i++) at[i] = p.copies ? reinterpret_cast<const uint16_t*>(ws + p.copy_at[i]) : static_cast<const uint16_t*>(given[i]);
    const int64_t ld = product::pitch(s.f32, s.features);
    o.x = Factor{{at[0], at[0]}, ld, s.rows};
    o.w = Factor{{at[1], at[2]}, ld, s.width};
    return o;
}
void make_copies(const Shape& s, const Plan& p, const void* x, const void* w_gate, const void* w_up, char* ws, hipStream_t stream) {
    auto to = [&](int i) { return reinterpret_cast<uint16_t*>(ws + p.copy_at[i]); };
    const product::Copy c[3] = {{x, to(0), s.rows, s.features}, {w_gate, to(1), s.width, s.features}, {w_up, to(2), s.width, s.features}};
    product::copy(s.f32, c, 3, stream);
}

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    const int64_t ld = product::pitch(s.f32, s.features), wide = product::padded(s.f32, s.width);
    double tiles;
    p.forward = product::cut_of(s.f32, s.rows, 2 * s.width, s.features, 1, false, &tiles);
    p.few = few::fits(s.f32, s.rows, 2 * s.width, s.features, tiles);
    p.copies = (s.f32 || s.features % 8) && !(p.few && s.inference);
    const int64_t pairs = p.forward.side == 64 ? 64 : p.forward.side / 2;  // results of a tile's row (Paired)
    p.forward.tiles_j = (s.width + pairs - 1) / pairs;
    p.launches_fwd = 1 + (p.copies && !p.few);
    p.most_tiles = p.few ? (s.width + 15) / 16 : p.forward.tiles();
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t r = at;
        at += up256(bytes);
        return r;
    };
    if (p.copies) {
        const int64_t rows[3] = {s.rows, s.width, s.width};
        for (int i = 0; i < 3; i++) p.copy_at[i] = take(2ull * rows[i] * ld);
    }
    if (!s.inference) {
        product::cuts_of(s.f32, {s.rows, s.features, 2 * s.width, 1}, {s.width, s.features, s.rows, 2}, p.dx, p.dw);
        p.launches_bwd = (p.copies && p.few) + 1 + product::launches_of(p.dx, p.dw, false);
        p.most_tiles = std::max(p.most_tiles, p.dx.tiles() * p.dx.splits + 2 * p.dw.tiles() * p.dw.splits);
        p.kept_at = take((uint64_t)Kept::kBytes * s.rows * wide);
        p.grad_at = take(4ull * s.rows * product::pitch(s.f32, s.width));
        p.parts_at = take(product::parts_bytes(p.dx, 1, false));
        p.parts_dw_at = take(product::parts_bytes(p.dw, 2, false));
    }
    p.workspace_bytes = at;
    return p;
}

void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    const int64_t ld = product::padded(s.f32, s.width);
    float* kept = s.inference ? nullptr : reinterpret_cast<float*>(a.ws + p.kept_at);
    if (p.few) {
        const FewArgs f{a.x, a.w_gate, a.w_up, s.rows, s.features, s.width, ld, a.y, kept, s.rows * ld};
        return s.f32 ? launch_few<float>(s.act, f, stream) : launch_few<uint16_t>(s.act, f, stream);
    }
    if (p.copies) make_copies(s, p, a.x, a.w_gate, a.w_up, a.ws, stream);
    const Operands o = operands_of(s, p, a.x, a.w_gate, a.w_up, a.ws);
    const FwdArgs f{o.x, o.w, s.rows, s.features, s.width, p.forward.tiles_i, p.forward.tiles_j, ld, a.y, kept, s.rows * ld};
    product::with_form(s.f32, p.forward.side, [&](auto form) { launch_forward<typename Paired<decltype(form)>::Type>(s.act, f, stream); });
}

void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    const int64_t ld = product::padded(s.f32, s.width), plane = s.rows * ld, wide = product::pitch(s.f32, s.width);
    if (p.copies && p.few) make_copies(s, p, a.x, a.w_gate, a.w_up, a.ws, stream);
    uint16_t *dg = reinterpret_cast<uint16_t*>(a.ws + p.grad_at), *du = dg + s.rows * wide;
    const GradArgs g{reinterpret_cast<float*>(a.ws + p.kept_at), plane, s.rows, s.width, ld, a.dy, dg, du, wide};
    const dim3 grid((unsigned)std::min<int64_t>((plane / 8 + 255) / 256, 8192));
    with_act(s.act, [&](auto kind) {
        if (s.f32)
            CANVAS_LAUNCH((k_grads<true, decltype(kind)::value>), grid, dim3(256), 0, stream, g);
        else
            CANVAS_LAUNCH((k_grads<false, decltype(kind)::value>), grid, dim3(256), 0, stream, g);
    });
    const Operands o = operands_of(s, p, a.x, a.w_gate, a.w_up, a.ws);
    product::Product d;
    d.f32 = s.f32;
    d.a = Factor{{dg, du}, wide, s.rows};
    d.a_rows = true;
    d.b = o.w;
    d.b.count = s.features;
    d.depth = s.width;
    d.segments = 2;
    d.out[0] = a.dx;
    d.ld = s.features;
    d.cut = p.dx;
    d.parts = p.dx.splits > 1 ? reinterpret_cast<float*>(a.ws + p.parts_at) : nullptr;
    product::Product w = d;
    w.a.count = s.width;
    w.a_rows = false;
    w.b = o.x;
    w.b.count = s.features;
    w.depth = s.rows;
    w.segments = 1;
    w.results = 2;
    w.out[0] = a.dw_gate;
    w.out[1] = a.dw_up;
    w.cut = p.dw;
    w.parts = p.dw.splits > 1 ? reinterpret_cast<float*>(a.ws + p.parts_dw_at) : nullptr;
    product::multiply(d, w, stream);
}

}  // namespace gated
}  // namespace canvas
