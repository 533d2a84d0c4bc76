// Residual norm, forward, and what forward and backward share on the host.  Both are bound by memory: five maps move forward, eight
// backward, and everything in between stays in registers.  Forward, over three sets of maps in turn: 64 x 64 x 56 x 56 in 30 us bf16 (4.3 TB/s) and 46 us fp32
// (5.6 TB/s), 128 x 256 x 14 x 14 in 17 us (3.7 TB/s), 128 x 512 x 7 x 7 in 14 us (2.3 TB/s, one round of workgroups), rows 4096 x 2048 in
// fp32 33 us (5.0 TB/s), without a gate 24 (5.7 TB/s), 8 x 1024 in bf16 4 us (the launch).
//
// Maps (planes of two pixels or more): a thread takes 16 bytes of pixels of `KC` channels, lanes side by side GX such pieces, the
// other lanes and waves the channels in turn; sums over the channels go through lane exchanges and LDS.  The last piece of a
// plane ends with it and may overlap the one before it: the pixels in common are computed twice, alike, and counted once in
// the sums of the weights' gradients.  Where a plane is shorter than 16 bytes a thread takes two pixels.
// Channels that no workgroup can hold (KC = 0) are read again for each of the passes, from the caches for the most part.
//
// Rows (planes of one pixel): TPR threads per row, KV times 16 bytes each.
//
// Workgroups of the backward kernels walk over tiles and keep the weights' gradients of their channels in registers (KC = 0: in
// LDS); one partial sum per workgroup is left, which a second launch adds in a fixed order.
#include "norm_kernels.hpp"

#include <algorithm>

#include "launch.hpp"
#include "norm_device.hpp"

namespace canvas {
namespace norm {
namespace {

template <class T>
__device__ __forceinline__ float act_of(bool silu, float g) {
    const float s = sigmoid<T>(g);
    return silu ? g * s : s;
}

// ---------------------------------------------------------------- maps

template <class T, int VEC, int KC, int PARTS>
__global__ __launch_bounds__(512) void k_maps_fwd(Shape s, Fwd a, int log_gx, int pieces, int64_t total) {
    extern __shared__ float lds[];
    const int GX = 1 << log_gx, gx = threadIdx.x & (GX - 1), cy = threadIdx.x >> log_gx, CY = blockDim.x >> log_gx;
    const Where at = where_of<VEC>(s, pieces, total, (int64_t)tile::xcd_sequence() * GX + gx);
    const float inv = 1.f / s.C / (s.down * s.down);
    const bool gated = (PARTS & kPost) && s.gate, silu = s.gate == 2;
    constexpr int K = KC ? KC : 1;
    Vec<T, VEC> x[K], z[K], g[K];
    auto load_z = [&](int k, int c) { z[k].load(a.z, at.base + c * s.P); };
    auto load_x = [&](int k, int c) {
        x[k].load(a.x, at.base + c * s.P);
        if (gated) g[k].load(a.g, at.base + c * s.P);
    };
    auto each = [&](auto f) { each_channel<KC>(cy, CY, s.C, f); };
    if (KC) each([&](int k, int c) {
            if (PARTS & kPost) load_z(k, c);
            load_x(k, c);
        });
    float r2[VEC], t[VEC];
    if (PARTS & kPost) {
#pragma unroll
        for (int e = 0; e < VEC; e++) r2[e] = 0.f;
        each([&](int k, int c) {
            if (!KC) load_z(k, c);
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                const float v = z[k].at(e) * s.down;
                r2[e] += v * v;
            }
        });
        over_channels<VEC>(r2, gx, GX, lds);
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            r2[e] = rsqrtf(r2[e] * inv + s.eps);
            if (a.r2 && cy == 0 && at.in) a.r2[at.pixel + e] = r2[e];
        }
    }
    auto joined = [&](int k, int e, float sw) {
        float y = x[k].at(e);
        if (PARTS & kPost) y += sw * (gated ? act_of<T>(silu, g[k].at(e)) : 1.f) * (z[k].at(e) * r2[e]);
        return y;
    };
#pragma unroll
    for (int e = 0; e < VEC; e++) t[e] = 0.f;
    float y[K][VEC];
    each([&](int k, int c) {
        if (!KC) {
            if (PARTS & kPost) load_z(k, c);
            load_x(k, c);
        }
        const float sw = PARTS & kPost ? a.scale[c] * a.w_post[c] : 0.f;
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            y[k][e] = joined(k, e, sw);
            const float v = y[k][e] * s.down;
            t[e] += v * v;
        }
        if ((PARTS & kPost) && at.in) store<T, VEC>(a.x_out, at.base + c * s.P, y[k]);
    });
    if (!(PARTS & kPre)) return;
    over_channels<VEC>(t, gx, GX, lds);
#pragma unroll
    for (int e = 0; e < VEC; e++) {
        t[e] = rsqrtf(t[e] * inv + s.eps);
        if (a.r1 && cy == 0 && at.in) a.r1[at.pixel + e] = t[e];
    }
    each([&](int k, int c) {
        if (!KC) {
            if (PARTS & kPost) load_z(k, c);
            load_x(k, c);
            const float sw = PARTS & kPost ? a.scale[c] * a.w_post[c] : 0.f;
#pragma unroll
            for (int e = 0; e < VEC; e++) y[k][e] = joined(k, e, sw);
        }
        const float w = a.w_pre[c];
#pragma unroll
        for (int e = 0; e < VEC; e++) y[k][e] *= t[e] * w;
        if (at.in) store<T, VEC>(a.u, at.base + c * s.P, y[k]);
    });
}

// ---------------------------------------------------------------- rows

template <class T, int TPR, int KV, int PARTS>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_rows_fwd(Shape s, Fwd a) {
    constexpr int V = 16 / sizeof(T), kRows = TPR < 256 ? 256 / TPR : 1;
    __shared__ float buf[16];
    const int t = threadIdx.x % TPR;
    const int64_t n = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRows + threadIdx.x / TPR;
    if (n >= s.N) return;  // (with several rows per workgroup a row is within a wave: no barriers)
    const int64_t row = n * s.C;
    const bool gated = (PARTS & kPost) && s.gate, silu = s.gate == 2;
    const float inv = 1.f / s.C / (s.down * s.down);
    Vec<T, V> x[KV], z[KV], g[KV];
#pragma unroll
    for (int k = 0; k < KV; k++) {
        const int c = (k * TPR + t) * V;
        load_row<T, V>(x[k], a.x, row, c, s.C);
        if (PARTS & kPost) load_row<T, V>(z[k], a.z, row, c, s.C);
        if (gated) load_row<T, V>(g[k], a.g, row, c, s.C);
    }
    float r2 = 0.f;
    if (PARTS & kPost) {
#pragma unroll
        for (int k = 0; k < KV; k++)
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float v = z[k].at(e) * s.down;
                r2 += v * v;
            }
        r2 = rsqrtf(over_row<TPR>(r2, buf) * inv + s.eps);
        if (a.r2 && t == 0) a.r2[n] = r2;
    }
    // x' before its rounding, computed again behind the sum of its squares
    auto joined = [&](int k, float (&y)[V]) {
        const int c = (k * TPR + t) * V;
        float sw[V], w[V];
        x[k].renew();
        if (PARTS & kPost) {
            z[k].renew();
            if (gated) g[k].renew();
            load_weights<V>(w, a.w_post, c, s.C);
            load_weights<V>(sw, a.scale, c, s.C);
        }
#pragma unroll
        for (int e = 0; e < V; e++) {
            y[e] = x[k].at(e);
            if (PARTS & kPost) y[e] += sw[e] * w[e] * (gated ? act_of<T>(silu, g[k].at(e)) : 1.f) * (z[k].at(e) * r2);
        }
    };
    float y[V], r1 = 0.f;
#pragma unroll
    for (int k = 0; k < KV; k++) {
        joined(k, y);
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float v = y[e] * s.down;
            r1 += v * v;
        }
        if (PARTS & kPost) store_row<T, V>(a.x_out, row, (k * TPR + t) * V, s.C, y);
    }
    if (!(PARTS & kPre)) return;
    r1 = rsqrtf(over_row<TPR>(r1, buf) * inv + s.eps);
    if (a.r1 && t == 0) a.r1[n] = r1;
#pragma unroll
    for (int k = 0; k < KV; k++) {
        const int c = (k * TPR + t) * V;
        float w1[V];
        load_weights<V>(w1, a.w_pre, c, s.C);
        if (KV > 1) joined(k, y);
#pragma unroll
        for (int e = 0; e < V; e++) y[e] *= r1 * w1[e];
        store_row<T, V>(a.u, row, c, s.C, y);
    }
}

// ---------------------------------------------------------------- sums of the weights' gradients

constexpr int kSumSlices = 16, kTogether = 16;
__global__ __launch_bounds__(64 * kSumSlices) void k_sums(Shape s, Bwd a, int partials) {
    __shared__ float buf[kSumSlices][64];
    const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6, i = blockIdx.x * 64 + lane, n = 2 * s.C;
    float v = 0.f;
    if (i < n)
        for (int first = slice; first < partials; first += kSumSlices * kTogether) {
            float w[kTogether];  // (all asked for before the first is added)
#pragma unroll
            for (int u = 0; u < kTogether; u++) {
                const int p = first + u * kSumSlices;
                w[u] = p < partials ? a.partial[(int64_t)p * n + i] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < kTogether; u++) v += w[u];
        }
    buf[slice][lane] = v;
    __syncthreads();
    if (slice || i >= n) return;
    v = 0.f;
#pragma unroll
    for (int k = 0; k < kSumSlices; k++) v += buf[k][lane];
    if (i >= s.C) {
        if (s.pre) a.dw_pre[i - s.C] = v;
    } else if (s.post) {
        a.dw_post[i] = a.scale[i] * v;
        a.dscale[i] = a.w_post[i] * v;
    }
}

// ---------------------------------------------------------------- launches

template <class T, int VEC, int KC, int PARTS>
void maps(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    const Tiling& t = p.fwd;
    const int64_t tiles = (p.total + (1 << t.log_gx) - 1) >> t.log_gx;
    // (a last row of workgroups that is not full has pieces behind the last one: they write nothing)
    CANVAS_LAUNCH((k_maps_fwd<T, VEC, KC, PARTS>), rows_of_workgroups(tiles, t.threads), dim3(t.threads), t.threads / 64 * (1 << t.log_gx) * VEC * 4, stream, s, a, t.log_gx,
                  p.pieces, p.total);
}
template <class T, int TPR, int KV, int PARTS>
void rows(const Shape& s, const Fwd& a, hipStream_t stream) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, kRows = kBlock / TPR;
    CANVAS_LAUNCH((k_rows_fwd<T, TPR, KV, PARTS>), rows_of_workgroups((s.N + kRows - 1) / kRows, kBlock), dim3(kBlock), 0, stream, s, a);
}
template <class T, int PARTS>
void run(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    if (p.tpr) {
        switch (p.tpr * 8 + p.kv) {
        case 16 * 8 + 1: return rows<T, 16, 1, PARTS>(s, a, stream);
        case 64 * 8 + 1: return rows<T, 64, 1, PARTS>(s, a, stream);
        case 64 * 8 + 2: return rows<T, 64, 2, PARTS>(s, a, stream);
        case 256 * 8 + 1: return rows<T, 256, 1, PARTS>(s, a, stream);
        case 512 * 8 + 1: return rows<T, 512, 1, PARTS>(s, a, stream);
        case 1024 * 8 + 1: return rows<T, 1024, 1, PARTS>(s, a, stream);
        default: return rows<T, 1024, 16 / V, PARTS>(s, a, stream);
        }
    }
    if (p.vec == 2) return maps<T, 2, 0, PARTS>(s, p, a, stream);
    switch (p.fwd.kc) {
    case 1: return maps<T, V, 1, PARTS>(s, p, a, stream);
    case 2: return maps<T, V, 2, PARTS>(s, p, a, stream);
    case 4: return maps<T, V, 4, PARTS>(s, p, a, stream);
    default: return maps<T, V, 0, PARTS>(s, p, a, stream);
    }
}
template <class T>
void run_parts(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    if (s.post && s.pre)
        run<T, kPost | kPre>(s, p, a, stream);
    else if (s.post)
        run<T, kPost>(s, p, a, stream);
    else
        run<T, kPre>(s, p, a, stream);
}

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    const int v = s.bf16 ? 8 : 4;
    if (s.P == 1) {
        // (one access per thread as long as there are threads: 4096 x 2560 in bf16 20 + 41 us by 512 threads, 28 + 48 by 256)
        const int sizes[][2] = {{16, 1}, {64, 1}, {64, 2}, {256, 1}, {512, 1}, {1024, 1}, {1024, 16 / v}};
        for (const auto& z : sizes) {
            p.tpr = z[0];
            p.kv = z[1];
            if (z[0] * z[1] * v >= s.C) break;
        }
        const int64_t per = p.tpr < 256 ? 256 / p.tpr : 1;
        p.partials = (int)std::min<int64_t>((s.N + per - 1) / per, p.tpr == 1024 ? 256 : 512);
        return p;
    }
    p.vec = s.P >= v ? v : 2;
    p.pieces = (int)((s.P + p.vec - 1) / p.vec);
    p.total = s.N * p.pieces;
    const bool held = p.vec == v && s.C <= 2048;
    // Pieces side by side: as many as make a workgroup's share of a plane's row a cache line, fewer where that leaves compute units
    // idle or a workgroup without room for all channels (32 x 2048 x 7 x 7, one piece and all channels held: forward 17, backward
    // 30 us; two pieces and channels read again: 35 and 75).  One piece alone, where two fill half of the compute units, loses
    // if the channels are held (16 x 256 x 14 x 14 backward 13 us, with two 12) and gains if not (64 x 4096 x 7 x 7: 71 + 157 us,
    // with two 87 + 168).  Down to four pieces, rather fewer of them than more than `rather` channels of a thread.
    auto tiling = [&](int rather) {
        Tiling t;
        t.log_gx = 3;
        while (t.log_gx > 0 && ((p.total >> t.log_gx) < (t.log_gx > 1 || !held ? 256 : 128) || (held && s.C > 4 * (512 >> t.log_gx)))) t.log_gx--;
        while (held && t.log_gx > 2 && s.C > rather * (256 >> t.log_gx)) t.log_gx--;
        t.threads = held && s.C <= 4 * (256 >> t.log_gx) ? 256 : 512;
        const int slots = t.threads >> t.log_gx, need = (s.C + slots - 1) / slots;
        t.kc = !held ? 0 : need > 2 ? 4 : need;
        return t;
    };
    // Forward: 256 threads are better than 512 (64 x 256 x 28 x 28 bf16 28 us, 32; 64 x 160 x 28 x 28 21, 25), eight pieces better than
    // four with half the channels (64 x 72 x 56 x 56 31 us, 35).  Backward: two channels leave registers for three waves per SIMD
    // (64 x 128 x 28 x 28 bf16 31 us, 38; 64 x 256 x 28 x 28 56, 74; 128 x 256 x 14 x 14 fp32 48, 57).
    p.fwd = tiling(4);
    p.bwd = tiling(2);
    const int64_t tiles = (p.total + (1 << p.bwd.log_gx) - 1) >> p.bwd.log_gx;
    // (workgroups that the registers of the held ones leave room for: 64 x 64 x 56 x 56 bf16 takes 47 us with three on a compute
    // unit, 51 with two; fp32 95 and 87.  Channels that are read again: two on a compute unit push each other's out of the cache,
    // 64 x 4096 x 7 x 7 fp32 450 us, with one 372; two pixels at a time 1000 x 2048 x 2 x 3 127 and 154)
    p.partials = (int)std::min<int64_t>(tiles, !held && p.vec > 2 ? 256 : s.bf16 && held && p.bwd.kc <= 2 && p.bwd.threads == 256 ? 768 : 512);
    return p;
}

void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    if (s.bf16)
        run_parts<uint16_t>(s, p, a, stream);
    else
        run_parts<float>(s, p, a, stream);
}

void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    if (p.tpr)
        rows_backward(s, p, a, stream);
    else
        maps_backward(s, p, a, stream);
    CANVAS_LAUNCH(k_sums, dim3((2 * s.C + 63) / 64), dim3(64 * kSumSlices), 0, stream, s, a, p.partials);
}

}  // namespace norm
}  // namespace canvas
