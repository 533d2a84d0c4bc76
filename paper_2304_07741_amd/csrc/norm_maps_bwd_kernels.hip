// Residual norm, backward on maps (planes of two pixels or more), tiled as the forward kernels of norm_kernels.hip.
//
// Three passes over a tile that stays in registers, with x' computed again from x, z and the gate in the first two:
//   T1 = sum_c du w_pre x'                                    per pixel
//   D = dx_out + du w_pre r1 - x' (r1^3 T1 / C) = dx;  dw_pre += du x' r1;  K += D m;  T2 = sum_c D m scale w_post,  m = act z r2
//   E = D scale w_post r2:  dz = E act - z (r2^2 T2 / C),  dgate = E z act'
// Bound by memory: eight maps move (five read, three written).  Some 50 operations per element are left beside them, which take
// about as long where 8 pixels of bf16 lie in 16 bytes, so what only depends on the pixel is multiplied per pixel, and the gate's
// kind is a constant of the kernel.  With the sums over the partials, over three sets of maps in turn: 64 x 64 x 56 x 56 in 48 us bf16
// (4.2 TB/s) and 86 us fp32 (4.8 TB/s), 64 x 256 x 28 x 28 in 63 us (3.3 TB/s), 128 x 256 x 14 x 14 in 38 us (2.7 TB/s; fp32 63 us, 3.3
// TB/s), 128 x 512 x 7 x 7 in 24 us (2.1 TB/s): four channels per thread leave two waves per SIMD, and the short planes' pieces overlap (56 pixels read for 49).
#include <atomic>

#include "../../include/canvas_norm.h"
#include "launch.hpp"
#include "norm_device.hpp"

namespace canvas {
namespace norm {
namespace {

// KC = 2 is held to the registers of three waves per SIMD (64 x 64 x 56 x 56 in bf16: 46 us, with two 54 us).
template <class T, int VEC, int KC, int PARTS, int GATE>
__global__ __launch_bounds__(512, KC == 2 ? 3 : 1) void k_maps_bwd(Shape s, Bwd a, int log_gx, int pieces, int64_t total) {
    extern __shared__ float lds[];
    const int GX = 1 << log_gx, gx = threadIdx.x & (GX - 1), cy = threadIdx.x >> log_gx, CY = blockDim.x >> log_gx;
    const float inv = 1.f / s.C;
    constexpr bool kIsPost = PARTS & kPost, kIsPre = PARTS & kPre;
    constexpr int K = KC ? KC : 1;
    float* sums = lds + (blockDim.x >> 6) * GX * VEC;  // KC = 0: [2][C]
    float kp[K], kx[K], sw[K], w1[K];
    auto each = [&](auto f) { each_channel<KC>(cy, CY, s.C, f); };
    auto weights = [&](int k, int c) {
        sw[k] = kIsPost ? a.scale[c] * a.w_post[c] : 0.f;
        w1[k] = kIsPre ? a.w_pre[c] : 0.f;
    };
#pragma unroll
    for (int k = 0; k < K; k++) kp[k] = kx[k] = sw[k] = w1[k] = 0.f;
    if (KC) {
        each(weights);
    } else {
        for (int i = threadIdx.x; i < 2 * s.C; i += blockDim.x) sums[i] = 0.f;
        __syncthreads();
    }
    const int64_t tiles = (total + GX - 1) >> log_gx;
    for (int64_t place = tile::xcd_sequence(); place < tiles; place += gridDim.x) {
        const Where at = where_of<VEC>(s, pieces, total, (place << log_gx) + gx);
        Vec<T, VEC> x[K], z[K], g[K], dy[K], du[K];
        auto load = [&](int k, int c, bool arriving) {
            const int64_t i = at.base + c * s.P;
            if (kIsPre) {
                x[k].load(a.x, i);
                du[k].load(a.du, i);
            }
            if (kIsPost) z[k].load(a.z, i);
            if (GATE) g[k].load(a.g, i);
            if (arriving && a.dx_out) dy[k].load(a.dx_out, i);
        };
        if (KC) each([&](int k, int c) { load(k, c, true); });
        // what a pass needs again: from the registers, computed anew, or from memory
        auto again = [&](int k, int c, bool arriving) {
            if (!KC) {
                weights(k, c);
                load(k, c, arriving);
                return;
            }
            if (kIsPre) {
                x[k].renew();
                du[k].renew();
            }
            if (kIsPost) z[k].renew();
            if (GATE) g[k].renew();
        };
        float r2[VEC], r1[VEC], t1[VEC], t2[VEC];
        bool once[VEC];  // false for pixels that the piece before counts
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            r2[e] = kIsPost ? a.r2[at.pixel + e] : 0.f;
            r1[e] = kIsPre ? a.r1[at.pixel + e] : 0.f;
            t1[e] = t2[e] = 0.f;
            once[e] = at.in && e >= at.skip;
        }
        // m, kept from the first pass for the second where there is room
        constexpr bool kKeep = KC == 1 || KC == 2;
        constexpr int KM = kKeep ? K : 1;
        float m[KM][VEC], d[K][VEC];
        auto branch = [&](int k) {
#pragma unroll
            for (int e = 0; e < VEC; e++) m[k % KM][e] = kIsPost ? act<T, GATE>(GATE ? g[k].at(e) : 0.f) * (z[k].at(e) * r2[e]) : 0.f;
        };
        auto joined = [&](int k, int e) { return kIsPost ? x[k].at(e) + sw[k] * m[k % KM][e] : x[k].at(e); };  // x'
        auto whole = [&](int k, int e, float y) {                                                              // D
            const float dy_e = a.dx_out ? dy[k].at(e) : 0.f;
            return kIsPre ? dy_e - y * t1[e] + du[k].at(e) * w1[k] * r1[e] : dy_e;
        };
        if (kIsPre) {
            each([&](int k, int c) {
                if (!KC) again(k, c, false);
                branch(k);
#pragma unroll
                for (int e = 0; e < VEC; e++) t1[e] += du[k].at(e) * w1[k] * joined(k, e);
            });
            over_channels<VEC>(t1, gx, GX, lds);
#pragma unroll
            for (int e = 0; e < VEC; e++) t1[e] = t1[e] * inv * r1[e] * r1[e] * r1[e];  // (the power alone may leave the range)
        }
        each([&](int k, int c) {
            again(k, c, true);
            if (!kKeep || !kIsPre) branch(k);
            float sp = 0.f, sx = 0.f;
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                const float y = kIsPre ? joined(k, e) : 0.f;
                d[k][e] = whole(k, e, y);
                if (kIsPost) {
                    const float p = d[k][e] * m[k % KM][e];
                    t2[e] += p * sw[k];
                    sp += once[e] ? p : 0.f;
                }
                if (kIsPre) sx += once[e] ? du[k].at(e) * y * r1[e] : 0.f;
            }
            if (KC) {
                kp[k] += sp;
                kx[k] += sx;
            } else {
                for (int o = GX >> 1; o; o >>= 1) {
                    sp += __shfl_xor(sp, o);
                    sx += __shfl_xor(sx, o);
                }
                if (gx == 0) {
                    sums[c] += sp;
                    sums[s.C + c] += sx;
                }
            }
            if (kIsPre && at.in) store<T, VEC>(a.dx, at.base + c * s.P, d[k]);
        });
        if (kIsPost) {
            over_channels<VEC>(t2, gx, GX, lds);
#pragma unroll
            for (int e = 0; e < VEC; e++) t2[e] = t2[e] * inv * r2[e] * r2[e];
            each([&](int k, int c) {
                again(k, c, true);
                if (!KC) branch(k);
                float dz[VEC], dg[VEC];
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    float av;
                    const float slope = act_slope<T, GATE>(GATE ? g[k].at(e) : 0.f, av);
                    const float D = KC ? d[k][e] : whole(k, e, kIsPre ? joined(k, e) : 0.f), E = D * (sw[k] * r2[e]), zv = z[k].at(e);
                    dz[e] = E * av - zv * t2[e];
                    dg[e] = E * zv * slope;
                }
                if (at.in) {
                    store<T, VEC>(a.dz, at.base + c * s.P, dz);
                    if (GATE) store<T, VEC>(a.dg, at.base + c * s.P, dg);
                }
            });
        }
    }
    float* out = a.partial + (int64_t)blockIdx.x * 2 * s.C;
    if (KC) {
        each([&](int k, int c) {
            for (int o = GX >> 1; o; o >>= 1) {
                kp[k] += __shfl_xor(kp[k], o);
                kx[k] += __shfl_xor(kx[k], o);
            }
            if (gx == 0) {
                out[c] = kp[k];
                out[s.C + c] = kx[k];
            }
        });
    } else {
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * s.C; i += blockDim.x) out[i] = sums[i];
    }
}

template <class T, int VEC, int KC, int PARTS, int GATE>
void maps(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    const Tiling& t = p.bwd;
    constexpr int kMost = 512 / 64 * 8 * VEC * 4 + 8 * CANVAS_NORM_MAX_CHANNELS;  // eight pieces side by side, all channels' sums
    const int lds = t.threads / 64 * (1 << t.log_gx) * VEC * 4 + (KC ? 0 : 8 * s.C);
    if (lds > 65536) {
        static std::atomic<uint64_t> asked{0};
        allow_lds(asked, reinterpret_cast<const void*>(&k_maps_bwd<T, VEC, KC, PARTS, GATE>), kMost);
    }
    CANVAS_LAUNCH((k_maps_bwd<T, VEC, KC, PARTS, GATE>), dim3(p.partials), dim3(t.threads), lds, stream, s, a, t.log_gx, p.pieces, p.total);
}
template <class T, int PARTS, int GATE>
void run(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    if (p.vec == 2) return maps<T, 2, 0, PARTS, GATE>(s, p, a, stream);
    switch (p.bwd.kc) {
    case 1: return maps<T, V, 1, PARTS, GATE>(s, p, a, stream);
    case 2: return maps<T, V, 2, PARTS, GATE>(s, p, a, stream);
    case 4: return maps<T, V, 4, PARTS, GATE>(s, p, a, stream);
    default: return maps<T, V, 0, PARTS, GATE>(s, p, a, stream);
    }
}
template <class T>
void run_parts(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    constexpr int kBoth = kPost | kPre;
    if (!s.post) return run<T, kPre, 0>(s, p, a, stream);
    switch (s.gate) {
    case 0: return s.pre ? run<T, kBoth, 0>(s, p, a, stream) : run<T, kPost, 0>(s, p, a, stream);
    case 1: return s.pre ? run<T, kBoth, 1>(s, p, a, stream) : run<T, kPost, 1>(s, p, a, stream);
    default: return s.pre ? run<T, kBoth, 2>(s, p, a, stream) : run<T, kPost, 2>(s, p, a, stream);
    }
}

}  // namespace

void maps_backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    if (s.bf16)
        run_parts<uint16_t>(s, p, a, stream);
    else
        run_parts<float>(s, p, a, stream);
}

}  // namespace norm
}  // namespace canvas
