// Residual norm, forward and backward.  Both are bound by memory: five maps move forward, eight backward, and everything in
// between stays in registers.
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
#include <atomic>

#include "device_util.hpp"
#include "launch.hpp"
#include "tile_util.hpp"
#include "wave_util.hpp"

namespace canvas {
namespace norm {
namespace {

constexpr int kPost = 1, kPre = 2;
constexpr float kLog2e = 1.4426950408889634f;

// N elements of a map as they are in memory.
template <class T, int N>
struct Vec {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ float at(int e) const {
        if (sizeof(T) == 4) return __uint_as_float(w[e]);
        return (e & 1) ? tile::hi_f32(w[e >> 1]) : tile::lo_f32(w[e >> 1]);
    }
    // What is computed from it behind this point is computed anew: kept results of an earlier pass take more registers than there are.
    __device__ __forceinline__ void renew() {
#pragma unroll
        for (int k = 0; k < kWords; k++) asm volatile("" : "+v"(w[k]));
    }
    __device__ __forceinline__ void load(const void* p, int64_t i) { __builtin_memcpy(w, static_cast<const T*>(p) + i, sizeof w); }
};
template <class T, int N>
__device__ __forceinline__ void store(void* p, int64_t i, const float (&v)[N]) {
    uint32_t w[Vec<T, N>::kWords];
    if (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < N; e++) w[e % Vec<T, N>::kWords] = __float_as_uint(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N / 2; e++) w[e] = tile::pack_bf16(v[2 * e], v[2 * e + 1]);
    }
    __builtin_memcpy(static_cast<T*>(p) + i, w, sizeof w);
}

// act(g) and act'(g)
struct Act {
    float a = 1.f, da = 0.f;
};
__device__ __forceinline__ Act act_of(int kind, float g) {
    Act r;
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-g * kLog2e));
    const float rest = s * (1.f - s);
    r.a = kind == 1 ? s : g * s;
    r.da = kind == 1 ? rest : s + g * rest;
    return r;
}

// ---------------------------------------------------------------- maps

// Where a thread is: piece number `q` of all (n, first pixel), `skip` pixels in common with the piece before it.
struct Where {
    bool in;
    int64_t pixel, base;  // of N * P; of the first channel
    int skip;
};
template <int VEC>
__device__ __forceinline__ Where where_of(const Shape& s, int pieces, int64_t total, int64_t q) {
    Where w;
    w.in = q < total;
    if (!w.in) q = total - 1;
    const int64_t n = (uint64_t)q < 0x80000000ull ? (int64_t)((uint32_t)q / (uint32_t)pieces) : q / pieces;
    const int g = (int)(q - n * pieces);
    int64_t p = (int64_t)g * VEC;
    w.skip = 0;
    if (p + VEC > s.P) {
        w.skip = (int)(p + VEC - s.P);
        p = s.P - VEC;
    }
    w.pixel = n * s.P + p;
    w.base = n * s.C * s.P + p;
    return w;
}

// Sums of v over the channel slots of each pixel: lanes gx, gx + GX, ... of all waves.  buf: a row of GX * VEC floats per wave.
template <int VEC>
__device__ __forceinline__ void over_channels(float (&v)[VEC], int gx, int GX, float* buf) {
#pragma unroll
    for (int e = 0; e < VEC; e++) v[e] = wave::over<16, wave::Sum>(v[e]);
    if (GX <= 8) {
#pragma unroll
        for (int e = 0; e < VEC; e++) v[e] = wave::step<8, wave::Sum>(v[e]);
    }
    if (GX <= 4) {
#pragma unroll
        for (int e = 0; e < VEC; e++) v[e] = wave::step<4, wave::Sum>(v[e]);
    }
    if (GX <= 2) {
#pragma unroll
        for (int e = 0; e < VEC; e++) v[e] = wave::step<2, wave::Sum>(v[e]);
    }
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, row = GX * VEC;
    __syncthreads();
    if ((int)(threadIdx.x & 63) < GX) {
#pragma unroll
        for (int e = 0; e < VEC; e++) buf[wave * row + gx * VEC + e] = v[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VEC; e++) v[e] = 0.f;
    for (int w = 0; w < waves; w++) {
#pragma unroll
        for (int e = 0; e < VEC; e++) v[e] += buf[w * row + gx * VEC + e];
    }
}

template <class T, int VEC, int KC, int PARTS>
__global__ __launch_bounds__(512) void k_maps_fwd(Shape s, Fwd a, int log_gx, int pieces, int64_t total) {
    extern __shared__ float lds[];
    const int GX = 1 << log_gx, gx = threadIdx.x & (GX - 1), cy = threadIdx.x >> log_gx, CY = blockDim.x >> log_gx;
    const Where at = where_of<VEC>(s, pieces, total, (int64_t)tile::xcd_sequence() * GX + gx);
    const float inv = 1.f / s.C;
    const bool gated = (PARTS & kPost) && s.gate;
    constexpr int K = KC ? KC : 1;
    Vec<T, VEC> x[K], z[K], g[K];
    auto load_z = [&](int k, int c) { z[k].load(a.z, at.base + c * s.P); };
    auto load_x = [&](int k, int c) {
        x[k].load(a.x, at.base + c * s.P);
        if (gated) g[k].load(a.g, at.base + c * s.P);
    };
    // f(k, c) for this thread's channels
    auto each = [&](auto f) {
        if constexpr (KC > 0) {
#pragma unroll
            for (int k = 0; k < KC; k++) {
                const int c = cy + k * CY;
                if (c < s.C) f(k, c);
            }
        } else {
            for (int c = cy; c < s.C; c += CY) f(0, c);
        }
    };
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
            for (int e = 0; e < VEC; e++) r2[e] += z[k].at(e) * z[k].at(e);
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
        if (PARTS & kPost) y += sw * (gated ? act_of(s.gate, g[k].at(e)).a : 1.f) * (z[k].at(e) * r2[e]);
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
            t[e] += y[k][e] * y[k][e];
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

template <class T, int VEC, int KC, int PARTS>
__global__ __launch_bounds__(512) void k_maps_bwd(Shape s, Bwd a, int log_gx, int pieces, int64_t total) {
    extern __shared__ float lds[];
    const int GX = 1 << log_gx, gx = threadIdx.x & (GX - 1), cy = threadIdx.x >> log_gx, CY = blockDim.x >> log_gx;
    const float inv = 1.f / s.C;
    const bool gated = (PARTS & kPost) && s.gate;
    constexpr int K = KC ? KC : 1;
    float* sums = lds + (blockDim.x >> 6) * GX * VEC;  // KC = 0: [2][C]
    float kp[K], kx[K], sw[K], w1[K];
    auto each = [&](auto f) {
        if constexpr (KC > 0) {
#pragma unroll
            for (int k = 0; k < KC; k++) {
                const int c = cy + k * CY;
                if (c < s.C) f(k, c);
            }
        } else {
            for (int c = cy; c < s.C; c += CY) f(0, c);
        }
    };
    auto weights = [&](int k, int c) {
        sw[k] = PARTS & kPost ? a.scale[c] * a.w_post[c] : 0.f;
        w1[k] = PARTS & kPre ? a.w_pre[c] : 0.f;
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
    const bool overlap = (int64_t)pieces * VEC > s.P;
    for (int64_t place = tile::xcd_sequence(); place < tiles; place += gridDim.x) {
        const Where at = where_of<VEC>(s, pieces, total, (place << log_gx) + gx);
        Vec<T, VEC> x[K], z[K], g[K], dy[K], du[K];
        auto load = [&](int k, int c, bool arriving) {
            const int64_t i = at.base + c * s.P;
            if (PARTS & kPre) {
                x[k].load(a.x, i);
                du[k].load(a.du, i);
            }
            if (PARTS & kPost) z[k].load(a.z, i);
            if (gated) g[k].load(a.g, i);
            if (arriving && a.dx_out) dy[k].load(a.dx_out, i);
        };
        auto renew = [&](int k) {
            if (PARTS & kPre) {
                x[k].renew();
                du[k].renew();
            }
            if (PARTS & kPost) z[k].renew();
            if (gated) g[k].renew();
        };
        if (KC) each([&](int k, int c) { load(k, c, true); });
        float r2[VEC], r1[VEC], t1[VEC], t2[VEC];
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            r2[e] = PARTS & kPost ? a.r2[at.pixel + e] : 0.f;
            r1[e] = PARTS & kPre ? a.r1[at.pixel + e] : 0.f;
            t1[e] = t2[e] = 0.f;
        }
        // m = act zh, kept from the first pass for the second where there is room
        constexpr bool kKeep = KC == 1 || KC == 2;
        constexpr int KM = kKeep ? K : 1;
        float m[KM][VEC], d[K][VEC];
        auto branch = [&](int k) {
#pragma unroll
            for (int e = 0; e < VEC; e++) m[k % KM][e] = PARTS & kPost ? (gated ? act_of(s.gate, g[k].at(e)).a : 1.f) * (z[k].at(e) * r2[e]) : 0.f;
        };
        auto unit = [&](int k, int e) { return (PARTS & kPost ? x[k].at(e) + sw[k] * m[k % KM][e] : x[k].at(e)) * r1[e]; };  // xh
        auto whole = [&](int k, int e, float xh) {                                                                       // D
            const float dy_e = a.dx_out ? dy[k].at(e) : 0.f;
            return PARTS & kPre ? dy_e + r1[e] * (du[k].at(e) * w1[k] - xh * t1[e]) : dy_e;
        };
        if (PARTS & kPre) {
            each([&](int k, int c) {
                if (!KC) {
                    weights(k, c);
                    load(k, c, false);
                }
                branch(k);
#pragma unroll
                for (int e = 0; e < VEC; e++) t1[e] += du[k].at(e) * w1[k] * unit(k, e);
            });
            over_channels<VEC>(t1, gx, GX, lds);
#pragma unroll
            for (int e = 0; e < VEC; e++) t1[e] *= inv;
        }
        each([&](int k, int c) {
            if (!KC) {
                weights(k, c);
                load(k, c, true);
            } else {
                renew(k);
            }
            if (!kKeep || !(PARTS & kPre)) branch(k);
            float sp = 0.f, sx = 0.f;
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                const float xh = PARTS & kPre ? unit(k, e) : 0.f;
                d[k][e] = whole(k, e, xh);
                float p = PARTS & kPost ? d[k][e] * m[k % KM][e] : 0.f, q = PARTS & kPre ? du[k].at(e) * xh : 0.f;
                t2[e] += p * sw[k];
                if (overlap && e < at.skip) p = q = 0.f;
                sp += p;
                sx += q;
            }
            if (!at.in) sp = sx = 0.f;
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
            if ((PARTS & kPre) && at.in) store<T, VEC>(a.dx, at.base + c * s.P, d[k]);
        });
        if (PARTS & kPost) {
            over_channels<VEC>(t2, gx, GX, lds);
#pragma unroll
            for (int e = 0; e < VEC; e++) t2[e] *= inv;
            each([&](int k, int c) {
                if (!KC) {
                    weights(k, c);
                    load(k, c, true);
                    branch(k);
                } else {
                    renew(k);
                }
                float dz[VEC], dg[VEC];
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    Act act;
                    if (gated) act = act_of(s.gate, g[k].at(e));
                    const float D = (KC ? d[k][e] : whole(k, e, PARTS & kPre ? unit(k, e) : 0.f)) * sw[k], zh = z[k].at(e) * r2[e];
                    dz[e] = r2[e] * (D * act.a - zh * t2[e]);
                    dg[e] = D * act.da * zh;
                }
                if (at.in) {
                    store<T, VEC>(a.dz, at.base + c * s.P, dz);
                    if (gated) store<T, VEC>(a.dg, at.base + c * s.P, dg);
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

// ---------------------------------------------------------------- rows

// Over the TPR threads of a row; buf: a float per wave of the workgroup.
template <int TPR>
__device__ __forceinline__ float over_row(float v, float* buf) {
    if (TPR == 16) {  // (rotations of a row of 16 lanes)
        v = wave::step<8, wave::Sum>(v);
        v = wave::step<4, wave::Sum>(v);
        v = wave::step<2, wave::Sum>(v);
        return wave::step<1, wave::Sum>(v);
    }
    v = wave::over<1, wave::Sum>(v);
    if (TPR == 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; w++) v += buf[w];
    return v;
}

// N elements from i on, those behind the row's end as zeros.
template <class T, int N>
__device__ __forceinline__ void load_row(Vec<T, N>& v, const void* p, int64_t row, int c, int C) {
    if (c + N <= C) {
        v.load(p, row + c);
        return;
    }
#pragma unroll
    for (int w = 0; w < Vec<T, N>::kWords; w++) v.w[w] = 0;
#pragma unroll
    for (int e = 0; e < N; e++)
        if (c + e < C) {
            if (sizeof(T) == 4)
                v.w[e % Vec<T, N>::kWords] = static_cast<const uint32_t*>(p)[row + c + e];
            else
                v.w[e >> 1] |= (uint32_t) static_cast<const uint16_t*>(p)[row + c + e] << ((e & 1) * 16);
        }
}
template <class T, int N>
__device__ __forceinline__ void store_row(void* p, int64_t row, int c, int C, const float (&v)[N]) {
    if (c + N <= C) {
        store<T, N>(p, row + c, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < N; e++)
        if (c + e < C) {
            if (sizeof(T) == 4)
                static_cast<float*>(p)[row + c + e] = v[e];
            else
                static_cast<uint16_t*>(p)[row + c + e] = f32_to_bf16(v[e]);
        }
}
template <int N>
__device__ __forceinline__ void load_weights(float (&w)[N], const float* p, int c, int C) {
    if (c + N <= C) {
        __builtin_memcpy(w, p + c, sizeof w);
        return;
    }
#pragma unroll
    for (int e = 0; e < N; e++) w[e] = c + e < C ? p[c + e] : 0.f;
}

template <int N>
__device__ __forceinline__ void store_floats(float* p, int c, int C, const float (&v)[N]) {
#pragma unroll
    for (int e = 0; e < N; e++)
        if (c + e < C) p[c + e] = v[e];
}

template <class T, int TPR, int KV, int PARTS>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_rows_fwd(Shape s, Fwd a) {
    constexpr int V = 16 / sizeof(T), kRows = TPR < 256 ? 256 / TPR : 1;
    __shared__ float buf[16];
    const int t = threadIdx.x % TPR;
    const int64_t n = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    if (n >= s.N) return;  // (with several rows per workgroup a row is within a wave: no barriers)
    const int64_t row = n * s.C;
    const bool gated = (PARTS & kPost) && s.gate;
    const float inv = 1.f / s.C;
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
            for (int e = 0; e < V; e++) r2 += z[k].at(e) * z[k].at(e);
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
            if (PARTS & kPost) y[e] += sw[e] * w[e] * (gated ? act_of(s.gate, g[k].at(e)).a : 1.f) * (z[k].at(e) * r2);
        }
    };
    float y[V], r1 = 0.f;
#pragma unroll
    for (int k = 0; k < KV; k++) {
        joined(k, y);
#pragma unroll
        for (int e = 0; e < V; e++) r1 += y[e] * y[e];
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

// Rows of 1024 threads have no registers for the sums and the weights of their channels: sums in LDS, weights read again; the
// longest have none for the values either, which are read again for each pass.
template <class T, int TPR, int KV, int PARTS>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_rows_bwd(Shape s, Bwd a) {
    constexpr int V = 16 / sizeof(T), kRows = TPR < 256 ? 256 / TPR : 1;
    constexpr bool kLong = TPR == 1024;
    constexpr bool kAgain = kLong && KV > 1;
    constexpr int KS = kLong ? 1 : KV, KX = kAgain ? 1 : KV;
    extern __shared__ float lds[];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const bool gated = (PARTS & kPost) && s.gate;
    const float inv = 1.f / s.C;
    float sw[KS][V], w1[KS][V], kp[KS][V], kx[KS][V];
    float* sums = lds + 16;  // kLong: [2][KV * V][TPR]
    auto weights = [&](int k, int c) {
        if (PARTS & kPost) {
            float w[V];
            load_weights<V>(w, a.w_post, c, s.C);
            load_weights<V>(sw[k], a.scale, c, s.C);
#pragma unroll
            for (int e = 0; e < V; e++) sw[k][e] *= w[e];
        }
        if (PARTS & kPre) load_weights<V>(w1[k], a.w_pre, c, s.C);
    };
#pragma unroll
    for (int k = 0; k < KV; k++) {
        if (!kLong) weights(k, (k * TPR + t) * V);
#pragma unroll
        for (int e = 0; e < V; e++) {
            if (kLong)
                sums[(k * V + e) * TPR + t] = sums[((KV + k) * V + e) * TPR + t] = 0.f;
            else
                kp[k % KS][e] = kx[k % KS][e] = 0.f;
        }
    }
    for (int64_t n = (int64_t)blockIdx.x * kRows + sub; n < s.N; n += (int64_t)gridDim.x * kRows) {
        const int64_t row = n * s.C;
        Vec<T, V> x[KX], z[KX], g[KX], dy[KX], du[KX];
        auto load = [&](int k, int c) {
            if (PARTS & kPre) {
                load_row<T, V>(x[k], a.x, row, c, s.C);
                load_row<T, V>(du[k], a.du, row, c, s.C);
            }
            if (PARTS & kPost) load_row<T, V>(z[k], a.z, row, c, s.C);
            if (gated) load_row<T, V>(g[k], a.g, row, c, s.C);
            if (a.dx_out) load_row<T, V>(dy[k], a.dx_out, row, c, s.C);
        };
        if (!kAgain) {
#pragma unroll
            for (int k = 0; k < KV; k++) load(k % KX, (k * TPR + t) * V);
        }
        const float r2 = PARTS & kPost ? a.r2[n] : 0.f, r1 = PARTS & kPre ? a.r1[n] : 0.f;
        float t1 = 0.f, t2 = 0.f;
        auto renew = [&](int k) {
            if (kAgain) load(0, (k * TPR + t) * V);
            if (PARTS & kPre) {
                x[k % KX].renew();
                du[k % KX].renew();
            }
            if (PARTS & kPost) z[k % KX].renew();
            if (gated) g[k % KX].renew();
            if (kLong) weights(0, (k * TPR + t) * V);
        };
        // m = act zh, kept from the first pass for the second
        float m[KX][V], d[KX][V];
        auto branch = [&](int k) {
#pragma unroll
            for (int e = 0; e < V; e++)
                m[k % KX][e] = PARTS & kPost ? (gated ? act_of(s.gate, g[k % KX].at(e)).a : 1.f) * (z[k % KX].at(e) * r2) : 0.f;
        };
        auto unit = [&](int k, int e) { return (PARTS & kPost ? x[k % KX].at(e) + sw[k % KS][e] * m[k % KX][e] : x[k % KX].at(e)) * r1; };  // xh
        auto whole = [&](int k, int e, float xh) {                                                                                     // D
            const float dy_e = a.dx_out ? dy[k % KX].at(e) : 0.f;
            return PARTS & kPre ? dy_e + r1 * (du[k % KX].at(e) * w1[k % KS][e] - xh * t1) : dy_e;
        };
        if (PARTS & kPre) {
#pragma unroll(kAgain ? 1 : KV)
            for (int k = 0; k < KV; k++) {
                if (kLong) renew(k);
                branch(k);
#pragma unroll
                for (int e = 0; e < V; e++) t1 += du[k % KX].at(e) * w1[k % KS][e] * unit(k, e);
            }
            t1 = over_row<TPR>(t1, lds) * inv;
        }
#pragma unroll(kAgain ? 1 : KV)
        for (int k = 0; k < KV; k++) {
            renew(k);
            if (kAgain || !(PARTS & kPre)) branch(k);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float xh = PARTS & kPre ? unit(k, e) : 0.f;
                d[k % KX][e] = whole(k, e, xh);
                if (PARTS & kPost) {
                    const float p = d[k % KX][e] * m[k % KX][e];
                    t2 += p * sw[k % KS][e];
                    if (kLong)
                        sums[(k * V + e) * TPR + t] += p;
                    else
                        kp[k % KS][e] += p;
                }
                if (PARTS & kPre) {
                    const float q = du[k % KX].at(e) * xh;
                    if (kLong)
                        sums[((KV + k) * V + e) * TPR + t] += q;
                    else
                        kx[k % KS][e] += q;
                }
            }
            if (PARTS & kPre) store_row<T, V>(a.dx, row, (k * TPR + t) * V, s.C, d[k % KX]);
        }
        if (PARTS & kPost) {
            t2 = over_row<TPR>(t2, lds) * inv;
#pragma unroll(kAgain ? 1 : KV)
            for (int k = 0; k < KV; k++) {
                renew(k);
                if (kAgain) branch(k);
                float dz[V], dg[V];
#pragma unroll
                for (int e = 0; e < V; e++) {
                    Act act;
                    if (gated) act = act_of(s.gate, g[k % KX].at(e));
                    const float D = (kAgain ? whole(k, e, PARTS & kPre ? unit(k, e) : 0.f) : d[k % KX][e]) * sw[k % KS][e], zh = z[k % KX].at(e) * r2;
                    dz[e] = r2 * (D * act.a - zh * t2);
                    dg[e] = D * act.da * zh;
                }
                store_row<T, V>(a.dz, row, (k * TPR + t) * V, s.C, dz);
                if (gated) store_row<T, V>(a.dg, row, (k * TPR + t) * V, s.C, dg);
            }
        }
    }
    // the rows of a workgroup in order, then its partial sums
    float* out = a.partial + (int64_t)blockIdx.x * 2 * s.C;
    if (kRows == 1) {
#pragma unroll
        for (int k = 0; k < KV; k++) {
            const int c = (k * TPR + t) * V;
            if (kLong) {
#pragma unroll
                for (int e = 0; e < V; e++) {
                    kp[0][e] = sums[(k * V + e) * TPR + t];
                    kx[0][e] = sums[((KV + k) * V + e) * TPR + t];
                }
            }
            store_floats<V>(out, c, s.C, kp[k % KS]);
            store_floats<V>(out + s.C, c, s.C, kx[k % KS]);
        }
        return;
    }
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
        for (int k = 0; k < KV; k++) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; e++) lds[threadIdx.x * V + e] = h ? kx[k % KS][e] : kp[k % KS][e];
            __syncthreads();
            for (int i = threadIdx.x; i < TPR * V; i += 256) {
                float v = 0.f;
#pragma unroll
                for (int r = 0; r < kRows; r++) v += lds[r * TPR * V + i];
                const int c = k * TPR * V + i;
                if (c < s.C) out[h * s.C + c] = v;
            }
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
void maps(const Shape& s, const Plan& p, const Fwd* f, const Bwd* b, hipStream_t stream) {
    const int64_t tiles = (p.total + (1 << p.log_gx) - 1) >> p.log_gx;
    const int lds = p.threads / 64 * (1 << p.log_gx) * VEC * 4;
    if (f) {
        CANVAS_LAUNCH((k_maps_fwd<T, VEC, KC, PARTS>), dim3((unsigned)tiles), dim3(p.threads), lds, stream, s, *f, p.log_gx, p.pieces, p.total);
    } else {
        const int all = lds + (KC ? 0 : 8 * s.C);
        if (all > 65536) {
            static std::atomic<uint64_t> asked{0};
            allow_lds(asked, reinterpret_cast<const void*>(&k_maps_bwd<T, VEC, KC, PARTS>), all);
        }
        CANVAS_LAUNCH((k_maps_bwd<T, VEC, KC, PARTS>), dim3(p.partials), dim3(p.threads), all, stream, s, *b, p.log_gx, p.pieces, p.total);
    }
}
template <class T, int TPR, int KV, int PARTS>
void rows(const Shape& s, const Plan& p, const Fwd* f, const Bwd* b, hipStream_t stream) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, kRows = kBlock / TPR;
    if (f)
        CANVAS_LAUNCH((k_rows_fwd<T, TPR, KV, PARTS>), dim3((unsigned)((s.N + kRows - 1) / kRows)), dim3(kBlock), 0, stream, s, *f);
    else {
        const int lds = kRows > 1 ? 256 * 64 / (int)sizeof(T) : 64 + (TPR == 1024 ? TPR * KV * 128 / (int)sizeof(T) : 0);
        if (lds > 65536) {
            static std::atomic<uint64_t> asked{0};
            allow_lds(asked, reinterpret_cast<const void*>(&k_rows_bwd<T, TPR, KV, PARTS>), lds);
        }
        CANVAS_LAUNCH((k_rows_bwd<T, TPR, KV, PARTS>), dim3(p.partials), dim3(kBlock), lds, stream, s, *b);
    }
}
template <class T, int PARTS>
void run(const Shape& s, const Plan& p, const Fwd* f, const Bwd* b, hipStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    if (p.tpr) {
        switch (p.tpr * 8 + p.kv) {
        case 16 * 8 + 1: return rows<T, 16, 1, PARTS>(s, p, f, b, stream);
        case 64 * 8 + 1: return rows<T, 64, 1, PARTS>(s, p, f, b, stream);
        case 64 * 8 + 2: return rows<T, 64, 2, PARTS>(s, p, f, b, stream);
        case 256 * 8 + 1: return rows<T, 256, 1, PARTS>(s, p, f, b, stream);
        case 256 * 8 + 2: return rows<T, 256, 2, PARTS>(s, p, f, b, stream);
        case 1024 * 8 + 1: return rows<T, 1024, 1, PARTS>(s, p, f, b, stream);
        default: return rows<T, 1024, 16 / V, PARTS>(s, p, f, b, stream);
        }
    }
    if (p.vec == 2) return maps<T, 2, 0, PARTS>(s, p, f, b, stream);
    switch (p.kc) {
    case 1: return maps<T, V, 1, PARTS>(s, p, f, b, stream);
    case 2: return maps<T, V, 2, PARTS>(s, p, f, b, stream);
    case 4: return maps<T, V, 4, PARTS>(s, p, f, b, stream);
    default: return maps<T, V, 0, PARTS>(s, p, f, b, stream);
    }
}
template <class T>
void run_parts(const Shape& s, const Plan& p, const Fwd* f, const Bwd* b, hipStream_t stream) {
    if (s.post && s.pre)
        run<T, kPost | kPre>(s, p, f, b, stream);
    else if (s.post)
        run<T, kPost>(s, p, f, b, stream);
    else
        run<T, kPre>(s, p, f, b, stream);
}

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    const int v = s.bf16 ? 8 : 4;
    if (s.P == 1) {
        const int sizes[][2] = {{16, 1}, {64, 1}, {64, 2}, {256, 1}, {256, 2}, {1024, 1}, {1024, 16 / v}};
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
    // Pieces side by side: as many as make a workgroup's share of a plane's row a cache line, fewer where that leaves compute units
    // idle or a workgroup without room for all channels.
    const bool held = p.vec == v && s.C <= 1024;
    p.log_gx = 3;
    while (p.log_gx > 1 && ((p.total >> p.log_gx) < 256 || (held && s.C > 4 * (512 >> p.log_gx)))) p.log_gx--;
    p.threads = held && s.C <= 4 * (256 >> p.log_gx) ? 256 : 512;
    const int slots = p.threads >> p.log_gx, need = (s.C + slots - 1) / slots;
    p.kc = !held ? 0 : need > 2 ? 4 : need;
    const int64_t tiles = (p.total + (1 << p.log_gx) - 1) >> p.log_gx;
    // (workgroups that the registers of the held ones leave room for: 64 x 64 x 56 x 56 bf16 takes 50 us with three on a compute
    // unit, 56 with two; fp32 97 and 90)
    p.partials = (int)std::min<int64_t>(tiles, !p.kc ? 256 : s.bf16 && p.kc <= 2 && p.threads == 256 ? 768 : 512);
    return p;
}

void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    if (s.bf16)
        run_parts<uint16_t>(s, p, &a, nullptr, stream);
    else
        run_parts<float>(s, p, &a, nullptr, stream);
}

void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    if (s.bf16)
        run_parts<uint16_t>(s, p, nullptr, &a, stream);
    else
        run_parts<float>(s, p, nullptr, &a, stream);
    CANVAS_LAUNCH(k_sums, dim3((2 * s.C + 63) / 64), dim3(64 * kSumSlices), 0, stream, s, a, p.partials);
}

}  // namespace norm
}  // namespace canvas
