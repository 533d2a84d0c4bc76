// What the kernels of the residual norm share: how maps are accessed, the gate, sums over channels.
#pragma once
#include <hip/hip_runtime.h>

#include "device_util.hpp"
#include "exp_util.hpp"
#include "norm_kernels.hpp"
#include "tile_util.hpp"
#include "wave_util.hpp"

namespace canvas {
namespace norm {

constexpr int kPost = 1, kPre = 2;

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

// act and act' of the gate: 0 none, 1 sigmoid, 2 g * sigmoid(g).
// For maps in fp32 with the rounding of the power's exponent made good, which is 4e-6 at gates of -80 (1 / (1 + E (1 + c)) is
// s (1 - (1 - s) c); an infinite gate leaves c without a value and (1 - s) s zero); maps in bf16 are rounded by 2e-3.
template <class T>
__device__ __forceinline__ float sigmoid(float g) {
    const float t = -g * kLog2e, s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t));
    return sizeof(T) == 4 ? fmaf(-s * (1.f - s), fmaxf(exp_rest(-g, t), -1.f), s) : s;
}
template <class T, int GATE>
__device__ __forceinline__ float act(float g) {
    return GATE == 0 ? 1.f : GATE == 1 ? sigmoid<T>(g) : g * sigmoid<T>(g);
}
template <class T, int GATE>
__device__ __forceinline__ float act_slope(float g, float& a) {
    if (GATE == 0) {
        a = 1.f;
        return 0.f;
    }
    const float s = sigmoid<T>(g);
    a = GATE == 1 ? s : g * s;
    return GATE == 1 ? s - s * s : s + a * (1.f - s);
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
    if (GX <= 1) {
#pragma unroll
        for (int e = 0; e < VEC; e++) v[e] = wave::step<1, wave::Sum>(v[e]);
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

// f(k, c) for the channels cy, cy + CY, ... of a thread: KC of them that it holds, or, with KC = 0, one after the other.
template <int KC, class F>
__device__ __forceinline__ void each_channel(int cy, int CY, int C, F f) {
    if constexpr (KC > 0) {
#pragma unroll
        for (int k = 0; k < KC; k++) {
            const int c = cy + k * CY;
            if (c < C) f(k, c);
        }
    } else {
#pragma unroll 4
        for (int c = cy; c < C; c += CY) f(0, c);
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

}  // namespace norm
}  // namespace canvas
