// What the kernels of the orthogonalised update share.
#pragma once
#include <hip/hip_runtime.h>

#include "device_util.hpp"
#include "ortho_kernels.hpp"
#include "tile_util.hpp"

namespace canvas {
namespace ortho {

// of the quintic Newton-Schulz step that K. Jordan et al. published in "Muon: an optimizer for hidden layers in neural networks" (2024)
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr double kEps = 1e-7;

// 1 / (|v| + 1e-7) from the sum of squares.  (An infinity: NaN, so that the whole matrix is, and not the one element alone.)
__device__ __forceinline__ double inverse_norm(double squares) { return 1.0 / (sqrt(squares) + kEps) + (squares - squares); }

__device__ __forceinline__ float direction(const Shape& s, const Args& a, int64_t i, float m_new) {
    if (!a.momentum) return a.grad[i];
    return s.nesterov ? (float)(a.grad[i] + a.mu * m_new) : m_new;  // (mu in 64 bits: gradient and momentum may cancel)
}

// One element of the outputs.
__device__ __forceinline__ void finish_one(const Shape& s, const Args& a, int64_t i, float o) {
    if (a.update) {
        if (s.bf16)
            static_cast<uint16_t*>(a.update)[i] = f32_to_bf16(o);
        else
            static_cast<float*>(a.update)[i] = o;
    }
    if (a.master) {
        const float w = (float)((1.0 - a.lr * a.decay) * a.master[i] - a.lr * o);
        a.master_out[i] = w;
        if (a.weights) {
            if (s.bf16)
                static_cast<uint16_t*>(a.weights)[i] = f32_to_bf16(w);
            else
                static_cast<float*>(a.weights)[i] = w;
        }
    }
}

// Eight elements side by side from an index on that eight divides, in matrices whose size it divides: 16 bytes at a time.
__device__ __forceinline__ void put_eight(bool bf16, void* to, int64_t i, const float (&v)[8]) {
    if (bf16) {
        const tile::u32x4 w = {tile::pack_bf16(v[0], v[1]), tile::pack_bf16(v[2], v[3]), tile::pack_bf16(v[4], v[5]), tile::pack_bf16(v[6], v[7])};
        *reinterpret_cast<tile::u32x4*>(static_cast<uint16_t*>(to) + i) = w;
    } else {
        float4* f = reinterpret_cast<float4*>(static_cast<float*>(to) + i);
        f[0] = make_float4(v[0], v[1], v[2], v[3]);
        f[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}
__device__ __forceinline__ void finish_eight(const Shape& s, const Args& a, int64_t i, const float (&o)[8]) {
    if (a.update) put_eight(s.bf16, a.update, i, o);
    if (!a.master) return;
    const float4* from = reinterpret_cast<const float4*>(a.master + i);
    const float4 f0 = from[0], f1 = from[1];
    const float old[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; k++) w[k] = (float)((1.0 - a.lr * a.decay) * old[k] - a.lr * o[k]);
    put_eight(false, a.master_out, i, w);
    if (a.weights) put_eight(s.bf16, a.weights, i, w);
}

}  // namespace ortho
}  // namespace canvas
