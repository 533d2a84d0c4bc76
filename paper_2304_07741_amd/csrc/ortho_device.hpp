// What the kernels of the orthogonalised update share.
#pragma once
#include <hip/hip_runtime.h>

#include "device_util.hpp"
#include "ortho_kernels.hpp"

namespace canvas {
namespace ortho {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr double kEps = 1e-7;

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

}  // namespace ortho
}  // namespace canvas
