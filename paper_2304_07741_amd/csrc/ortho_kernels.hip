// Newton-Schulz products in fp32, one thread per element of a result.
#include "ortho_kernels.hpp"

#include "device_util.hpp"
#include "launch.hpp"

namespace canvas {
namespace ortho {
namespace {

constexpr int kThreads = 256, kTile = 16;
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr double kEps = 1e-7;

__device__ __forceinline__ float direction(const Shape& s, const Args& a, int64_t i, float m_new) {
    if (!a.momentum) return a.grad[i];
    return s.nesterov ? (float)(a.grad[i] + a.mu * m_new) : m_new;  // (mu in 64 bits: gradient and momentum may cancel)
}

__global__ __launch_bounds__(kThreads) void k_mix(Shape s, Args a, double* sums) {
    __shared__ double buf[kThreads];
    const int64_t len = s.R * s.K, base = blockIdx.y * len;
    double t = 0;
    for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < len; k += (int64_t)gridDim.x * kThreads) {
        const int64_t i = base + k;
        float m = 0.f;
        if (a.momentum) {
            m = (float)(a.mu * a.momentum[i] + a.grad[i]);
            a.momentum_out[i] = m;
        }
        const double v = direction(s, a, i, m);
        t += v * v;
    }
    buf[threadIdx.x] = t;
    __syncthreads();
    for (int o = kThreads / 2; o; o >>= 1) {
        if ((int)threadIdx.x < o) buf[threadIdx.x] += buf[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) sums[blockIdx.y * gridDim.x + blockIdx.x] = buf[0];
}

__global__ __launch_bounds__(kThreads) void k_start(Shape s, Args a, const double* sums, int parts, float* x) {
    double t = 0;
    for (int k = 0; k < parts; k++) t += sums[blockIdx.y * parts + k];
    const double inv = 1.0 / (sqrt(t) + kEps);
    const int64_t len = s.R * s.K, k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (k >= len) return;
    const int64_t i = blockIdx.y * len + k;
    const int64_t row = k / s.K, col = k - row * s.K;
    x[blockIdx.y * len + (s.tall ? col * s.n + row : k)] = (float)(direction(s, a, i, a.momentum ? a.momentum_out[i] : 0.f) * inv);
}

// c[i][j] = p sum_k a[i][k] b(k, j) + q d[i][j],  b(k, j) = b[j][k] with NT, else b[k][j]
template <bool NT>
__global__ __launch_bounds__(kTile* kTile) void k_product(const float* a, const float* b, const float* d, float* c, int64_t rows, int64_t cols, int64_t depth,
                                                          float p, float q, int64_t step_a, int64_t step_b, int64_t step_c) {
    __shared__ float ta[kTile][kTile + 1], tb[kTile][kTile + 1];
    a += blockIdx.z * step_a;
    b += blockIdx.z * step_b;
    c += blockIdx.z * step_c;
    const int64_t i0 = (int64_t)blockIdx.y * kTile, j0 = (int64_t)blockIdx.x * kTile;
    const int ty = threadIdx.x / kTile, tx = threadIdx.x % kTile;
    float t = 0.f;
    for (int64_t k0 = 0; k0 < depth; k0 += kTile) {
        ta[ty][tx] = i0 + ty < rows && k0 + tx < depth ? a[(i0 + ty) * depth + k0 + tx] : 0.f;
        if (NT)
            tb[tx][ty] = j0 + ty < cols && k0 + tx < depth ? b[(j0 + ty) * depth + k0 + tx] : 0.f;
        else
            tb[ty][tx] = k0 + ty < depth && j0 + tx < cols ? b[(k0 + ty) * cols + j0 + tx] : 0.f;
        __syncthreads();
        for (int k = 0; k < kTile; k++) t += ta[ty][k] * tb[k][tx];
        __syncthreads();
    }
    const int64_t i = i0 + ty, j = j0 + tx;
    if (i < rows && j < cols) c[i * cols + j] = p * t + (q != 0.f ? q * d[blockIdx.z * step_c + i * cols + j] : 0.f);
}

__global__ __launch_bounds__(kThreads) void k_finish(Shape s, Args a, const float* x) {
    const int64_t len = s.R * s.K, k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (k >= len) return;
    const int64_t i = blockIdx.y * len + k;
    const int64_t row = k / s.K, col = k - row * s.K;
    const float o = x[blockIdx.y * len + (s.tall ? col * s.n + row : k)];
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

uint64_t up256(uint64_t v) { return (v + 255) & ~(uint64_t)255; }
unsigned blocks(int64_t n, int64_t per) { return (unsigned)((n + per - 1) / per); }

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    p.parts = (int)((s.R * s.K + 16 * kThreads - 1) / (16 * kThreads));
    if (p.parts > 256) p.parts = 256;
    p.launches = 3 + 3 * s.steps;
    p.workspace_bytes = up256(8ull * s.G * p.parts) + 2 * up256(4ull * s.G * s.m * s.n) + 2 * up256(4ull * s.G * s.m * s.m);
    return p;
}

void step(const Shape& s, const Plan& p, const Args& a, hipStream_t stream) {
    char* at = a.ws;
    auto take = [&](uint64_t bytes) {
        char* r = at;
        at += up256(bytes);
        return r;
    };
    double* sums = (double*)take(8ull * s.G * p.parts);
    float* x = (float*)take(4ull * s.G * s.m * s.n);
    float* x2 = (float*)take(4ull * s.G * s.m * s.n);
    float* q = (float*)take(4ull * s.G * s.m * s.m);
    float* b = (float*)take(4ull * s.G * s.m * s.m);
    const unsigned G = (unsigned)s.G, all = blocks(s.R * s.K, kThreads);
    CANVAS_LAUNCH(k_mix, dim3(p.parts, G), dim3(kThreads), 0, stream, s, a, sums);
    CANVAS_LAUNCH(k_start, dim3(all, G), dim3(kThreads), 0, stream, s, a, sums, p.parts, x);
    const dim3 tt(kTile * kTile), gq(blocks(s.m, kTile), blocks(s.m, kTile), G), gx(blocks(s.n, kTile), blocks(s.m, kTile), G);
    for (int k = 0; k < s.steps; k++) {
        CANVAS_LAUNCH(k_product<true>, gq, tt, 0, stream, x, x, (const float*)nullptr, q, s.m, s.m, s.n, 1.f, 0.f, s.m * s.n, s.m * s.n, s.m * s.m);
        CANVAS_LAUNCH(k_product<true>, gq, tt, 0, stream, q, q, q, b, s.m, s.m, s.m, kC, kB, s.m * s.m, s.m * s.m, s.m * s.m);
        CANVAS_LAUNCH(k_product<false>, gx, tt, 0, stream, b, x, x, x2, s.m, s.n, s.m, 1.f, kA, s.m * s.m, s.m * s.n, s.m * s.n);
        float* t = x;
        x = x2;
        x2 = t;
    }
    CANVAS_LAUNCH(k_finish, dim3(all, G), dim3(kThreads), 0, stream, s, a, x);
}

}  // namespace ortho
}  // namespace canvas
