// Residual norm, forward and backward: a workgroup takes 64 pixels, its four waves the channels in turn.  Every pass over the
// channels reads memory again.
#include "norm_kernels.hpp"

#include "device_util.hpp"
#include "launch.hpp"

namespace canvas {
namespace norm {
namespace {

constexpr int kPix = 64, kSlots = 4;

template <class T>
__device__ __forceinline__ float ld(const void* p, int64_t i);
template <>
__device__ __forceinline__ float ld<float>(const void* p, int64_t i) {
    return static_cast<const float*>(p)[i];
}
template <>
__device__ __forceinline__ float ld<uint16_t>(const void* p, int64_t i) {
    return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}
__device__ __forceinline__ void st(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st(uint16_t* p, int64_t i, float v) { p[i] = f32_to_bf16(v); }

__device__ __forceinline__ void gate_of(int kind, float g, float& a, float& da) {
    if (kind == 0) {
        a = 1.f;
        da = 0.f;
        return;
    }
    const float s = 1.f / (1.f + expf(-g));
    a = kind == 1 ? s : g * s;
    da = kind == 1 ? s * (1.f - s) : s * (1.f + g * (1.f - s));
}

// Sum over the slots of one pixel.
__device__ __forceinline__ float over_slots(float v, float (*buf)[kPix]) {
    __syncthreads();
    buf[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    float s = 0.f;
    for (int k = 0; k < kSlots; k++) s += buf[k][threadIdx.x];
    return s;
}

template <class T>
__global__ __launch_bounds__(kPix* kSlots) void k_fwd(Shape s, Fwd a) {
    __shared__ float buf[kSlots][kPix];
    const int64_t total = s.N * s.P, q = (int64_t)blockIdx.x * kPix + threadIdx.x;
    const bool in = q < total;
    const int64_t n = in ? q / s.P : 0, base = n * s.C * s.P + (in ? q - n * s.P : 0);
    float r2 = 0.f, r1 = 0.f;
    if (s.post) {
        float t = 0.f;
        if (in)
            for (int c = threadIdx.y; c < s.C; c += kSlots) {
                const float z = ld<T>(a.z, base + c * s.P);
                t += z * z;
            }
        r2 = 1.f / sqrtf(over_slots(t, buf) / s.C + s.eps);
    }
    if (in && s.post && a.r2 && threadIdx.y == 0) a.r2[q] = r2;
    auto joined = [&](int c) {
        const int64_t i = base + c * s.P;
        float y = ld<T>(a.x, i);
        if (s.post) {
            float g, dg;
            gate_of(s.gate, s.gate ? ld<T>(a.g, i) : 0.f, g, dg);
            y += a.scale[c] * g * (ld<T>(a.z, i) * r2 * a.w_post[c]);
        }
        return y;
    };
    float t = 0.f;
    if (in)
        for (int c = threadIdx.y; c < s.C; c += kSlots) {
            const float y = joined(c);
            t += y * y;
            if (s.post) st((T*)a.x_out, base + c * s.P, y);
        }
    if (!s.pre) return;
    r1 = 1.f / sqrtf(over_slots(t, buf) / s.C + s.eps);
    if (!in) return;
    if (a.r1 && threadIdx.y == 0) a.r1[q] = r1;
    for (int c = threadIdx.y; c < s.C; c += kSlots) st((T*)a.u, base + c * s.P, joined(c) * r1 * a.w_pre[c]);
}

template <class T>
__global__ __launch_bounds__(kPix* kSlots) void k_bwd(Shape s, Bwd a) {
    __shared__ float buf[kSlots][kPix];
    const int64_t total = s.N * s.P, q = (int64_t)blockIdx.x * kPix + threadIdx.x;
    const bool in = q < total;
    const int64_t n = in ? q / s.P : 0, base = n * s.C * s.P + (in ? q - n * s.P : 0);
    const float r2 = in && s.post ? a.r2[q] : 0.f, r1 = in && s.pre ? a.r1[q] : 0.f;
    auto unit = [&](int c) {  // xh
        const int64_t i = base + c * s.P;
        float y = ld<T>(a.x, i);
        if (s.post) {
            float g, dg;
            gate_of(s.gate, s.gate ? ld<T>(a.g, i) : 0.f, g, dg);
            y += a.scale[c] * g * (ld<T>(a.z, i) * r2 * a.w_post[c]);
        }
        return y * r1;
    };
    float t1 = 0.f;
    if (s.pre) {
        float t = 0.f;
        if (in)
            for (int c = threadIdx.y; c < s.C; c += kSlots) t += ld<T>(a.du, base + c * s.P) * a.w_pre[c] * unit(c);
        t1 = over_slots(t, buf) / s.C;
    }
    auto whole = [&](int c, float& du_xh) {  // D
        const int64_t i = base + c * s.P;
        float d = a.dx_out ? ld<T>(a.dx_out, i) : 0.f;
        du_xh = 0.f;
        if (s.pre) {
            const float du = ld<T>(a.du, i), xh = unit(c);
            du_xh = du * xh;
            d += r1 * (du * a.w_pre[c] - xh * t1);
        }
        return d;
    };
    float t2 = 0.f;
    if (s.post) {
        float t = 0.f;
        if (in)
            for (int c = threadIdx.y; c < s.C; c += kSlots) {
                const int64_t i = base + c * s.P;
                float g, dg, un;
                gate_of(s.gate, s.gate ? ld<T>(a.g, i) : 0.f, g, dg);
                t += whole(c, un) * g * (a.scale[c] * a.w_post[c]) * (ld<T>(a.z, i) * r2);
            }
        t2 = over_slots(t, buf) / s.C;
    }
    for (int c = threadIdx.y; c < s.C; c += kSlots) {
        const int64_t i = base + c * s.P;
        float kp = 0.f, kx = 0.f;
        if (in) {
            const float d = whole(c, kx);
            if (s.pre) st((T*)a.dx, i, d);
            if (s.post) {
                float g, dg;
                gate_of(s.gate, s.gate ? ld<T>(a.g, i) : 0.f, g, dg);
                const float zh = ld<T>(a.z, i) * r2, sw = a.scale[c] * a.w_post[c];
                kp = d * g * zh;
                st((T*)a.dz, i, r2 * (d * g * sw - zh * t2));
                if (s.gate) st((T*)a.dg, i, d * dg * sw * zh);
            }
        }
        for (int o = 32; o; o >>= 1) {
            kp += __shfl_xor(kp, o);
            kx += __shfl_xor(kx, o);
        }
        if (threadIdx.x == 0) {
            a.partial[((int64_t)blockIdx.x * 2) * s.C + c] = kp;
            a.partial[((int64_t)blockIdx.x * 2 + 1) * s.C + c] = kx;
        }
    }
}

__global__ __launch_bounds__(256) void k_sums(Shape s, Bwd a, int partials) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= s.C) return;
    float kp = 0.f, kx = 0.f;
    for (int b = 0; b < partials; b++) {
        kp += a.partial[((int64_t)b * 2) * s.C + c];
        kx += a.partial[((int64_t)b * 2 + 1) * s.C + c];
    }
    if (s.post) {
        a.dw_post[c] = a.scale[c] * kp;
        a.dscale[c] = a.w_post[c] * kp;
    }
    if (s.pre) a.dw_pre[c] = kx;
}

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    p.partials = (int)((s.N * s.P + kPix - 1) / kPix);
    return p;
}

void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    const dim3 block(kPix, kSlots);
    if (s.bf16)
        CANVAS_LAUNCH(k_fwd<uint16_t>, dim3(p.partials), block, 0, stream, s, a);
    else
        CANVAS_LAUNCH(k_fwd<float>, dim3(p.partials), block, 0, stream, s, a);
}

void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    const dim3 block(kPix, kSlots);
    if (s.bf16)
        CANVAS_LAUNCH(k_bwd<uint16_t>, dim3(p.partials), block, 0, stream, s, a);
    else
        CANVAS_LAUNCH(k_bwd<float>, dim3(p.partials), block, 0, stream, s, a);
    CANVAS_LAUNCH(k_sums, dim3((s.C + 255) / 256), dim3(256), 0, stream, s, a, p.partials);
}

}  // namespace norm
}  // namespace canvas
