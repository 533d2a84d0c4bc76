// Log probabilities of given tokens: a workgroup of 256 threads per row, which reads the row once for its largest logit, once
// for the sums and once for every alternative.
#include "logprob_kernels.hpp"

#include "device_util.hpp"
#include "launch.hpp"

namespace canvas {
namespace logprob {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float ld(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float ld(const uint16_t* p, int64_t i) { return bf16_to_f32(p[i]); }
__device__ __forceinline__ void st(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st(uint16_t* p, int64_t i, float v) { p[i] = f32_to_bf16(v); }

// Order of the alternatives as whole numbers: NaN first, then larger logits (zeros of both signs are equal), then lower
// indices.  0 is no alternative.
constexpr uint32_t kNan = 0xffc00000u;
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) {
    const uint32_t u = __float_as_uint(v + 0.f);
    const uint32_t o = v != v ? kNan : (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return (uint64_t)o << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return o == kNan ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

template <class V, class F>
__device__ V over_row(V v, V* buf, F join) {
    __syncthreads();
    buf[threadIdx.x] = v;
    __syncthreads();
    for (int o = kThreads / 2; o; o >>= 1) {
        if ((int)threadIdx.x < o) buf[threadIdx.x] = join(buf[threadIdx.x], buf[threadIdx.x + o]);
        __syncthreads();
    }
    return buf[0];
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_fwd(Shape s, Fwd a) {
    __shared__ uint64_t ibuf[kThreads];
    __shared__ float fbuf[kThreads];
    const int64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.logits) + row * a.pitch;
    const uint8_t* mask = a.mask ? a.mask + row * a.mask_pitch : nullptr;
    const float inf = __builtin_inff();
    auto at = [&](int64_t i) { return mask && !mask[i] ? -inf : ld(z, i); };
    float m = -inf;
    for (int64_t i = threadIdx.x; i < s.classes; i += kThreads) m = fmaxf(m, at(i));  // (fmaxf drops NaN: the sums below have it)
    m = over_row(m, fbuf, [](float x, float y) { return fmaxf(x, y); });
    const float most = m == -inf ? 0.f : m;
    float sum = 0.f, along = 0.f;
    for (int64_t i = threadIdx.x; i < s.classes; i += kThreads) {
        const float v = at(i);
        const float d = (v - most) * a.it, e = v == -inf ? 0.f : expf(d);
        sum += e;
        if (e != 0.f) along += e * d;
    }
    auto add = [](float x, float y) { return x + y; };
    sum = over_row(sum, fbuf, add);
    along = over_row(along, fbuf, add);
    const bool empty = sum == 0.f;
    const float log_sum = empty ? -inf : logf(sum), entropy = empty ? 0.f : log_sum - along / sum;
    if (threadIdx.x == 0) {
        if (a.ws) reinterpret_cast<Row*>(a.ws)[row] = Row{most, log_sum, entropy, 0.f};
        if (a.entropy) a.entropy[row] = entropy;
        if (a.tokens) {
            const int64_t t = a.tokens[row];
            float lp = 0.f;
            if (t >= 0 && t < s.classes) {
                const float v = at(t);
                lp = empty || (v == -inf && !(sum != sum)) ? -inf : (v - most) * a.it - log_sum;
            }
            a.logprob[row] = lp;
        }
    }
    uint64_t last = ~(uint64_t)0;
    for (int k = 0; k < s.top; k++) {
        uint64_t best = 0;
        for (int64_t i = threadIdx.x; i < s.classes; i += kThreads) {
            const float v = at(i);
            if (v == -inf) continue;
            const uint64_t key = key_of(v, (uint32_t)i);
            if (key < last && key > best) best = key;
        }
        best = over_row(best, ibuf, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
        if (threadIdx.x == 0) {
            a.top_index[row * s.top + k] = best ? (int32_t)~(uint32_t)best : -1;
            a.top_logprob[row * s.top + k] = best ? (value_of(best) - most) * a.it - log_sum : -inf;
        }
        last = best;
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_bwd(Shape s, Bwd a) {
    const int64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.logits) + row * a.pitch;
    T* dz = static_cast<T*>(a.dlogits) + row * a.dpitch;
    const uint8_t* mask = a.mask ? a.mask + row * a.mask_pitch : nullptr;
    const Row r = reinterpret_cast<const Row*>(a.ws)[row];
    const float inf = __builtin_inff();
    const int64_t t = a.tokens ? a.tokens[row] : -1;
    const bool given = t >= 0 && t < s.classes, empty = r.log_sum == -inf;
    const float g = given && a.dlogprob ? a.dlogprob[row] : 0.f, h = a.dentropy ? a.dentropy[row] : 0.f;
    for (int64_t i = threadIdx.x; i < s.classes; i += kThreads) {
        const bool hidden = empty || (mask && !mask[i]);
        const float v = hidden ? -inf : ld(z, i);
        const float lp = (v - r.most) * a.it - r.log_sum, p = v == -inf && r.log_sum == r.log_sum ? 0.f : expf(lp);
        float d = -g * p - (p == 0.f ? 0.f : h * p * (lp + r.entropy));
        if (i == t) d += g;
        st(dz, i, hidden ? 0.f : d * a.it);
    }
}

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    p.workspace_bytes = (uint64_t)s.rows * sizeof(Row);
    return p;
}

void forward(const Shape& s, const Plan&, const Fwd& a, hipStream_t stream) {
    if (s.bf16)
        CANVAS_LAUNCH(k_fwd<uint16_t>, dim3((unsigned)s.rows), dim3(kThreads), 0, stream, s, a);
    else
        CANVAS_LAUNCH(k_fwd<float>, dim3((unsigned)s.rows), dim3(kThreads), 0, stream, s, a);
}

void backward(const Shape& s, const Plan&, const Bwd& a, hipStream_t stream) {
    if (s.bf16)
        CANVAS_LAUNCH(k_bwd<uint16_t>, dim3((unsigned)s.rows), dim3(kThreads), 0, stream, s, a);
    else
        CANVAS_LAUNCH(k_bwd<float>, dim3((unsigned)s.rows), dim3(kThreads), 0, stream, s, a);
}

}  // namespace logprob
}  // namespace canvas
