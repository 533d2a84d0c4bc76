// Residual norm, backward on rows of tokens (planes of one pixel): the passes of norm_maps_bwd_kernels.hip with one pixel per row,
// TPR threads per row and KV times 16 bytes each.  Workgroups walk over rows and keep the sums of their channels.
// Bound by memory.  With the sums over the partials, over three sets of rows in turn: 4096 x 2048 in fp32 52 us (5.2 TB/s), 8192 x 512 in bf16
// 20 us (3.3 TB/s), 2048 x 4096 in bf16 40 us (3.4 TB/s; over one set 36, by 256 threads of 32 bytes 39), 4096 x 8192 in bf16 119 us
// (4.5 TB/s), 512 x 16384 in bf16 74 us (1.8 TB/s), whose values are read up to three times.
#include <atomic>

#include "launch.hpp"
#include "norm_device.hpp"

namespace canvas {
namespace norm {
namespace {

// Rows that 1024 threads of 16 bytes do not hold leave no registers for the values, the weights and the sums of their channels: values and
// weights are read again for each pass, the sums are in LDS.
template <class T, int TPR, int KV, int PARTS, int GATE>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_rows_bwd(Shape s, Bwd a) {
    constexpr int V = 16 / sizeof(T), kRows = TPR < 256 ? 256 / TPR : 1;
    constexpr bool kLong = TPR == 1024 && KV > 1;
    constexpr int KS = kLong ? 1 : KV, KX = kLong ? 1 : KV;
    extern __shared__ float lds[];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    constexpr bool kIsPost = PARTS & kPost, kIsPre = PARTS & kPre;
    const float inv = 1.f / s.C;
    float sw[KS][V], w1[KS][V], kp[KS][V], kx[KS][V];
    float* sums = lds + 16;  // kLong: [2][KV * V][TPR]
    auto weights = [&](int k, int c) {
        if (kIsPost) {
            float w[V];
            load_weights<V>(w, a.w_post, c, s.C);
            load_weights<V>(sw[k], a.scale, c, s.C);
#pragma unroll
            for (int e = 0; e < V; e++) sw[k][e] *= w[e];
        }
        if (kIsPre) load_weights<V>(w1[k], a.w_pre, c, s.C);
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
            if (kIsPre) {
                load_row<T, V>(x[k], a.x, row, c, s.C);
                load_row<T, V>(du[k], a.du, row, c, s.C);
            }
            if (kIsPost) load_row<T, V>(z[k], a.z, row, c, s.C);
            if (GATE) load_row<T, V>(g[k], a.g, row, c, s.C);
            if (a.dx_out) load_row<T, V>(dy[k], a.dx_out, row, c, s.C);
        };
        if (!kLong) {
#pragma unroll
            for (int k = 0; k < KV; k++) load(k % KX, (k * TPR + t) * V);
        }
        const float r2 = kIsPost ? a.r2[n] : 0.f, r1 = kIsPre ? a.r1[n] : 0.f;
        float t1 = 0.f, t2 = 0.f;
        auto renew = [&](int k) {
            if (kLong) load(0, (k * TPR + t) * V);
            if (kIsPre) {
                x[k % KX].renew();
                du[k % KX].renew();
            }
            if (kIsPost) z[k % KX].renew();
            if (GATE) g[k % KX].renew();
            if (kLong) weights(0, (k * TPR + t) * V);
        };
        // m, kept from the first pass for the second
        float m[KX][V], d[KX][V];
        auto branch = [&](int k) {
#pragma unroll
            for (int e = 0; e < V; e++) m[k % KX][e] = kIsPost ? act<T, GATE>(GATE ? g[k % KX].at(e) : 0.f) * (z[k % KX].at(e) * r2) : 0.f;
        };
        auto joined = [&](int k, int e) { return kIsPost ? x[k % KX].at(e) + sw[k % KS][e] * m[k % KX][e] : x[k % KX].at(e); };  // x'
        auto whole = [&](int k, int e, float y) {                                                                               // D
            const float dy_e = a.dx_out ? dy[k % KX].at(e) : 0.f;
            return kIsPre ? dy_e - y * t1 + du[k % KX].at(e) * w1[k % KS][e] * r1 : dy_e;
        };
        if (kIsPre) {
#pragma unroll(kLong ? 1 : KV)
            for (int k = 0; k < KV; k++) {
                if (kLong) renew(k);
                branch(k);
#pragma unroll
                for (int e = 0; e < V; e++) t1 += du[k % KX].at(e) * w1[k % KS][e] * joined(k, e);
            }
            t1 = over_row<TPR>(t1, lds) * inv * r1 * r1 * r1;
        }
#pragma unroll(kLong ? 1 : KV)
        for (int k = 0; k < KV; k++) {
            renew(k);
            if (kLong || !kIsPre) branch(k);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float y = kIsPre ? joined(k, e) : 0.f;
                d[k % KX][e] = whole(k, e, y);
                if (kIsPost) {
                    const float p = d[k % KX][e] * m[k % KX][e];
                    t2 += p * sw[k % KS][e];
                    if (kLong)
                        sums[(k * V + e) * TPR + t] += p;
                    else
                        kp[k % KS][e] += p;
                }
                if (kIsPre) {
                    const float q = du[k % KX].at(e) * y * r1;
                    if (kLong)
                        sums[((KV + k) * V + e) * TPR + t] += q;
                    else
                        kx[k % KS][e] += q;
                }
            }
            if (kIsPre) store_row<T, V>(a.dx, row, (k * TPR + t) * V, s.C, d[k % KX]);
        }
        if (kIsPost) {
            t2 = over_row<TPR>(t2, lds) * inv * r2 * r2;
#pragma unroll(kLong ? 1 : KV)
            for (int k = 0; k < KV; k++) {
                renew(k);
                if (kLong) branch(k);
                float dz[V], dg[V];
#pragma unroll
                for (int e = 0; e < V; e++) {
                    float av;
                    const float slope = act_slope<T, GATE>(GATE ? g[k % KX].at(e) : 0.f, av);
                    const float D = kLong ? whole(k, e, kIsPre ? joined(k, e) : 0.f) : d[k % KX][e], E = D * (sw[k % KS][e] * r2), zv = z[k % KX].at(e);
                    dz[e] = E * av - zv * t2;
                    dg[e] = E * zv * slope;
                }
                store_row<T, V>(a.dz, row, (k * TPR + t) * V, s.C, dz);
                if (GATE) store_row<T, V>(a.dg, row, (k * TPR + t) * V, s.C, dg);
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

template <class T, int TPR, int KV, int PARTS, int GATE>
void rows(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, kRows = kBlock / TPR;
    constexpr int lds = kRows > 1 ? 256 * 64 / (int)sizeof(T) : 64 + (TPR == 1024 && KV > 1 ? TPR * KV * 128 / (int)sizeof(T) : 0);
    if (lds > 65536) {
        static std::atomic<uint64_t> asked{0};
        allow_lds(asked, reinterpret_cast<const void*>(&k_rows_bwd<T, TPR, KV, PARTS, GATE>), lds);
    }
    CANVAS_LAUNCH((k_rows_bwd<T, TPR, KV, PARTS, GATE>), dim3(p.partials), dim3(kBlock), lds, stream, s, a);
}
template <class T, int PARTS, int GATE>
void run(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    switch (p.tpr * 8 + p.kv) {
    case 16 * 8 + 1: return rows<T, 16, 1, PARTS, GATE>(s, p, a, stream);
    case 64 * 8 + 1: return rows<T, 64, 1, PARTS, GATE>(s, p, a, stream);
    case 64 * 8 + 2: return rows<T, 64, 2, PARTS, GATE>(s, p, a, stream);
    case 256 * 8 + 1: return rows<T, 256, 1, PARTS, GATE>(s, p, a, stream);
    case 512 * 8 + 1: return rows<T, 512, 1, PARTS, GATE>(s, p, a, stream);
    case 1024 * 8 + 1: return rows<T, 1024, 1, PARTS, GATE>(s, p, a, stream);
    default: return rows<T, 1024, 16 / V, PARTS, GATE>(s, p, a, stream);
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

void rows_backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream) {
    if (s.bf16)
        run_parts<uint16_t>(s, p, a, stream);
    else
        run_parts<float>(s, p, a, stream);
}

}  // namespace norm
}  // namespace canvas
