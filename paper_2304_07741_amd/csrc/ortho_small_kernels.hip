// Orthogonalised updates of small matrices: one workgroup per matrix keeps X, A and B in LDS in fp32 through all steps, in one launch.
// The products run on the fp32 matrix instructions (16 x 16 x 4): at these sizes launches and barriers cost more than products.
//
// Rows of X are padded to a multiple of 16 floats plus 4 and those of A and B likewise, so that both the reads of 16 rows (16 bytes
// each, operands that are summed along the rows) and those of 4 x 16 elements of a column block fall on different banks.
//
// Bound by latency: three dependent products per step, each of reads from LDS, a few matrix instructions and a barrier.  Eight of
// 8 x 72, five steps: 13 us, of which the launch is 4 (17 launches of the kernels for large matrices: 68 us).
#include "ortho_small_kernels.hpp"

#include <atomic>

#include "device_util.hpp"
#include "launch.hpp"
#include "ortho_device.hpp"

namespace canvas {
namespace ortho {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;

typedef float f32x4 __attribute__((ext_vector_type(4)));

// C += P[rows i0..][k] Q[rows j0..][k] over 16 k's from k0 on: the element t of each lane's 16 bytes is the k of instruction t.
__device__ __forceinline__ f32x4 rows_by_rows(const float* p, const float* q, f32x4 acc) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(q);
#pragma unroll
    for (int t = 0; t < 4; t++) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[t], b[t], acc, 0, 0, 0);
    return acc;
}

__global__ __launch_bounds__(kThreads) void k_small(Shape s, Args a) {
    extern __shared__ __align__(16) float lds[];
    __shared__ double s_sum[kWaves];
    const SmallPlan p = small_plan(s);
    const int mp = p.mp, np = p.np, ld = p.ld, lq = mp + 4, T = mp / 16;
    float *x = lds, *q = x + mp * ld, *b = q + mp * lq, *parts = b + mp * lq;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int len = (int)(s.R * s.K);
    const int64_t base = (int64_t)blockIdx.x * len;

    for (int i = tid; i < mp * ld; i += kThreads) x[i] = 0.f;
    __syncthreads();
    double t = 0;
    for (int k = tid; k < len; k += kThreads) {
        const int64_t i = base + k;
        float m = 0.f;
        if (a.momentum) {
            m = (float)(a.mu * a.momentum[i] + a.grad[i]);
            a.momentum_out[i] = m;
        }
        const float v = direction(s, a, i, m);
        t += (double)v * v;
        const int row = k / (int)s.K, col = k - row * (int)s.K;
        x[s.tall ? col * ld + row : row * ld + col] = v;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    if (lane == 0) s_sum[wave] = t;
    __syncthreads();
    t = 0;
#pragma unroll
    for (int w = 0; w < kWaves; w++) t += s_sum[w];
    const double inv = inverse_norm(t);
    for (int i = tid; i < mp * ld; i += kThreads) x[i] = (float)(x[i] * inv);
    __syncthreads();

    // A and B by tiles; where there are fewer tiles than waves the sum over k is cut into slices, added in their order
    const int tiles = T * T, slices = tiles >= kWaves ? 1 : kWaves / tiles, chunks = np / 16;
    for (int step = 0; step < s.steps; step++) {
        for (int u = wave; u < tiles * slices; u += kWaves) {
            const int tile = u / slices, sl = u - tile * slices, ti = tile / T, tj = tile - ti * T;
            f32x4 acc = {};
            const float *pi = x + (ti * 16 + lr) * ld + lg * 4, *pj = x + (tj * 16 + lr) * ld + lg * 4;
            for (int c = chunks * sl / slices; c < chunks * (sl + 1) / slices; c++) acc = rows_by_rows(pi + c * 16, pj + c * 16, acc);
#pragma unroll
            for (int e = 0; e < 4; e++) parts[u * 256 + (lg * 4 + e) * 16 + lr] = acc[e];
        }
        __syncthreads();
        for (int i = tid; i < tiles * 256; i += kThreads) {
            const int tile = i >> 8, at = i & 255, ti = tile / T, tj = tile - ti * T;
            float v = 0.f;
            for (int sl = 0; sl < slices; sl++) v += parts[(tile * slices + sl) * 256 + at];
            q[(ti * 16 + (at >> 4)) * lq + tj * 16 + (at & 15)] = v;
        }
        __syncthreads();
        for (int tile = wave; tile < tiles; tile += kWaves) {
            const int ti = tile / T, tj = tile - ti * T;
            f32x4 acc = {};
            const float *pi = q + (ti * 16 + lr) * lq + lg * 4, *pj = q + (tj * 16 + lr) * lq + lg * 4;
            for (int c = 0; c < T; c++) acc = rows_by_rows(pi + c * 16, pj + c * 16, acc);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int i = ti * 16 + lg * 4 + e, j = tj * 16 + lr;
                b[i * lq + j] = kC * acc[e] + kB * q[i * lq + j];
            }
        }
        __syncthreads();
        // X = a X + (b A + c A A) X by blocks of 16 columns, each read and written by one wave.  (a X joins the sum at its end: as its first
        // term it would have every later one rounded to its own size, which doubles the error where singular values spread.)
        for (int jt = wave; jt < chunks; jt += kWaves) {
            float* col = x + lg * 4 * ld + jt * 16 + lr;
            f32x4 acc[4] = {}, old[4];
#pragma unroll
            for (int c = 0; c < 4; c++) {
                if (c >= T) break;
                f32x4& v = old[c];
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = col[(c * 16 + e) * ld];
#pragma unroll
                for (int ti = 0; ti < 4; ti++)
                    if (ti < T) {
                        const f32x4 w = *reinterpret_cast<const f32x4*>(b + (ti * 16 + lr) * lq + c * 16 + lg * 4);
#pragma unroll
                        for (int e = 0; e < 4; e++) acc[ti] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], v[e], acc[ti], 0, 0, 0);
                    }
            }
#pragma unroll
            for (int ti = 0; ti < 4; ti++)
                if (ti < T)
#pragma unroll
                    for (int e = 0; e < 4; e++) col[(ti * 16 + e) * ld] = fmaf(kA, old[ti][e], acc[ti][e]);
        }
        __syncthreads();
    }
    for (int k = tid; k < len; k += kThreads) {
        const int row = k / (int)s.K, col = k - row * (int)s.K;
        finish_one(s, a, base + k, x[s.tall ? col * ld + row : row * ld + col]);
    }
}

}  // namespace

void step_small(const Shape& s, const Args& a, hipStream_t stream) {
    const int lds = small_plan(s).lds;
    if (lds > 65536) {
        static std::atomic<uint64_t> asked{0};
        allow_lds(asked, reinterpret_cast<const void*>(&k_small), kMostSmallLds);
    }
    CANVAS_LAUNCH(k_small, dim3((unsigned)s.G), dim3(kThreads), lds, stream, s, a);
}

}  // namespace ortho
}  // namespace canvas
