// The norm over many tensors and their scaling.
//
// Two passes over memory: squares, added up in 64 bits by each thread over its elements, then by each workgroup, then by every workgroup of the second
// pass for itself, always in the same order; and the scaling.  The second pass goes through the tensors backwards: what the first one read last is still in the
// last-level cache.  Bound by memory: 2^28 elements of bf16, squares 91 us (5.9 TB/s), scaling 189 (5.7); 25.5 M elements of both types to fp32 19 and 33.  Chunks of 16384 elements, 64 a
// thread: all of a chunk's loads are in flight at once.
#include "clip_kernels.hpp"

#include <algorithm>

#include "device_util.hpp"
#include "launch.hpp"
#include "tile_util.hpp"

namespace canvas {
namespace clip {
namespace {

using tile::u32x4;
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kThreads = 256, kMostParts = 2048;
constexpr int64_t kAloneElements = 1 << 14;  // up to which one workgroup does all of it

struct Item {
    const void* in;
    void* out;
    int64_t count;
    uint32_t first;  // chunk
    uint16_t bf16, out_bf16;
};
struct Items {
    Item item[kBatch];
    int n;
    uint32_t chunks;
};

// The tensor that a chunk belongs to.
__device__ __forceinline__ int item_of(const Items& a, uint32_t chunk) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.item[mid].first <= chunk)
            lo = mid;
        else
            hi = mid - 1;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
__device__ __forceinline__ bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (e & 1) ? tile::hi_f32(w[e >> 1]) : tile::lo_f32(w[e >> 1]);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = a[e], v[4 + e] = b[e];
}
__device__ __forceinline__ float load1(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
// PAST: past the last-level cache.
template <bool PAST, class V>
__device__ __forceinline__ void put(V* p, const V& v) {
    if (PAST)
        __builtin_nontemporal_store(v, p);
    else
        *p = v;
}
template <bool PAST>
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
    put<PAST>(reinterpret_cast<u32x4*>(p), u32x4{tile::pack_bf16(v[0], v[1]), tile::pack_bf16(v[2], v[3]), tile::pack_bf16(v[4], v[5]), tile::pack_bf16(v[6], v[7])});
}
template <bool PAST>
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    put<PAST>(reinterpret_cast<f32x4*>(p), f32x4{v[0], v[1], v[2], v[3]});
    put<PAST>(reinterpret_cast<f32x4*>(p) + 1, f32x4{v[4], v[5], v[6], v[7]});
}
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

constexpr int kTurns = kChunk / (8 * kThreads);
template <class T>
__device__ __forceinline__ double squares(const T* p, int n) {
    double t = 0;
    if (n == kChunk && aligned(p)) {
        float v[kTurns][8];
#pragma unroll
        for (int k = 0; k < kTurns; k++) load8(p + (k * kThreads + threadIdx.x) * 8, v[k]);
#pragma unroll
        for (int k = 0; k < kTurns; k++)
#pragma unroll
            for (int e = 0; e < 8; e++) t = fma((double)v[k][e], (double)v[k][e], t);
        return t;
    }
    int done = 0;
    if (aligned(p)) {
        done = n & ~7;
        for (int i = threadIdx.x * 8; i < done; i += 8 * kThreads) {
            float v[8];
            load8(p + i, v);
#pragma unroll
            for (int e = 0; e < 8; e++) t = fma((double)v[e], (double)v[e], t);
        }
    }
    for (int i = done + threadIdx.x; i < n; i += kThreads) {
        const double v = load1(p + i);
        t = fma(v, v, t);
    }
    return t;
}

// Over the workgroup, in a fixed order; the sum is thread 0's.
__device__ __forceinline__ double over_threads(double t) {
    __shared__ double buf[kThreads];
    buf[threadIdx.x] = t;
    __syncthreads();
    for (int o = kThreads / 2; o; o >>= 1) {
        if ((int)threadIdx.x < o) buf[threadIdx.x] += buf[threadIdx.x + o];
        __syncthreads();
    }
    return buf[0];
}

__global__ __launch_bounds__(kThreads) void k_squares(Items a, double* parts) {
    double t = 0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const Item& item = a.item[item_of(a, c)];
        const int64_t from = (int64_t)(c - item.first) * kChunk;
        const int n = (int)(item.count - from < kChunk ? item.count - from : kChunk);
        t += item.bf16 ? squares(static_cast<const uint16_t*>(item.in) + from, n) : squares(static_cast<const float*>(item.in) + from, n);
    }
    t = over_threads(t);
    if (threadIdx.x == 0) parts[blockIdx.x] = t;
}

__device__ __forceinline__ double norm_of(const double* parts, int n) {
    double t = 0;
    for (int k = threadIdx.x; k < n; k += kThreads) t += parts[k];
    return sqrt(over_threads(t));
}
// (NaN stays; a largest norm of infinity asks for no scaling, whatever the norm)
__device__ __forceinline__ double scale_of(double norm, double most) {
    const double r = norm > 0 || norm != norm ? most / norm : 1.0;
    return most == __builtin_inf() || r >= 1.0 ? 1.0 : r;
}
__global__ __launch_bounds__(kThreads) void k_norm(const double* parts, int n, double most, double* kept, float* norm, float* scale) {
    const double t = norm_of(parts, n);
    if (threadIdx.x) return;
    *kept = t;
    *norm = (float)t;
    if (scale) *scale = (float)scale_of(t, most);
}

// (a scale below fp32's smallest normal number: products in 64 bits)
struct Scaling {
    double scale;
    float s;
    __device__ __forceinline__ explicit Scaling(double v) : scale(v), s((float)v) {}
    __device__ __forceinline__ float of(float v) const { return s >= 1.2e-38f || !(scale > 0) ? v * s : (float)(v * scale); }
};
template <bool PAST, class T, class O>
__device__ __forceinline__ void scaled(const T* p, O* to, int n, double scale) {
    const Scaling by(scale);
    if (n == kChunk && aligned(p) && aligned(to)) {
        float v[kTurns][8];
#pragma unroll
        for (int k = 0; k < kTurns; k++) load8(p + (k * kThreads + threadIdx.x) * 8, v[k]);
#pragma unroll
        for (int k = 0; k < kTurns; k++) {
#pragma unroll
            for (int e = 0; e < 8; e++) v[k][e] = by.of(v[k][e]);
            store8<PAST>(to + (k * kThreads + threadIdx.x) * 8, v[k]);
        }
        return;
    }
    int done = 0;
    if (aligned(p) && aligned(to)) {
        done = n & ~7;
        for (int i = threadIdx.x * 8; i < done; i += 8 * kThreads) {
            float v[8];
            load8(p + i, v);
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = by.of(v[e]);
            store8<PAST>(to + i, v);
        }
    }
    for (int i = done + threadIdx.x; i < n; i += kThreads) store1(to + i, by.of(load1(p + i)));
}

// kept: the norm where a launch of its own has left it; else the parts are added here, and workgroup 0 of the first launch writes the results.
template <bool PAST>
__global__ __launch_bounds__(kThreads) void k_scale(Items a, const double* parts, int n, const double* kept, double most, float* norm, float* scale) {
    const double t = kept ? *kept : norm_of(parts, n), s = scale_of(t, most);
    if (!kept && norm && blockIdx.x == 0 && threadIdx.x == 0) {
        *norm = (float)t;
        if (scale) *scale = (float)s;
    }
    for (uint32_t k = blockIdx.x; k < a.chunks; k += gridDim.x) {
        const uint32_t c = a.chunks - 1 - k;
        const Item& item = a.item[item_of(a, c)];
        if (s == 1.0 && item.in == item.out) continue;  // (nothing changes)
        const int64_t from = (int64_t)(c - item.first) * kChunk;
        const int n = (int)(item.count - from < kChunk ? item.count - from : kChunk);
        if (item.bf16) {
            const uint16_t* p = static_cast<const uint16_t*>(item.in) + from;
            if (item.out_bf16)
                scaled<PAST>(p, static_cast<uint16_t*>(item.out) + from, n, s);
            else
                scaled<PAST>(p, static_cast<float*>(item.out) + from, n, s);
        } else {
            const float* p = static_cast<const float*>(item.in) + from;
            if (item.out_bf16)
                scaled<PAST>(p, static_cast<uint16_t*>(item.out) + from, n, s);
            else
                scaled<PAST>(p, static_cast<float*>(item.out) + from, n, s);
        }
    }
}

// Few elements: one workgroup does all of it, in one launch (two tensors of 3000 elements 7 us; in two launches 12 of 60000 in all take 13.6).
constexpr int kAlone = 1024;
__global__ __launch_bounds__(kAlone) void k_alone(Items a, double most, float* norm, float* scale) {
    __shared__ double buf[kAlone / 64];
    double t = 0;
    for (int k = 0; k < a.n; k++) {
        const Item& item = a.item[k];
        for (int64_t i = threadIdx.x; i < item.count; i += kAlone) {
            const double v = item.bf16 ? load1(static_cast<const uint16_t*>(item.in) + i) : load1(static_cast<const float*>(item.in) + i);
            t = fma(v, v, t);
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = t;
    __syncthreads();
    t = 0;
#pragma unroll
    for (int w = 0; w < kAlone / 64; w++) t += buf[w];
    const double all = sqrt(t), s = scale_of(all, most);
    if (threadIdx.x == 0) {
        *norm = (float)all;
        if (scale) *scale = (float)s;
    }
    const Scaling by(s);
    for (int k = 0; k < a.n; k++) {
        const Item& item = a.item[k];
        if (s == 1.0 && item.in == item.out) continue;
        for (int64_t i = threadIdx.x; i < item.count; i += kAlone) {
            const float v = by.of(item.bf16 ? load1(static_cast<const uint16_t*>(item.in) + i) : load1(static_cast<const float*>(item.in) + i));
            if (item.out_bf16)
                store1(static_cast<uint16_t*>(item.out) + i, v);
            else
                store1(static_cast<float*>(item.out) + i, v);
        }
    }
}

}  // namespace

void make_plan(Plan& p) {
    Batch b;
    auto close = [&] {
        if (b.tensors.empty()) return;
        p.batches.push_back(b);
        b = Batch();
    };
    for (size_t i = 0; i < p.tensors.size(); i++) {
        const int64_t chunks = (p.tensors[i].count + kChunk - 1) / kChunk;
        if (!chunks) continue;
        if ((int)b.tensors.size() == kBatch || b.chunks + chunks > INT32_MAX) close();
        b.tensors.push_back((int)i);
        b.chunks += chunks;
    }
    close();
    int64_t all = 0, bytes = 0;
    for (const Tensor& t : p.tensors) {
        all += t.count;
        bytes += t.count * ((t.bf16 ? 2 : 4) + (t.out_bf16 ? 2 : 4));
    }
    // Far more than the last-level cache (256 MB) holds: what is written goes past it, for the gradients that are read a second time to stay.  (2^28 elements of
    // bf16, 1.07 GB read and written, 279 us instead of 312; 10^8 of fp32, 0.8 GB, 234 and 237; but 6 10^7 from bf16 to fp32, 0.36 GB, 141 instead of 108)
    p.past = bytes > (int64_t)768 << 20;
    p.one = p.batches.size() == 1 && all <= kAloneElements;
    const int most = std::max<int>(64, kMostParts / (int)std::max<size_t>(1, p.batches.size()));
    for (Batch& c : p.batches) {
        c.parts = (int)std::min<int64_t>(c.chunks, most);
        c.first_part = p.parts;
        p.parts += c.parts;
    }
    p.alone = p.parts > kMostParts || p.batches.empty();
    const int n = (int)p.batches.size();
    p.launches = p.one ? 1 : 2 * n + p.alone;
    p.launches_norm = n + 1;
    p.workspace_bytes = 8ull * (p.parts + 1);
    p.workspace_bytes = (p.workspace_bytes + 255) & ~(uint64_t)255;
}

void step(const Plan& p, const Args& a, hipStream_t stream) {
    double *parts = reinterpret_cast<double*>(a.ws), *kept = parts + p.parts;
    auto items = [&](const Batch& b) {
        Items t{};
        for (int i : b.tensors) {
            t.item[t.n++] = Item{a.grads[i], a.outs ? a.outs[i] : nullptr, p.tensors[i].count, t.chunks, p.tensors[i].bf16, p.tensors[i].out_bf16};
            t.chunks += (uint32_t)((p.tensors[i].count + kChunk - 1) / kChunk);
        }
        return t;
    };
    if (p.one && a.outs) {
        CANVAS_LAUNCH(k_alone, dim3(1), dim3(kAlone), 0, stream, items(p.batches[0]), a.most, a.norm, a.scale);
        return;
    }
    for (const Batch& b : p.batches) CANVAS_LAUNCH(k_squares, dim3(b.parts), dim3(kThreads), 0, stream, items(b), parts + b.first_part);
    const bool alone = p.alone || !a.outs;
    if (alone) CANVAS_LAUNCH(k_norm, dim3(1), dim3(kThreads), 0, stream, parts, p.parts, a.most, kept, a.norm, a.scale);
    if (!a.outs) return;
    for (size_t k = p.batches.size(); k--;) {
        const Batch& b = p.batches[k];
        const unsigned grid = (unsigned)std::min<int64_t>(b.chunks, 2048);
        if (p.past)
            CANVAS_LAUNCH(k_scale<true>, dim3(grid), dim3(kThreads), 0, stream, items(b), parts, p.parts, alone ? kept : nullptr, a.most, k ? nullptr : a.norm, k ? nullptr : a.scale);
        else
            CANVAS_LAUNCH(k_scale<false>, dim3(grid), dim3(kThreads), 0, stream, items(b), parts, p.parts, alone ? kept : nullptr, a.most, k ? nullptr : a.norm, k ? nullptr : a.scale);
    }
}

}  // namespace clip
}  // namespace canvas
