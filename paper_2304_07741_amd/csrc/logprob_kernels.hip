// Log probabilities of given tokens.
//
// Forward: a row, or a segment of a long one, is read once, 16 bytes per load.  Every thread keeps the largest logit m that it
// has met, S = sum exp(z - z_m) and sum exp(z - z_m) (z - z_m), rescaled whenever m grows, so every exponential is
// taken once; the threads' are joined in a fixed order.  Segments leave theirs, and their best keys, to a second launch.
//
// Alternatives: classes are ordered by whole numbers of 64 bits (order_of the logit, then the complement of the index), all
// different.  Every thread finds its best class on the way; the k-th best of the threads' best is a lower bound for the k-th
// best of all, and only the threads whose best reaches it, k or few more, can hold classes that do: at most as many times a
// thread's classes, few in general.  Theirs are read again, spread over the workgroup; what reaches the bound is collected in
// LDS and ranked by counting.
//
// Backward: element by element from the row's (m, log S, entropy, 1 / S).
//
// Both are bound by memory on many rows, here over three sets of logits in turn: 4096 x 32768 in bf16 forward 53 us (5.0 TB/s; 44 where the
// last-level cache still holds some of them, 62 behind a backward whose gradients are still being written), backward 108 us (5.0
// TB/s), in fp32 93 and 188 us (5.7 TB/s).  With alternatives the search at a row's end is not hidden by other rows' loads: 1500 x 50021
// with five of them takes 43 us, without 39.  Few rows are bound by latency: 256 x 1000 4 us per launch.
#include "logprob_kernels.hpp"

#include <algorithm>

#include "../../include/canvas_logprob.h"
#include "device_util.hpp"
#include "exp_util.hpp"
#include "launch.hpp"
#include "tile_util.hpp"
#include "wave_util.hpp"

namespace canvas {
namespace logprob {
namespace {

using tile::u32x4;
constexpr float kInf = __builtin_inff(), kLowest = -3.402823466e38f;
constexpr int kMostClassesLog = 20;
constexpr uint32_t kMostClasses = 1u << kMostClassesLog;
static_assert(kMostClasses == CANVAS_LOGPROB_MAX_CLASSES && CANVAS_LOGPROB_MAX_TOP <= 64, "limits of the kernels");
constexpr int kJoin = 256;  // threads per row of the launch that joins segments

template <class T>
struct Type;
template <>
struct Type<float> {
    static constexpr int kVec = 4, kLow = 0;
    static __device__ __forceinline__ float at(const u32x4& v, int e) { return __uint_as_float(v[e]); }
    static __device__ __forceinline__ void hide(u32x4& v, int e) { v[e] = 0xff800000u; }
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
};
template <>
struct Type<uint16_t> {
    static constexpr int kVec = 8, kLow = 16;  // (16 bits tell bf16 numbers apart)
    static __device__ __forceinline__ float at(const u32x4& v, int e) { return (e & 1) ? tile::hi_f32(v[e >> 1]) : tile::lo_f32(v[e >> 1]); }
    static __device__ __forceinline__ void hide(u32x4& v, int e) { v[e >> 1] = (e & 1) ? (v[e >> 1] & 0xffffu) | 0xff800000u : (v[e >> 1] & 0xffff0000u) | 0xff80u; }
    static __device__ __forceinline__ float one(const uint16_t* p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ void put(uint16_t* p, float v) { *p = f32_to_bf16(v); }
};

// kVec logits, or their bytes of the mask, from index i on, some of them behind `end` (-inf, and 0): one by one, in few registers.
template <class T>
__device__ __forceinline__ u32x4 last_logits(const T* z, int i, int end) {
    constexpr int V = Type<T>::kVec;
    u32x4 v{};
#pragma unroll 1
    for (int e = 0; e < V; e++) {
        const uint32_t x = __float_as_uint(i + e < end ? Type<T>::one(z + i + e) : -kInf);
        if (V == 4) {
            v = u32x4{v[1], v[2], v[3], x};
        } else {
            v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16 | (x & 0xffff0000u)};
        }
    }
    return v;
}
template <int V>
__device__ __forceinline__ uint64_t mask_bytes(const uint8_t* mask, int i, int end) {
    uint64_t w = 0;
    if (i + V <= end) {
        __builtin_memcpy(&w, mask + i, V);
    } else {
#pragma unroll 1
        for (int e = V - 1; e >= 0; e--) w = w << 8 | (i + e < end ? mask[i + e] : 0);
    }
    return w;
}
__device__ __forceinline__ bool allowed(uint64_t w, int e) { return ((e < 4 ? (uint32_t)w : (uint32_t)(w >> 32)) >> ((e & 3) * 8)) & 0xffu; }
template <class T>
__device__ __forceinline__ void hide_masked(u32x4& v, uint64_t w) {
#pragma unroll
    for (int e = 0; e < Type<T>::kVec; e++)
        if (!allowed(w, e)) Type<T>::hide(v, e);
}

template <int V>
__device__ __forceinline__ u32x4 nothing() {
    return V == 4 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
}

// Vector number `at` of `end` logits; -inf behind them and where the mask hides them.
template <class T>
__device__ __forceinline__ u32x4 load_vector(const T* z, int at, int end, const uint8_t* mask) {
    using Y = Type<T>;
    constexpr int V = Y::kVec;
    const int i = at * V;
    u32x4 v;
    if (i + V <= end)
        __builtin_memcpy(&v, z + i, 16);
    else if (i < end)
        v = last_logits(z, i, end);
    else
        v = nothing<V>();
    if (mask && i < end) {
        hide_masked<T>(v, mask_bytes<V>(mask, i, end));
    }
    return v;
}

// Vectors at, at + STRIDE, ... of `end` logits, -inf behind them, and their bytes of the mask.  All of the whole ones are asked for before
// any is looked at; the one that the row ends in comes one by one.
template <class T, int N, int STRIDE>
__device__ __forceinline__ void load_turn(u32x4 (&v)[N], uint64_t (&w)[N], const T* z, const uint8_t* mask, int at, int end) {
    constexpr int V = Type<T>::kVec;
#pragma unroll
    for (int q = 0; q < N; q++) {
        const int i = (at + q * STRIDE) * V;
        v[q] = nothing<V>();
        w[q] = 0;
        if (i + V <= end) {
            __builtin_memcpy(&v[q], z + i, 16);
            if (mask) __builtin_memcpy(&w[q], mask + i, V);
        }
    }
    const int mine = end / V - at;
    if (end % V && mine >= 0 && mine < N * STRIDE && mine % STRIDE == 0) {
        const int i = end / V * V;
        const u32x4 ending = last_logits(z, i, end);
        const uint64_t bytes = mask ? mask_bytes<V>(mask, i, end) : 0;
#pragma unroll
        for (int q = 0; q < N; q++)
            if (mine == q * STRIDE) {
                v[q] = ending;
                w[q] = bytes;
            }
    }
}

// The order of logits as whole numbers: NaN above all, zeros of both signs equal.  -inf is kNone, below every other.
constexpr uint32_t kNan = 0xffc00000u, kNone = 0x007fffffu;
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t u = __float_as_uint(v + 0.f);
    return v != v ? kNan : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return o == kNan ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t key_of(uint32_t o, uint32_t index) { return o <= kNone ? 0 : (uint64_t)o << 32 | (uint32_t)~index; }

// Over the THREADS threads of a row: a wave, or a workgroup through `buf` (a place per wave; a barrier before it is used again is
// the caller's).
template <int THREADS>
__device__ __forceinline__ float largest_of_row(float v, float* buf) {
    v = wave::over<1, wave::Max>(v);
    if (THREADS == 64) return v;
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; w++) v = fmaxf(v, buf[w]);
    return v;
}
template <int THREADS>
__device__ __forceinline__ void sums_of_row(float& a, float& b, float2* buf) {
    a = wave::over<1, wave::Sum>(a);
    b = wave::over<1, wave::Sum>(b);
    if (THREADS == 64) return;
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; w++) {
        a += buf[w].x;
        b += buf[w].y;
    }
}

constexpr int kTogether = 8;  // keys compared at a time: the list has as many places more
constexpr int kSpare = 8;     // threads more than k that may reach the bound: the search for it ends the earlier, and seldom has to tell ties apart
// The k largest of the keys that the THREADS threads of the workgroup hold, in descending order to `put(rank, key)`, 0 past the
// last one.  best: this thread's largest key; LOW: bits of the order that are the same in all keys of one order.  own(f) calls f
// for each of the thread's keys if they are at hand (pieces = 0); else they fall into `pieces`, and piece(thread, number, f)
// calls f for each key of one.  lds: THREADS keys, then k + kSpare times the keys of a thread and kTogether.
template <int THREADS, int LOW, class OWN, class PIECE, class PUT>
__device__ void select_keys(int k, uint64_t best, int pieces, uint64_t* lds, OWN own, PIECE piece, PUT put) {
    __shared__ uint64_t s_bound;
    __shared__ uint32_t s_count, s_holders, s_holder[64 + kSpare];  // (at most k + kSpare threads reach the bound)
    uint64_t* list = lds + THREADS;
    lds[threadIdx.x] = best;
    if (threadIdx.x == 0) s_count = s_holders = 0;
    __syncthreads();
    if (threadIdx.x < 64) {
        constexpr int kEach = THREADS / 64;
        uint32_t o[kEach], low[kEach];
#pragma unroll
        for (int e = 0; e < kEach; e++) {
            const uint64_t b = lds[e * 64 + threadIdx.x];
            o[e] = (uint32_t)(b >> 32);
            low[e] = (uint32_t)b;
        }
        auto count = [&](auto pred) {
            int n = 0;
#pragma unroll
            for (int e = 0; e < kEach; e++) n += __popcll(__ballot(pred(o[e], low[e])));
            return n;
        };
        // (each one more is read again, or, in a wave, ranked by the few)
        const int spare = pieces || THREADS == 64 ? 2 : kSpare;
        uint64_t bound = 1;  // (of so few threads that hold anything: everything)
        if (count([](uint32_t x, uint32_t) { return x != 0; }) > k + spare) {
            // a t that k threads or few more reach, bit by bit; where too many equal it, the lower indices among those
            uint32_t t = 0;
            int n = THREADS;
            for (int bit = 31; bit >= LOW && n > k + spare; bit--) {
                const uint32_t c = t | 1u << bit;
                const int m = count([=](uint32_t x, uint32_t) { return x >= c; });
                if (m >= k) {
                    t = c;
                    n = m;
                }
            }
            uint32_t l = 0;
            if (n > k + spare) {
                const int r = k - count([=](uint32_t x, uint32_t) { return x >> LOW > t >> LOW; });
                n = THREADS;
                l = ~(kMostClasses - 1u);
                for (int bit = kMostClassesLog - 1; bit >= 0 && n > r + spare; bit--) {
                    const uint32_t c = l | 1u << bit;
                    const int m = count([=](uint32_t x, uint32_t y) { return x >> LOW == t >> LOW && y >= c; });
                    if (m >= r) {
                        l = c;
                        n = m;
                    }
                }
                // (the bits below LOW are all the same in keys of one order: take them from the keys themselves)
#pragma unroll
                for (int e = 0; e < kEach; e++) {
                    const uint64_t who = __ballot(o[e] >> LOW == t >> LOW);
                    if (who) t = __builtin_amdgcn_readlane(o[e], __builtin_ctzll(who));
                }
            }
            bound = (uint64_t)t << 32 | l;
        }
        if (threadIdx.x == 0) s_bound = bound;
    }
    __syncthreads();
    const uint64_t bound = s_bound;
    // (the places in both lists do not matter: the ranks do not depend on them)
    auto candidate = [&](uint64_t key) {
        if (key >= bound) list[atomicAdd(&s_count, 1u)] = key;
    };
    if (pieces == 0) {
        if (best >= bound) own(candidate);
    } else {
        if (best >= bound) s_holder[atomicAdd(&s_holders, 1u)] = threadIdx.x;
        __syncthreads();
        const int items = (int)s_holders * pieces;
        for (int i = threadIdx.x; i < items; i += THREADS) {
            const int h = i / pieces;
            piece((int)s_holder[h], i - h * pieces, candidate);
        }
    }
    __syncthreads();
    const int n = (int)s_count;
    if (threadIdx.x < kTogether) list[n + threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const uint64_t key = list[i];
        int rank = 0;
        for (int j = 0; j < n; j += kTogether) {
#pragma unroll
            for (int e = 0; e < kTogether; e++) rank += list[j + e] > key;
        }
        if (rank < k) put(rank, key);
    }
    for (int i = n + threadIdx.x; i < k; i += THREADS) put(i, (uint64_t)0);
}

// Of differences of logits, for powers of two.  (Finite: a difference of zero times an infinity has no value.)
__device__ __forceinline__ float scale_of(float it) { return fminf(it * kLog2e, -kLowest); }

// What a segment leaves for the join.
struct alignas(16) Part {
    float m, sum, along, unused;
};

__device__ __forceinline__ void write_row(const Fwd& a, int64_t row, const Row& r) {
    if (a.ws) reinterpret_cast<Row*>(a.ws)[row] = r;
    if (a.entropy) a.entropy[row] = r.entropy;
}
// The largest logit so far (the lowest finite value before any), S and sum relative to it, the latter in units of log 2.
struct Running {
    float m = kLowest, sum = 0.f, along = 0.f;
    // Relative to a larger m.  (-300: below it the factor is zero, and the product must not be 0 * inf)
    __device__ __forceinline__ void raise(float to, float scale) {
        const float d = (m - to) * scale, f = __builtin_amdgcn_exp2f(d);
        along = f * (along + sum * fmaxf(d, -300.f));
        sum *= f;
        m = to;
    }
    __device__ __forceinline__ void add(float v, float scale) {
        const float d = (v - m) * scale, x = __builtin_amdgcn_exp2f(d);
        sum += x;
        along += x * fmaxf(d, -300.f);
    }
};

__device__ __forceinline__ Row row_of(const Running& r) {
    const bool empty = r.sum == 0.f;
    return Row{r.m, empty ? -kInf : logf(r.sum), empty ? 0.f : logf(r.sum) - r.along / r.sum, empty ? 0.f : 1.f / r.sum};
}
template <class T>
__device__ __forceinline__ void write_token(const Shape& s, const Fwd& a, int64_t row, const Row& r) {
    if (!a.tokens) return;
    const int64_t t = a.tokens[row];
    float lp = 0.f;
    if (t >= 0 && t < s.classes) {
        const bool hidden = a.mask && !a.mask[row * a.mask_pitch + t];
        const float v = hidden ? -kInf : Type<T>::one(static_cast<const T*>(a.logits) + row * a.pitch + t);
        lp = r.log_sum == -kInf ? -kInf : (v - r.most) * a.it - r.log_sum;
    }
    a.logprob[row] = lp;
}
__device__ __forceinline__ void write_top(const Shape& s, const Fwd& a, int64_t row, const Row& r, int rank, uint64_t key) {
    a.top_index[row * s.top + rank] = key ? (int32_t)~(uint32_t)key : -1;
    a.top_logprob[row * s.top + rank] = key ? (value_of((uint32_t)(key >> 32)) - r.most) * a.it - r.log_sum : -kInf;
}

// One segment of `length` classes per workgroup of THREADS threads, or, with a wave per segment and nothing to select, four of them;
// kSweep vectors of a thread in flight.
constexpr int kSweep = 4;
constexpr int segments_of(int threads, bool top) { return threads == 64 && !top ? 4 : 1; }
template <class T, int THREADS, bool TOP>
__global__ __launch_bounds__(THREADS * segments_of(THREADS, TOP)) void k_fwd(Shape s, Plan p, Fwd a) {
    using Y = Type<T>;
    constexpr int V = Y::kVec;
    extern __shared__ uint64_t lds[];
    __shared__ float most[4];
    __shared__ float2 sums[4];
    const int tid = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t tasks = s.rows * p.segments, per = segments_of(THREADS, TOP);
    const float scale = scale_of(a.it);
    for (int64_t first = (int64_t)blockIdx.x * per; first < tasks; first += (int64_t)gridDim.x * per) {
        const int64_t task = first + (per > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
        if (per > 1 && task >= tasks) break;  // (a wave of its own: no barriers on this path)
        const int64_t row = p.segments == 1 ? task : task / p.segments;
        const int64_t begin = (task - row * p.segments) * p.length;
        const int end = (int)(p.length < s.classes - begin ? p.length : s.classes - begin);
        const T* z = static_cast<const T*>(a.logits) + row * a.pitch + begin;
        const uint8_t* mask = a.mask ? a.mask + row * a.mask_pitch + begin : nullptr;
        const int vectors = (end + V - 1) / V;

        Running r;
        float best_value = -kInf;  // this thread's largest logit, and the first vector that has it
        int best_at = tid;
        u32x4 v[kSweep];
        for (int at = 0; at < vectors; at += kSweep * THREADS) {
            if ((at + kSweep * THREADS) * V <= end) {
#pragma unroll
                for (int q = 0; q < kSweep; q++) __builtin_memcpy(&v[q], z + (at + q * THREADS + tid) * V, 16);
                if (mask) {
                    uint64_t w[kSweep] = {};
#pragma unroll
                    for (int q = 0; q < kSweep; q++) __builtin_memcpy(&w[q], mask + (at + q * THREADS + tid) * V, V);
#pragma unroll
                    for (int q = 0; q < kSweep; q++) hide_masked<T>(v[q], w[q]);
                }
            } else {
                uint64_t w[kSweep];
                load_turn<T, kSweep, THREADS>(v, w, z, mask, at + tid, end);
                if (mask) {
#pragma unroll
                    for (int q = 0; q < kSweep; q++) hide_masked<T>(v[q], w[q]);
                }
            }
            float m = r.m;
#pragma unroll
            for (int q = 0; q < kSweep; q++) {
                float w = Y::at(v[q], 0);
#pragma unroll
                for (int e = 1; e < V; e++) w = fmaxf(w, Y::at(v[q], e));  // (drops NaN: the sums have it)
                if (TOP && w > best_value) {
                    best_value = w;
                    best_at = at + q * THREADS + tid;
                }
                m = fmaxf(m, w);
            }
            r.raise(m, scale);
#pragma unroll
            for (int q = 0; q < kSweep; q++) {
                tile::pin(v[q]);  // (unpacked again, not kept)
#pragma unroll
                for (int e = 0; e < V; e++) r.add(Y::at(v[q], e), scale);
            }
        }
        const float own = r.sum;
        r.raise(largest_of_row<THREADS>(r.m, most), scale);
        sums_of_row<THREADS>(r.sum, r.along, sums);
        r.along *= kLn2;
        const Row whole = row_of(r);
        if (tid == 0) {
            if (p.segments == 1) {
                write_row(a, row, whole);
                write_token<T>(s, a, row, whole);
            } else {
                reinterpret_cast<Part*>(a.ws + p.parts_at)[task] = Part{r.m, r.sum, r.along, 0.f};
            }
        }
        if (TOP) {
            // f(key) for the classes of a thread's vector
            auto piece = [&](int thread, int number, auto f) {
                const int at = number * THREADS + thread;
                const u32x4 w = load_vector(z, at, end, mask);
#pragma unroll
                for (int e = 0; e < V; e++) f(key_of(order_of(Y::at(w, e)), (uint32_t)begin + at * V + e));
            };
            const int pieces = (vectors + THREADS - 1) / THREADS;
            uint64_t best = 0;
            if (own != own) {  // NaN or an infinity among them
#pragma unroll 1
                for (int q = 0; q < pieces; q++) piece(tid, q, [&](uint64_t key) { best = key > best ? key : best; });
            } else if (own > 0.f) {
                u32x4 w = v[0];
                if (pieces <= kSweep) {  // (a short segment is still in the registers)
#pragma unroll
                    for (int q = 1; q < kSweep; q++)
                        if (best_at == q * THREADS + tid) w = v[q];
                } else {
                    w = load_vector(z, best_at, end, mask);
                }
                int e = V - 1;
#pragma unroll
                for (int k = V - 2; k >= 0; k--)
                    if (Y::at(w, k) == best_value) e = k;
                best = key_of(order_of(best_value), (uint32_t)begin + best_at * V + e);
            }
            uint64_t* keys = reinterpret_cast<uint64_t*>(a.ws + p.keys_at) + task * s.top;
            auto own_keys = [&](auto f) {
#pragma unroll
                for (int q = 0; q < kSweep; q++) {
                    if (q * THREADS >= vectors) break;
#pragma unroll
                    for (int e = 0; e < V; e++) f(key_of(order_of(Y::at(v[q], e)), (uint32_t)begin + (q * THREADS + tid) * V + e));
                }
            };
            select_keys<THREADS, Y::kLow>(s.top, best, pieces <= kSweep ? 0 : pieces, lds, own_keys, piece, [&](int rank, uint64_t key) {
                if (p.segments == 1)
                    write_top(s, a, row, whole, rank, key);
                else
                    keys[rank] = key;
            });
        }
        if (TOP || THREADS > 64) __syncthreads();  // (the buffers above are free again)
    }
}

// Joins the segments of a row: at most kMaxSegments of them (with the most alternatives 52 hold the most classes).
constexpr int kListKeys = 6144;  // places of the list of candidates
constexpr int kMaxSegments = 64, kJoinKeys = kMaxSegments * 64 / kJoin;
template <class T>
__global__ __launch_bounds__(kJoin) void k_join(Shape s, Plan p, Fwd a) {
    extern __shared__ uint64_t lds[];
    for (int64_t row = blockIdx.x; row < s.rows; row += gridDim.x) {
        const Part* parts = reinterpret_cast<const Part*>(a.ws + p.parts_at) + row * p.segments;
        const int lane = threadIdx.x & 63;
        const Part mine = lane < p.segments ? parts[lane] : Part{kLowest, 0.f, 0.f, 0.f};
        Running whole{mine.m, mine.sum, mine.along * kLog2e};
        whole.raise(wave::over<1, wave::Max>(mine.m), scale_of(a.it));
        whole.sum = wave::over<1, wave::Sum>(whole.sum);
        whole.along = wave::over<1, wave::Sum>(whole.along) * kLn2;
        const Row r = row_of(whole);
        if (threadIdx.x == 0) {
            write_row(a, row, r);
            write_token<T>(s, a, row, r);
        }
        if (s.top > 0) {
            const uint64_t* from = reinterpret_cast<const uint64_t*>(a.ws + p.keys_at) + row * p.segments * s.top;
            const int n = p.segments * s.top;
            uint64_t key[kJoinKeys], best = 0;
#pragma unroll
            for (int q = 0; q < kJoinKeys; q++) {
                const int i = q * kJoin + threadIdx.x;
                key[q] = i < n ? from[i] : 0;
            }
#pragma unroll
            for (int q = 0; q < kJoinKeys; q++) best = key[q] > best ? key[q] : best;
            select_keys<kJoin, Type<T>::kLow>(
                s.top, best, 0, lds,
                [&](auto f) {
#pragma unroll
                    for (int q = 0; q < kJoinKeys; q++) f(key[q]);
                },
                [](int, int, auto) {},
                [&](int rank, uint64_t k) { write_top(s, a, row, r, rank, k); });
            __syncthreads();
        }
    }
}

// A wave takes kBwdVecs vectors of 64 x 16 bytes of a row.
constexpr int kBwdVecs = 4;
template <class T>
__global__ __launch_bounds__(256) void k_bwd(Shape s, Bwd a, int pieces) {
    using Y = Type<T>;
    constexpr int V = Y::kVec;
    const int lane = threadIdx.x & 63;
    const int64_t tasks = s.rows * pieces;
    for (int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); task < tasks; task += (int64_t)gridDim.x * 4) {
        const int64_t row = pieces == 1 ? task : task / pieces, begin = (task - row * pieces) * (64 * V * kBwdVecs);
        constexpr int kPiece = 64 * V * kBwdVecs;
        const int end = (int)(s.classes - begin < kPiece ? s.classes - begin : kPiece);
        const T* z = static_cast<const T*>(a.logits) + row * a.pitch + begin;
        T* dz = static_cast<T*>(a.dlogits) + row * a.dpitch + begin;
        const uint8_t* mask = a.mask ? a.mask + row * a.mask_pitch + begin : nullptr;
        u32x4 v[kBwdVecs];
#pragma unroll
        for (int q = 0; q < kBwdVecs; q++) v[q] = load_vector<T>(z, q * 64 + lane, end, nullptr);
        uint64_t allow[kBwdVecs];
        if (mask) {
#pragma unroll
            for (int q = 0; q < kBwdVecs; q++) {
                const int i = (q * 64 + lane) * V;
                allow[q] = i < end ? mask_bytes<V>(mask, i, end) : 0;
            }
        }
        const Row r = reinterpret_cast<const Row*>(a.ws)[row];
        const int64_t t = a.tokens ? a.tokens[row] : -1;
        const bool given = t >= 0 && t < s.classes, empty = r.log_sum == -kInf;
        const float g = given && a.dlogprob ? a.dlogprob[row] * a.it : 0.f, h = a.dentropy ? a.dentropy[row] * a.it : 0.f;
#pragma unroll
        for (int q = 0; q < kBwdVecs; q++) {
            const int i = (q * 64 + lane) * V;
            if (i >= end) break;
            float d[V];
#pragma unroll
            for (int e = 0; e < V; e++) {
                // (p from the exponent before log S rounds it; a NaN is in what the row left.  Gradients of 8 bits take the exponential as
                // it is: its 3e-6 at worst is far below their 2e-3, and the other's three operations more cost 9 us at 4096 x 32768)
                const float x = fmaxf((Y::at(v[q], e) - r.most) * a.it, -300.f);
                const float p = (sizeof(T) == 4 ? exp_finite(x) : __builtin_amdgcn_exp2f(x * kLog2e)) * r.inverse;
                d[e] = -p * (g + h * (x - r.log_sum + r.entropy));
                if (begin + i + e == t) d[e] += g;
                if (empty) d[e] = 0.f;
            }
            if (mask) {
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (!allowed(allow[q], e)) d[e] = 0.f;
            }
            if (i + V <= end) {
                u32x4 w;
                if (V == 4) {
#pragma unroll
                    for (int e = 0; e < 4; e++) w[e] = __float_as_uint(d[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++) w[e] = tile::pack_bf16(d[2 * e & (V - 1)], d[(2 * e + 1) & (V - 1)]);
                }
                __builtin_memcpy(dz + i, &w, 16);
            } else {
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (i + e < end) Y::put(dz + i + e, d[e]);
            }
        }
    }
}

// (the kernels walk over what more workgroups than a launch can have would take)
unsigned grid_of(int64_t n, int threads) { return (unsigned)std::min(n, most_workgroups(threads)); }
uint64_t up256(uint64_t v) { return (v + 255) & ~(uint64_t)255; }
int64_t classes_per_thread(int64_t length, int threads, int vec) { return (length + (int64_t)threads * vec - 1) / ((int64_t)threads * vec) * vec; }

template <class T, int THREADS, bool TOP>
void fwd(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    const int64_t tasks = s.rows * p.segments;
    const size_t lds = TOP ? 8ull * (THREADS + kTogether + (s.top + kSpare) * classes_per_thread(p.length, THREADS, Type<T>::kVec)) : 0;
    constexpr int per = segments_of(THREADS, TOP);
    CANVAS_LAUNCH((k_fwd<T, THREADS, TOP>), dim3(grid_of((tasks + per - 1) / per, THREADS * per)), dim3(THREADS * per), lds, stream, s, p, a);
}
template <class T>
void forward_of(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    if (p.threads == 64)
        s.top ? fwd<T, 64, true>(s, p, a, stream) : fwd<T, 64, false>(s, p, a, stream);
    else
        s.top ? fwd<T, 256, true>(s, p, a, stream) : fwd<T, 256, false>(s, p, a, stream);
    if (p.segments > 1) {
        const size_t lds = s.top ? 8ull * (kJoin + kTogether + (s.top + kSpare) * kJoinKeys) : 0;
        CANVAS_LAUNCH(k_join<T>, dim3(grid_of(s.rows, kJoin)), dim3(kJoin), lds, stream, s, p, a);
    }
}
template <class T>
void backward_of(const Shape& s, const Bwd& a, hipStream_t stream) {
    const int piece = 64 * Type<T>::kVec * kBwdVecs;
    const int pieces = (int)((s.classes + piece - 1) / piece);
    CANVAS_LAUNCH(k_bwd<T>, dim3(grid_of((s.rows * pieces + 3) / 4, 256)), dim3(256), 0, stream, s, a, pieces);
}

}  // namespace

Plan plan_of(const Shape& s) {
    Plan p;
    const int vec = s.bf16 ? 8 : 4;
    // With alternatives a segment is as long as the list in LDS allows: k + kSpare times a thread's classes, 48 KB.
    const int64_t most = s.top ? (int64_t)256 * (kListKeys / (s.top + kSpare) / vec * vec) : s.classes;
    int64_t n = (s.classes + most - 1) / most;
    // A few rows leave most compute units idle: segments of 2048 classes or more until there are about as many as those.  (Four rows
    // of 131072 classes with 20 alternatives in 64 segments and their join take 12.8 us, in 16 of them 15.8, unsplit 17.9; of 40960
    // classes 12.3, with a mask 12.9, unsplit 10.9 and 14.3.)
    if (s.rows * n < 256 && s.classes > 40960) {
        const int64_t want = 256 / s.rows, some = s.classes / 2048;
        n = std::max(n, std::min(want, some));
    }
    n = std::min<int64_t>(n, kMaxSegments);
    p.length = ((s.classes + n - 1) / n + vec - 1) / vec * vec;
    p.segments = (int)((s.classes + p.length - 1) / p.length);
    // A wave takes a short row in one turn of its loads, in two if there are few alternatives, and twice as many where there are waves for
    // all compute units (bf16, five alternatives: 4000 x 1000 11 us, with 256 threads 26; 4000 x 3000 13 and 25; 4000 x 5003 18 and
    // 30, but 256 x 5003 with a mask 12.5 and 10.3; with 20 of them 256 x 3000 9.1 and 8.2).  It selects alternatives as long as half of its
    // threads bound them (4000 x 1000 with 32 12 and 30 us, with 64, in fp32, 499 and 25; 4000 x 8192 with 32 92 and 32), and
    // segments have the compute units to themselves (four rows of 131072, masked: 16.3 and 15.6 us).
    const int64_t turns = (s.rows >= 2048 ? 2 : 1) * (s.top <= 8 ? 2 : 1);
    p.threads = p.length <= turns * 64 * vec * kSweep && (!s.top || (s.top <= 32 && p.segments == 1)) ? 64 : 256;
    const uint64_t tasks = (uint64_t)s.rows * p.segments;
    p.workspace_bytes = up256((uint64_t)s.rows * sizeof(Row));
    if (p.segments > 1) {
        p.parts_at = p.workspace_bytes;
        p.keys_at = p.parts_at + up256(tasks * sizeof(Part));
        p.workspace_bytes = p.keys_at + up256(tasks * s.top * 8);
        p.launches_fwd = 2;
    }
    return p;
}

void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream) {
    if (s.bf16)
        forward_of<uint16_t>(s, p, a, stream);
    else
        forward_of<float>(s, p, a, stream);
}

void backward(const Shape& s, const Plan&, const Bwd& a, hipStream_t stream) {
    if (s.bf16)
        backward_of<uint16_t>(s, a, stream);
    else
        backward_of<float>(s, a, stream);
}

}  // namespace logprob
}  // namespace canvas
