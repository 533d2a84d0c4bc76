// Calls of the operators around a block with the runtime's launch functions in this program's place: nothing reaches a GPU, addresses
// are numbers.  First argument: what is looked at; prints "<what> cases <n> wrong <m>".
//
//   overlap   calls whose tensors share bytes where a call writes are refused before anything is launched, others are not
//   lds       every launch with more than 64 KB of LDS has asked for as much, whatever shapes came before it
//   threads   no launch has 2^32 threads or more along a dimension, over all shapes that the headers accept
#include <hip/hip_runtime.h>

#include <algorithm>
#include <chrono>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "../../include/canvas_logprob.h"
#include "../../include/canvas_norm.h"
#include "../../include/canvas_ortho.h"

struct Launch {
    const void* kernel;
    dim3 grid, block;
    size_t lds;
};
static std::vector<Launch> g_launches;
static std::map<const void*, int> g_allowed;  // LDS that was asked for, by kernel

extern "C" hipError_t hipLaunchKernel(const void* kernel, dim3 grid, dim3 block, void**, size_t lds, hipStream_t) {
    g_launches.push_back(Launch{kernel, grid, block, lds});
    return hipSuccess;
}
static Launch g_configuration;  // of the launch that is being made
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t) {
    g_configuration = Launch{nullptr, grid, block, lds};
    return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = g_configuration.grid;
    *block = g_configuration.block;
    *lds = g_configuration.lds;
    *stream = nullptr;
    return hipSuccess;
}
extern "C" hipError_t hipFuncSetAttribute(const void* kernel, hipFuncAttribute attr, int value) {
    if (attr == hipFuncAttributeMaxDynamicSharedMemorySize) g_allowed[kernel] = value;
    return hipSuccess;
}
extern "C" hipError_t hipGetDevice(int* d) {
    *d = 0;
    return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return hipSuccess; }

static long g_cases = 0, g_wrong = 0;
static void expect(bool ok, const std::string& what) {
    g_cases++;
    if (!ok && g_wrong++ < 20) printf("wrong: %s (%s)\n", what.c_str(), canvas_last_error());
}

// ---------------------------------------------------------------- calls with tensors far apart

static void* place(int k) { return reinterpret_cast<void*>((uint64_t)(k + 1) << 44); }
static uint8_t* const kSpace = static_cast<uint8_t*>(place(40));
static int norm_forward_and_backward(int64_t n, int64_t c, int64_t p, canvas_dtype dt, uint32_t parts, int gate) {
    const int64_t shape[4] = {n, c, p, 1};
    canvas_norm* h = nullptr;
    if (int rc = canvas_norm_compile(shape, dt, parts, (canvas_gate)gate, 1e-6f, nullptr, &h)) return rc;
    canvas_norm_info info;
    canvas_norm_query(h, &info);
    auto f = [](int k) { return static_cast<float*>(place(k)); };
    g_launches.clear();
    int rc = canvas_norm_forward(h, place(0), place(1), place(2), f(3), f(4), f(5), place(6), place(7), kSpace, info.workspace_bytes, nullptr);
    if (!rc) rc = canvas_norm_backward(h, place(0), place(1), place(2), f(3), f(4), f(5), place(8), place(9), place(10), place(11), place(12), f(13), f(14), f(15), kSpace, info.workspace_bytes, nullptr);
    canvas_norm_destroy(h);
    return rc;
}
static int ortho_step(int64_t g, int64_t r, int64_t k, canvas_dtype dt, int steps) {
    const int64_t shape[3] = {g, r, k};
    canvas_ortho* h = nullptr;
    if (int rc = canvas_ortho_compile(shape, dt, steps, CANVAS_ORTHO_NESTEROV, &h)) return rc;
    canvas_ortho_info info;
    canvas_ortho_query(h, &info);
    auto f = [](int k) { return static_cast<float*>(place(k)); };
    g_launches.clear();
    const int rc = canvas_ortho_step(h, f(0), f(1), f(2), 0.9, f(3), f(4), 0.1, 0.0, place(5), place(6), kSpace, info.workspace_bytes, nullptr);
    canvas_ortho_destroy(h);
    return rc;
}

static int logprob_forward_and_backward(int64_t rows, int64_t classes, canvas_dtype dt, int top) {
    canvas_logprob* h = nullptr;
    if (int rc = canvas_logprob_compile(rows, classes, dt, top, nullptr, &h)) return rc;
    canvas_logprob_info info;
    canvas_logprob_query(h, &info);
    auto f = [](int k) { return static_cast<float*>(place(k)); };
    g_launches.clear();
    int rc = canvas_logprob_forward(h, place(0), classes, 1.f, nullptr, 0, (int64_t*)place(1), f(2), f(3), f(4), (int32_t*)place(5), kSpace, info.workspace_bytes, nullptr);
    if (!rc) rc = canvas_logprob_backward(h, place(0), classes, 1.f, nullptr, 0, (int64_t*)place(1), f(6), f(7), place(8), classes, kSpace, info.workspace_bytes, nullptr);
    canvas_logprob_destroy(h);
    return rc;
}

// ---------------------------------------------------------------- threads

static void threads() {
    constexpr uint64_t kMost = (uint64_t)1 << 32;
    auto look = [](int rc, bool may_refuse, const std::string& what) {
        if (may_refuse && rc == CANVAS_UNSUPPORTED) return expect(g_launches.empty(), what + " refused");
        bool ok = rc == CANVAS_OK && !g_launches.empty();
        for (const Launch& l : g_launches)
            ok &= (uint64_t)l.grid.x * l.block.x < kMost && (uint64_t)l.grid.y * l.block.y < 65536 && l.grid.z == 1 && l.block.x <= 1024 && l.grid.x > 0 && l.grid.y > 0;
        expect(ok, what);
    };
    const int64_t pixels[] = {1, 1 << 20, (1 << 24) + 1, (1 << 26) - 1, (1 << 26) + 3, (1 << 27) + 1, (1 << 28) - 16, (1 << 28) + 1, (1 << 30) + 5, 0x7fffffff};
    for (canvas_dtype dt : {CANVAS_F32, CANVAS_BF16})
        for (int64_t p : {1, 2, 3, 8, 49})
            for (int64_t np : pixels)
                for (int64_t c : {1, 16, 64, 129, 512, 1024})
                    for (uint32_t parts = 1; parts <= 3; parts++)
                        look(norm_forward_and_backward(std::max<int64_t>(1, np / p), c, p, dt, parts, 0), false,
                             "norm " + std::to_string(np / p) + " x " + std::to_string(c) + " x " + std::to_string(p));
    for (canvas_dtype dt : {CANVAS_F32, CANVAS_BF16})
        for (int64_t rows : pixels)
            for (int64_t classes : {1, 10, 2000, 9000})
                for (int top : {0, 5, 64}) {
                    if (rows * classes > (int64_t)1 << 41) continue;
                    look(logprob_forward_and_backward(rows, classes, dt, top), false, "logprob " + std::to_string(rows) + " x " + std::to_string(classes) + " top " + std::to_string(top));
                }
    for (int64_t g : {1, 7, 1000, 65535})
        for (int64_t m : {1, 2, 33, 64, 65, 300, 4000, 16384})
            for (int64_t n : pixels)
                for (int tall = 0; tall < 2; tall++)
                    for (int steps : {0, 1, 5}) {
                        g_launches.clear();
                        look(ortho_step(g, tall ? n : m, tall ? m : n, CANVAS_BF16, steps), true, "ortho " + std::to_string(g) + " of " + std::to_string(m) + " x " + std::to_string(n));
                    }
}

// ---------------------------------------------------------------- lds

static void lds() {
    auto look = [](int rc, const std::string& what) {
        bool ok = rc == CANVAS_OK && !g_launches.empty();
        for (const Launch& l : g_launches) ok &= l.lds <= 65536 || (g_allowed.count(l.kernel) && (int64_t)l.lds <= g_allowed[l.kernel] && l.lds <= 163840);
        expect(ok, what);
    };
    for (canvas_dtype dt : {CANVAS_F32, CANVAS_BF16})
        for (uint32_t parts = 1; parts <= 3; parts++)
            for (int gate = 0; gate <= ((parts & 1) ? 2 : 0); gate++)
                for (int64_t p : {1, 2, 9, 64})
                    for (int64_t c : {8200, 9000, 16384, 8300, 12000})
                        look(norm_forward_and_backward(3, c, p, dt, parts, gate), "norm " + std::to_string(c) + " channels, " + std::to_string(p) + " pixels");
    const int64_t small[][2] = {{63, 65}, {64, 100}, {64, 256}, {48, 480}, {16, 1400}, {63, 65}};
    for (canvas_dtype dt : {CANVAS_F32, CANVAS_BF16})
        for (const auto& s : small) look(ortho_step(2, s[0], s[1], dt, 5), "ortho " + std::to_string(s[0]) + " x " + std::to_string(s[1]));
}

// ---------------------------------------------------------------- overlap

struct Tensor {
    const char* name;
    uint64_t bytes;
    bool written;
    uint64_t at = 0;
    void* p() const { return reinterpret_cast<void*>(at); }
};
template <class CALL>
static int call(CALL f, const std::vector<Tensor>& t, bool& launched) {
    g_launches.clear();
    const int rc = f(t);
    launched = !g_launches.empty();
    return rc;
}
// Every tensor apart, then each pair of which one is written: at one place, the one's end on the other's beginning, and side by side.
template <class CALL, class MAY>
static void pairs(const std::string& what, std::vector<Tensor> t, CALL f, MAY may) {
    uint64_t at = 1ull << 32;
    for (Tensor& x : t) {
        x.at = at;
        at += (x.bytes + 4095) / 4096 * 4096 + (1 << 20);
    }
    bool launched;
    expect(call(f, t, launched) == CANVAS_OK && launched, what + ": all apart");
    for (size_t i = 0; i < t.size(); i++)
        for (size_t j = 0; j < t.size(); j++) {
            if (i == j || !t[i].written) continue;
            const std::string pair = what + ": " + t[i].name + " and " + t[j].name;
            std::vector<Tensor> v = t;
            const uint64_t room = at;  // behind all others
            const uint64_t last_i = (t[i].bytes - 1) / 16 * 16, last_j = (t[j].bytes - 1) / 16 * 16;
            v[i].at = v[j].at = room;
            const bool fine = may(t[i].name, t[j].name);
            expect((call(f, v, launched) == (fine ? CANVAS_OK : CANVAS_BAD_ARG)) && launched == fine, pair + " at one place");
            if (last_i || last_j) {
                v[i].at = room;
                v[j].at = room + last_i;
                if (last_i) expect(call(f, v, launched) == CANVAS_BAD_ARG && !launched, pair + ", the second on the first's end");
                v[i].at = room + last_j;
                v[j].at = room;
                if (last_j) expect(call(f, v, launched) == CANVAS_BAD_ARG && !launched, pair + ", the first on the second's end");
            }
            v[i].at = room;
            v[j].at = room + (t[i].bytes + 15) / 16 * 16;
            expect(call(f, v, launched) == CANVAS_OK && launched, pair + " side by side");
        }
}

static void norm_overlap() {
    for (int64_t P : {1, 6, 49})
        for (uint32_t parts = 1; parts <= 3; parts++)
            for (int gate = 0; gate <= ((parts & 1) ? 2 : 0); gate++) {
                const int64_t shape[4] = {3, 40, P, 1};
                const uint64_t map = 2ull * 3 * 40 * P, vec = 160;
                const bool post = parts & CANVAS_NORM_POST, pre = parts & CANVAS_NORM_PRE;
                canvas_norm* h = nullptr;
                if (canvas_norm_compile(shape, CANVAS_BF16, parts, (canvas_gate)gate, 1e-6f, nullptr, &h)) return expect(false, "norm compile");
                canvas_norm_info info;
                canvas_norm_query(h, &info);
                const std::string what = "norm parts " + std::to_string(parts) + " pixels " + std::to_string(P) + " gate " + std::to_string(gate);
                std::vector<Tensor> f{{"x", map, false}, {"workspace", info.workspace_bytes, true}};
                if (post) f.insert(f.end(), {{"z", map, false}, {"w_post", vec, false}, {"scale", vec, false}, {"x_out", map, true}});
                if (gate) f.push_back({"gate", map, false});
                if (pre) f.insert(f.end(), {{"w_pre", vec, false}, {"u", map, true}});
                auto get = [](const std::vector<Tensor>& t, const char* name) -> void* {
                    for (const Tensor& x : t)
                        if (!strcmp(x.name, name)) return x.p();
                    return nullptr;
                };
                auto none = [](const char*, const char*) { return false; };
                auto fl = [&](const std::vector<Tensor>& t, const char* n) { return static_cast<float*>(get(t, n)); };
                pairs(what, f,
                      [&](const std::vector<Tensor>& t) {
                          return canvas_norm_forward(h, get(t, "x"), get(t, "z"), get(t, "gate"), fl(t, "w_post"), fl(t, "scale"), fl(t, "w_pre"), get(t, "x_out"),
                                                     get(t, "u"), get(t, "workspace"), info.workspace_bytes, nullptr);
                      },
                      none);
                std::vector<Tensor> b{{"dx_out", map, false}, {"workspace", info.workspace_bytes, true}};
                if (post) b.insert(b.end(), {{"z", map, false}, {"w_post", vec, false}, {"scale", vec, false}, {"dz", map, true}, {"dw_post", vec, true}, {"dscale", vec, true}});
                if (gate) b.insert(b.end(), {{"gate", map, false}, {"dgate", map, true}});
                if (pre) b.insert(b.end(), {{"x", map, false}, {"w_pre", vec, false}, {"du", map, false}, {"dx", map, true}, {"dw_pre", vec, true}});
                pairs(what + " backward", b,
                      [&](const std::vector<Tensor>& t) {
                          return canvas_norm_backward(h, get(t, "x"), get(t, "z"), get(t, "gate"), fl(t, "w_post"), fl(t, "scale"), fl(t, "w_pre"), get(t, "dx_out"),
                                                      get(t, "du"), get(t, "dx"), get(t, "dz"), get(t, "dgate"), fl(t, "dw_post"), fl(t, "dscale"), fl(t, "dw_pre"),
                                                      get(t, "workspace"), info.workspace_bytes, nullptr);
                      },
                      none);
                canvas_norm_destroy(h);
            }
}

static void logprob_overlap() {
    const int64_t rows = 9, classes = 100;
    for (int64_t pitch : {100, 137}) {
        canvas_logprob* h = nullptr;
        if (canvas_logprob_compile(rows, classes, CANVAS_F32, 3, nullptr, &h)) return expect(false, "logprob compile");
        canvas_logprob_info info;
        canvas_logprob_query(h, &info);
        const uint64_t map = 4ull * ((rows - 1) * pitch + classes);
        const std::string what = "logprob pitch " + std::to_string(pitch);
        std::vector<Tensor> f{{"logits", map, false}, {"mask", (uint64_t)((rows - 1) * 128 + classes), false}, {"tokens", 8 * rows, false}, {"logprob", 4 * rows, true},
                              {"entropy", 4 * rows, true}, {"top_logprob", 12 * rows, true}, {"top_index", 12 * rows, true}, {"workspace", info.workspace_bytes, true}};
        if (pitch == classes)  // (with gaps between the rows a small tensor finds room in them)
            pairs(what, f,
                  [&](const std::vector<Tensor>& t) {
                      return canvas_logprob_forward(h, t[0].p(), pitch, 1.f, (uint8_t*)t[1].p(), 128, (int64_t*)t[2].p(), (float*)t[3].p(), (float*)t[4].p(), (float*)t[5].p(),
                                                    (int32_t*)t[6].p(), t[7].p(), info.workspace_bytes, nullptr);
                  },
                  [](const char*, const char*) { return false; });
        std::vector<Tensor> b{{"logits", map, false}, {"dlogits", map, true}, {"tokens", 8 * rows, false}, {"dlogprob", 4 * rows, false}, {"dentropy", 4 * rows, false}, {"workspace", info.workspace_bytes, false}};
        auto backward = [&](uint64_t logits, int64_t pitch, uint64_t dlogits, int64_t dpitch) {
            g_launches.clear();
            const int rc = canvas_logprob_backward(h, (void*)logits, pitch, 1.f, nullptr, 0, (int64_t*)(1ull << 20), (float*)(1ull << 21), (float*)(1ull << 22), (void*)dlogits, dpitch,
                                                   (void*)(1ull << 23), info.workspace_bytes, nullptr);
            return rc == CANVAS_OK ? g_launches.empty() ? -100 : 0 : g_launches.empty() ? rc : -101;
        };
        if (pitch == classes)
            pairs(what + " backward", b,
                  [&](const std::vector<Tensor>& t) {
                      return canvas_logprob_backward(h, t[0].p(), pitch, 1.f, nullptr, 0, (int64_t*)t[2].p(), (float*)t[3].p(), (float*)t[4].p(), t[1].p(), pitch, t[5].p(),
                                                     info.workspace_bytes, nullptr);
                  },
                  [](const char* a, const char* b) { return !strcmp(a, "dlogits") && !strcmp(b, "logits"); });
        // rows between each other's rows, by brute force over the bytes
        const uint64_t at = 1ull << 32;
        for (int64_t dpitch : {100, 137, 200, 250})
            for (int64_t lp : {100, 137, 200, 250})
                for (int64_t off = -1200; off <= 1200; off += 7) {
                    bool meet = false;
                    for (int64_t i = 0; i < rows; i++)
                        for (int64_t j = 0; j < rows; j++) {
                            const int64_t d = off + j * dpitch - i * lp;
                            meet |= d < classes && d > -classes;
                        }
                    const bool same = off == 0 && dpitch == lp;
                    const int want = same || !meet ? 0 : CANVAS_BAD_ARG;
                    expect(backward(at, lp, at + 4 * off, dpitch) == want, "logprob pitches " + std::to_string(lp) + " and " + std::to_string(dpitch) + " offset " + std::to_string(off));
                }
        canvas_logprob_destroy(h);
    }
}

// Gradients beside the logits in one wide buffer, a billion rows of them: told apart without looking at every row.
static void many_rows_overlap() {
    canvas_logprob* h = nullptr;
    if (canvas_logprob_compile(1 << 30, 10, CANVAS_F32, 0, nullptr, &h)) return expect(false, "logprob compile");
    canvas_logprob_info info;
    canvas_logprob_query(h, &info);
    const uint64_t at = 1ull << 44;
    const auto begin = std::chrono::steady_clock::now();
    for (int64_t off : {-20ll * ((1 << 30) - 1) - 10, -20ll * (1 << 29) - 5, -21ll, -20ll, -11ll, -10ll, -1ll, 0ll, 1ll, 9ll, 10ll, 11ll, 20ll, 20ll * (1 << 29) + 10, 20ll * ((1 << 30) - 1) + 9, 20ll << 30}) {
        const int64_t left = ((off % 20) + 20) % 20;
        const bool apart = left == 10 || off >= 20ll * ((1 << 30) - 1) + 10, same = off == 0;
        g_launches.clear();
        const int rc = canvas_logprob_backward(h, (void*)at, 20, 1.f, nullptr, 0, (int64_t*)place(3), (float*)place(4), (float*)place(5), (void*)(at + 4 * off), 20, kSpace, info.workspace_bytes, nullptr);
        expect(rc == (apart || same ? CANVAS_OK : CANVAS_BAD_ARG) && g_launches.empty() == (rc != CANVAS_OK), "a billion rows, offset " + std::to_string(off));
    }
    const double s = std::chrono::duration<double>(std::chrono::steady_clock::now() - begin).count();
    expect(s < 0.5, "a billion rows: " + std::to_string(s) + " s");
    canvas_logprob_destroy(h);
}

static void ortho_overlap() {
    for (int64_t R : {8, 200}) {
        const int64_t shape[3] = {2, R, 80};
        const uint64_t f32 = 4ull * 2 * R * 80, bf16 = f32 / 2;
        canvas_ortho* h = nullptr;
        if (canvas_ortho_compile(shape, CANVAS_BF16, 5, 0, &h)) return expect(false, "ortho compile");
        canvas_ortho_info info;
        canvas_ortho_query(h, &info);
        std::vector<Tensor> t{{"grad", f32, false}, {"momentum", f32, false}, {"momentum_out", f32, true}, {"master", f32, false}, {"master_out", f32, true},
                              {"weights", bf16, true}, {"update", bf16, true}, {"workspace", info.workspace_bytes, true}};
        pairs("ortho rows " + std::to_string(R), t,
              [&](const std::vector<Tensor>& t) {
                  return canvas_ortho_step(h, (float*)t[0].p(), (float*)t[1].p(), (float*)t[2].p(), 0.9, (float*)t[3].p(), (float*)t[4].p(), 0.1, 0.0, t[5].p(), t[6].p(),
                                           t[7].p(), info.workspace_bytes, nullptr);
              },
              [](const char* a, const char* b) {
                  return (!strcmp(a, "momentum_out") && !strcmp(b, "momentum")) || (!strcmp(a, "master_out") && !strcmp(b, "master"));
              });
        canvas_ortho_destroy(h);
    }
}

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "overlap") {
        norm_overlap();
        logprob_overlap();
        many_rows_overlap();
        ortho_overlap();
    }
    if (what == "lds") lds();
    if (what == "threads") threads();
    printf("%s cases %ld wrong %ld\n", what.c_str(), g_cases, g_wrong);
    return g_cases && !g_wrong ? 0 : 1;
}
