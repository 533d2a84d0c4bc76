// Calls of gated pairs, heads and the clipping of gradients with the runtime's launch functions in this program's place: nothing reaches a GPU, addresses
// are numbers.  Prints "launches cases <n> wrong <m>": no launch has 2^32 threads or more along a dimension, none is empty, as many are made as the plan says,
// and none asks for more LDS than it may, over shapes that the headers accept.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <string>
#include <vector>

#include "../../include/canvas_clip.h"
#include "../../include/canvas_gated.h"
#include "../../include/canvas_head.h"

struct Launch {
    dim3 grid, block;
    size_t lds;
};
static std::vector<Launch> g_launches;

extern "C" hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t lds, hipStream_t) {
    g_launches.push_back(Launch{grid, block, lds});
    return hipSuccess;
}
static Launch g_configuration;  // of the launch that is being made
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t) {
    g_configuration = Launch{grid, block, lds};
    return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = g_configuration.grid;
    *block = g_configuration.block;
    *lds = g_configuration.lds;
    *stream = nullptr;
    return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return hipSuccess; }

static long g_cases = 0, g_wrong = 0;
static void expect(bool ok, const std::string& what) {
    g_cases++;
    if (!ok && g_wrong++ < 20) printf("wrong: %s (%s)\n", what.c_str(), canvas_last_error());
}
static void look(int rc, int64_t launches, const std::string& what) {
    if (rc == CANVAS_UNSUPPORTED) return expect(g_launches.empty(), what + " refused");
    bool ok = rc == CANVAS_OK && (int64_t)g_launches.size() == launches;
    for (const Launch& l : g_launches)
        ok &= (uint64_t)l.grid.x * l.block.x < (uint64_t)1 << 32 && l.grid.y < 65536 && l.grid.z == 1 && l.block.x <= 1024 && l.grid.x > 0 && l.grid.y > 0 && l.lds == 0;
    expect(ok, what + " " + std::to_string(g_launches.size()) + " launches for " + std::to_string(launches));
}

static void* place(int k) { return reinterpret_cast<void*>((uint64_t)(k + 1) << 50); }
static float* number(int k) { return static_cast<float*>(place(k)); }

int main() {
    const int64_t many[] = {1, 16, 17, 32, 33, 100, 1500, 40000, 1 << 20, (1 << 24) + 1, (1 << 27) - 3, 0x7fffffff}, some[] = {1, 8, 40, 129, 1000, 8192, 50021, 1 << 18};
    for (canvas_dtype dt : {CANVAS_F32, CANVAS_BF16})
        for (int64_t rows : many)
            for (int64_t c : {1, 8, 100, 1000, 1 << 18})
                for (int64_t f : some)
                    for (uint32_t flags : {0u, (uint32_t)CANVAS_OPT_INFERENCE}) {
                        canvas_options opt{};
                        opt.flags = flags;
                        const std::string what = std::to_string(rows) + " x " + std::to_string(c) + " x " + std::to_string(f) + (dt == CANVAS_F32 ? " fp32" : " bf16");
                        g_launches.clear();
                        canvas_gated* g = nullptr;
                        int rc = canvas_gated_compile(rows, c, f, dt, CANVAS_GATED_SILU, &opt, &g);
                        canvas_gated_info info{};
                        if (!rc) {
                            canvas_gated_query(g, &info);
                            rc = canvas_gated_forward(g, place(0), place(1), place(2), place(3), place(50), info.workspace_bytes, nullptr);
                            if (!rc && !flags) rc = canvas_gated_backward(g, place(0), place(1), place(2), place(4), place(5), place(6), place(7), place(50), info.workspace_bytes, nullptr);
                            canvas_gated_destroy(g);
                        }
                        look(rc, info.n_launches_fwd + info.n_launches_bwd, "gated " + what);
                        g_launches.clear();
                        canvas_head* h = nullptr;
                        rc = canvas_head_compile(rows, c, f, dt, &opt, &h);
                        canvas_head_info in{};
                        if (!rc) {
                            canvas_head_query(h, &in);
                            rc = canvas_head_forward(h, place(0), place(1), 1.f, nullptr, (int64_t*)place(2), number(3), number(4), place(50), in.workspace_bytes, nullptr);
                            if (!rc && !flags)
                                rc = canvas_head_backward(h, place(0), place(1), 1.f, nullptr, (int64_t*)place(2), number(5), number(6), place(7), place(8), place(50), in.workspace_bytes, nullptr);
                            canvas_head_destroy(h);
                        }
                        look(rc, in.n_launches_fwd + in.n_launches_bwd, "head " + what);
                    }
    for (int64_t n : {1, 2, 95, 96, 97, 1000, 65536})
        for (int64_t count : {0, 1, 100, 20000, 1 << 24, 1 << 30}) {
            std::vector<int64_t> counts(n, count);
            std::vector<canvas_dtype> types(n, CANVAS_BF16);
            std::vector<const void*> in(n);
            std::vector<void*> out(n);
            for (int64_t i = 0; i < n; i++) {
                in[i] = (char*)place(0) + i * ((uint64_t)1 << 31);
                out[i] = (char*)place(200) + i * ((uint64_t)1 << 31);
            }
            g_launches.clear();
            canvas_clip* c = nullptr;
            int rc = canvas_clip_compile((int32_t)n, counts.data(), types.data(), nullptr, &c);
            canvas_clip_info info{};
            if (!rc) {
                canvas_clip_query(c, &info);
                rc = canvas_clip_step(c, in.data(), out.data(), 1.0, number(500), nullptr, place(501), info.workspace_bytes, nullptr);
            }
            look(rc, info.n_launches, "clip " + std::to_string(n) + " of " + std::to_string(count));
            g_launches.clear();
            if (!rc) {
                rc = canvas_clip_step(c, in.data(), nullptr, 1.0, number(500), nullptr, place(501), info.workspace_bytes, nullptr);
                look(rc, info.n_launches_norm, "norm of " + std::to_string(n) + " of " + std::to_string(count));
                canvas_clip_destroy(c);
            }
        }
    printf("launches cases %ld wrong %ld\n", g_cases, g_wrong);
    return 0;
}
