// Calls of heads with and without a mask, the runtime's launch functions in this program's place: nothing reaches a GPU, addresses are numbers.  Prints "calls <n> wrong <m>":
// as many launches are made as the query says, of plans that copy a masked weight piece by piece, as a whole, in forward or not at all.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>

#include "../../include/canvas_head.h"

static int g_launches = 0;
static dim3 g_grid, g_block;
static size_t g_lds;

extern "C" hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) {
    g_launches++;
    return hipSuccess;
}
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t) {
    g_grid = grid;
    g_block = block;
    g_lds = lds;
    return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = g_grid;
    *block = g_block;
    *lds = g_lds;
    *stream = nullptr;
    return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return hipSuccess; }

static void* place(int k) { return reinterpret_cast<void*>((uint64_t)(k + 1) << 50); }

int main() {
    long calls = 0, wrong = 0, more = 0;
    for (canvas_dtype dt : {CANVAS_F32, CANVAS_BF16})
        for (int64_t rows : {1, 16, 32, 33, 300, 5000, 40000})
            for (int64_t features : {1, 8, 40, 65, 512, 2048, 4000})
                for (int64_t classes : {1, 100, 4000, 50021, 200000})
                    for (bool masked : {false, true}) {
                        canvas_head* h = nullptr;
                        if (canvas_head_compile(rows, features, classes, dt, nullptr, &h)) continue;
                        canvas_head_info in{};
                        canvas_head_query(h, &in);
                        const uint8_t* mask = masked ? static_cast<const uint8_t*>(place(9)) : nullptr;
                        const int64_t* tokens = static_cast<const int64_t*>(place(2));
                        g_launches = 0;
                        int rc = canvas_head_forward(h, place(0), place(1), 1.f, mask, tokens, (float*)place(3), (float*)place(4), place(50), in.workspace_bytes, nullptr);
                        bool ok = !rc && g_launches == in.n_launches_fwd;
                        g_launches = 0;
                        rc = canvas_head_backward(h, place(0), place(1), 1.f, mask, tokens, (float*)place(5), (float*)place(6), place(7), place(8), place(50), in.workspace_bytes, nullptr);
                        ok &= !rc && g_launches == in.n_launches_bwd + (masked ? in.n_launches_bwd_mask : 0);
                        // twice the products of forward, and those that are made again
                        const double f = in.flops_fwd;
                        ok &= in.flops_bwd >= 2 * f && in.flops_bwd <= 3 * f;
                        if (!ok && wrong++ < 20)
                            printf("wrong: %ld x %ld x %ld type %d mask %d: %d launches for %d + %d\n", (long)rows, (long)features, (long)classes, (int)dt, (int)masked, g_launches, in.n_launches_bwd,
                                   in.n_launches_bwd_mask);
                        calls++;
                        more += masked && in.n_launches_bwd_mask > 1;
                        canvas_head_destroy(h);
                    }
    printf("calls %ld wrong %ld several %ld\n", calls, wrong, more);
    return 0;
}
