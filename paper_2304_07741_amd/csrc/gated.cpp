// C ABI of the gated pair of FCs (include/canvas_gated.h): checks, workspace, launches.
#include "../../include/canvas_gated.h"

#include <memory>

#include "abi.hpp"
#include "gated_kernels.hpp"
#include "launch.hpp"

struct canvas_gated {
    canvas::gated::Shape s;
    canvas::gated::Plan plan;
    canvas_gated_info info{};
};

namespace {
using canvas::set_last_error;
using namespace canvas::abi;
}  // namespace

extern "C" {

int canvas_gated_compile(int64_t rows, int64_t features, int64_t width, canvas_dtype dt, canvas_gated_act act, const canvas_options* opt, canvas_gated** out) {
    return guarded([&]() -> int {
        if (!out) return set_last_error(CANVAS_BAD_ARG, "null output handle");
        *out = nullptr;
        if (dt != CANVAS_F32 && dt != CANVAS_BF16) return set_last_error(CANVAS_BAD_ARG, "unknown dtype");
        if (act != CANVAS_GATED_SIGMOID && act != CANVAS_GATED_SILU && act != CANVAS_GATED_GELU) return set_last_error(CANVAS_BAD_ARG, "unknown activation");
        uint32_t flags = 0;
        if (int rc = check_options(opt, CANVAS_OPT_INFERENCE, flags)) return rc;
        if (rows < 1 || features < 1 || width < 1) return set_last_error(CANVAS_BAD_ARG, "every size must be at least 1");
        if (rows > INT32_MAX || features > CANVAS_GATED_MAX_SIDE || width > CANVAS_GATED_MAX_SIDE) return set_last_error(CANVAS_UNSUPPORTED, "too many rows, features or results");
        auto h = std::make_unique<canvas_gated>();
        canvas::gated::Shape& s = h->s;
        s.rows = rows;
        s.features = features;
        s.width = width;
        s.f32 = dt == CANVAS_F32;
        s.act = act;
        s.inference = (flags & CANVAS_OPT_INFERENCE) != 0;
        h->plan = canvas::gated::plan_of(s);
        if (h->plan.most_tiles > canvas::most_workgroups(512)) return set_last_error(CANVAS_UNSUPPORTED, "too many tiles of results for one launch");
        canvas_gated_info& I = h->info;
        I.n_launches_fwd = h->plan.launches_fwd;
        I.n_launches_bwd = h->plan.launches_bwd;
        I.workspace_bytes = h->plan.workspace_bytes;
        const double t = (double)rows, c = (double)features, f = (double)width, e = s.f32 ? 4 : 2;
        I.flops_fwd = 4 * t * c * f;
        I.min_bytes_fwd = e * (t * c + 2 * f * c + t * f);
        if (!s.inference) {
            I.flops_bwd = 8 * t * c * f;
            I.min_bytes_bwd = e * (2 * t * c + 4 * f * c + t * f);
        }
        *out = h.release();
        return CANVAS_OK;
    });
}

int canvas_gated_query(const canvas_gated* gated, canvas_gated_info* info) {
    if (!gated || !info) return set_last_error(CANVAS_BAD_ARG, "null argument");
    *info = gated->info;
    return CANVAS_OK;
}

int canvas_gated_forward(canvas_gated* gated, const void* x, const void* w_gate, const void* w_up, void* y, void* workspace, size_t workspace_bytes,
                         void* stream) {
    return guarded([&]() -> int {
        if (!gated) return set_last_error(CANVAS_BAD_ARG, "null gated handle");
        int rc;
        if ((rc = need(x, "x")) || (rc = need(w_gate, "w_gate")) || (rc = need(w_up, "w_up")) || (rc = need(y, "y"))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, gated->plan.workspace_bytes))) return rc;
        const canvas::gated::Shape& s = gated->s;
        const uint64_t e = s.f32 ? 4 : 2, nx = e * s.rows * s.features, nw = e * s.width * s.features, ny = e * s.rows * s.width;
        rc = check_apart({{"y", y, ny}, {"workspace", workspace, gated->plan.workspace_bytes}}, {{"x", x, nx}, {"w_gate", w_gate, nw}, {"w_up", w_up, nw}});
        if (rc) return rc;
        const canvas::gated::Fwd a{x, w_gate, w_up, y, static_cast<char*>(workspace)};
        (void)hipGetLastError();
        canvas::gated::forward(s, gated->plan, a, (hipStream_t)stream);
        return launched();
    });
}

int canvas_gated_backward(canvas_gated* gated, const void* x, const void* w_gate, const void* w_up, const void* dy, void* dx, void* dw_gate, void* dw_up,
                          void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!gated) return set_last_error(CANVAS_BAD_ARG, "null gated handle");
        const canvas::gated::Shape& s = gated->s;
        if (s.inference) return set_last_error(CANVAS_UNSUPPORTED, "this plan was compiled for inference: it has no backward pass");
        int rc;
        if ((rc = need(x, "x")) || (rc = need(w_gate, "w_gate")) || (rc = need(w_up, "w_up")) || (rc = need(dy, "dy"))) return rc;
        if ((rc = need(dx, "dx")) || (rc = need(dw_gate, "dw_gate")) || (rc = need(dw_up, "dw_up"))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, gated->plan.workspace_bytes))) return rc;
        const uint64_t e = s.f32 ? 4 : 2, nx = e * s.rows * s.features, nw = e * s.width * s.features, ny = e * s.rows * s.width;
        rc = check_apart({{"dx", dx, nx}, {"dw_gate", dw_gate, nw}, {"dw_up", dw_up, nw}, {"workspace", workspace, gated->plan.workspace_bytes}},
                         {{"x", x, nx}, {"w_gate", w_gate, nw}, {"w_up", w_up, nw}, {"dy", dy, ny}});
        if (rc) return rc;
        const canvas::gated::Bwd a{x, w_gate, w_up, dy, dx, dw_gate, dw_up, static_cast<char*>(workspace)};
        (void)hipGetLastError();
        canvas::gated::backward(s, gated->plan, a, (hipStream_t)stream);
        return launched();
    });
}

void canvas_gated_destroy(canvas_gated* gated) { delete gated; }

}  // extern "C"
