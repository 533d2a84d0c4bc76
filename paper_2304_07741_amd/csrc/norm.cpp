// C ABI of the residual norm (include/canvas_norm.h): checks, workspace, launches.
#include "../../include/canvas_norm.h"

#include <cmath>
#include <memory>

#include "abi.hpp"
#include "norm_kernels.hpp"

struct canvas_norm {
    canvas::norm::Shape s;
    canvas::norm::Plan plan;
    bool inference = false;
    canvas_norm_info info{};
    uint64_t r1_at = 0, partial_at = 0;  // bytes into the workspace; r2 is at its beginning
};

namespace {
using canvas::set_last_error;
using namespace canvas::abi;

uint64_t up256(uint64_t v) { return (v + 255) & ~(uint64_t)255; }
uint64_t map_bytes(const canvas::norm::Shape& s) { return (s.bf16 ? 2ull : 4ull) * s.N * s.C * s.P; }

int check_weights(const canvas_norm* h, const void* z, const void* gate, const float* w_post, const float* scale, const float* w_pre) {
    int rc = CANVAS_OK;
    if (h->s.post) {
        if ((rc = need(z, "z")) || (rc = need(w_post, "w_post")) || (rc = need(scale, "scale"))) return rc;
        if (h->s.gate && (rc = need(gate, "gate"))) return rc;
    }
    return h->s.pre ? need(w_pre, "w_pre") : rc;
}
}  // namespace

extern "C" {

int canvas_norm_compile(const int64_t shape[4], canvas_dtype dt, uint32_t parts, canvas_gate gate, float eps, const canvas_options* opt,
                        canvas_norm** out) {
    return guarded([&]() -> int {
        if (!out) return set_last_error(CANVAS_BAD_ARG, "null output handle");
        *out = nullptr;
        if (!shape) return set_last_error(CANVAS_BAD_ARG, "null shape");
        if (dt != CANVAS_F32 && dt != CANVAS_BF16) return set_last_error(CANVAS_BAD_ARG, "unknown dtype");
        uint32_t flags = 0;
        if (int rc = check_options(opt, CANVAS_OPT_INFERENCE, flags)) return rc;
        if (!parts || (parts & ~(CANVAS_NORM_POST | CANVAS_NORM_PRE))) return set_last_error(CANVAS_BAD_ARG, "parts must be CANVAS_NORM_POST, CANVAS_NORM_PRE or both");
        if (gate != CANVAS_GATE_NONE && gate != CANVAS_GATE_SIGMOID && gate != CANVAS_GATE_SILU) return set_last_error(CANVAS_BAD_ARG, "unknown gate");
        if (gate != CANVAS_GATE_NONE && !(parts & CANVAS_NORM_POST)) return set_last_error(CANVAS_BAD_ARG, "a gate needs CANVAS_NORM_POST");
        if (!(eps > 0.f) || !std::isfinite(eps)) return set_last_error(CANVAS_BAD_ARG, "eps must be finite and positive");
        for (int i = 0; i < 4; i++)
            if (shape[i] < 1) return set_last_error(CANVAS_BAD_ARG, "every size must be at least 1");
        if (shape[1] > CANVAS_NORM_MAX_CHANNELS) return set_last_error(CANVAS_UNSUPPORTED, "too many channels");
        const int64_t most = INT32_MAX;
        if (shape[0] > most || shape[2] > most || shape[3] > most || shape[2] * shape[3] > most || shape[0] > most / (shape[2] * shape[3]))
            return set_last_error(CANVAS_UNSUPPORTED, "N * H * W must be below 2^31");
        auto h = std::make_unique<canvas_norm>();
        canvas::norm::Shape& s = h->s;
        s.N = shape[0];
        s.C = (int)shape[1];
        s.P = shape[2] * shape[3];
        s.bf16 = dt == CANVAS_BF16;
        s.post = (parts & CANVAS_NORM_POST) != 0;
        s.pre = (parts & CANVAS_NORM_PRE) != 0;
        s.gate = (int)gate;
        s.eps = eps;
        while (s.down * s.down * s.C > 1.f) s.down *= 0.5f;
        h->inference = (flags & CANVAS_OPT_INFERENCE) != 0;
        h->plan = canvas::norm::plan_of(s);
        canvas_norm_info& I = h->info;
        const uint64_t stat = up256(4ull * s.N * s.P);
        h->r1_at = s.post ? stat : 0;
        h->partial_at = h->r1_at + (s.pre ? stat : 0);
        I.workspace_bytes = h->inference ? 0 : h->partial_at + 8ull * h->plan.partials * s.C;
        I.n_launches_fwd = 1;
        I.n_launches_bwd = h->inference ? 0 : 2;
        const double map = (s.bf16 ? 2.0 : 4.0) * s.N * s.C * s.P, gates = gate ? 1 : 0;
        I.min_bytes_fwd = map * (1 + (s.post ? 2 + gates : 0) + (s.pre ? 1 : 0));
        I.min_bytes_bwd = map * (1 + (s.post ? 2 + 2 * gates : 0) + (s.pre ? 3 : 0));
        *out = h.release();
        return CANVAS_OK;
    });
}

int canvas_norm_query(const canvas_norm* norm, canvas_norm_info* info) {
    if (!norm || !info) return set_last_error(CANVAS_BAD_ARG, "null argument");
    *info = norm->info;
    return CANVAS_OK;
}

int canvas_norm_forward(canvas_norm* norm, const void* x, const void* z, const void* gate, const float* w_post, const float* scale,
                        const float* w_pre, void* x_out, void* u, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!norm) return set_last_error(CANVAS_BAD_ARG, "null norm handle");
        int rc = need(x, "x");
        if (rc || (rc = check_weights(norm, z, gate, w_post, scale, w_pre))) return rc;
        if (norm->s.post && (rc = need(x_out, "x_out"))) return rc;
        if (norm->s.pre && (rc = need(u, "u"))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, norm->info.workspace_bytes))) return rc;
        const canvas::norm::Shape& s = norm->s;
        const uint64_t map = map_bytes(s), vec = 4ull * s.C;
        rc = check_apart({{"x_out", s.post ? x_out : nullptr, map}, {"u", s.pre ? u : nullptr, map}, {"workspace", norm->inference ? nullptr : workspace, norm->info.workspace_bytes}},
                         {{"x", x, map},
                          {"z", s.post ? z : nullptr, map},
                          {"gate", s.gate ? gate : nullptr, map},
                          {"w_post", s.post ? w_post : nullptr, vec},
                          {"scale", s.post ? scale : nullptr, vec},
                          {"w_pre", s.pre ? w_pre : nullptr, vec}});
        if (rc) return rc;
        char* ws = static_cast<char*>(workspace);
        canvas::norm::Fwd a{x, z, gate, w_post, scale, w_pre, x_out, u, nullptr, nullptr};
        if (!norm->inference) {
            a.r2 = reinterpret_cast<float*>(ws);
            a.r1 = reinterpret_cast<float*>(ws + norm->r1_at);
        }
        (void)hipGetLastError();
        canvas::norm::forward(norm->s, norm->plan, a, (hipStream_t)stream);
        return launched();
    });
}

int canvas_norm_backward(canvas_norm* norm, const void* x, const void* z, const void* gate, const float* w_post, const float* scale,
                         const float* w_pre, const void* dx_out, const void* du, void* dx, void* dz, void* dgate, float* dw_post, float* dscale,
                         float* dw_pre, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!norm) return set_last_error(CANVAS_BAD_ARG, "null norm handle");
        if (norm->inference) return set_last_error(CANVAS_UNSUPPORTED, "this plan was compiled for inference: it has no backward pass");
        const canvas::norm::Shape& s = norm->s;
        int rc = check_weights(norm, z, gate, w_post, scale, w_pre);
        if (rc) return rc;
        if (s.post && ((rc = need(dz, "dz")) || (rc = need(dw_post, "dw_post")) || (rc = need(dscale, "dscale")))) return rc;
        if (s.gate && (rc = need(dgate, "dgate"))) return rc;
        if (s.pre && ((rc = need(x, "x")) || (rc = need(du, "du")) || (rc = need(dx, "dx")) || (rc = need(dw_pre, "dw_pre")))) return rc;
        if ((dx_out || !s.pre) && (rc = need(dx_out, "dx_out"))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, norm->info.workspace_bytes))) return rc;
        const uint64_t map = map_bytes(s), vec = 4ull * s.C;
        rc = check_apart({{"dx", s.pre ? dx : nullptr, map},
                          {"dz", s.post ? dz : nullptr, map},
                          {"dgate", s.gate ? dgate : nullptr, map},
                          {"dw_post", s.post ? dw_post : nullptr, vec},
                          {"dscale", s.post ? dscale : nullptr, vec},
                          {"dw_pre", s.pre ? dw_pre : nullptr, vec},
                          {"workspace", workspace, norm->info.workspace_bytes}},
                         {{"x", s.pre ? x : nullptr, map},
                          {"z", s.post ? z : nullptr, map},
                          {"gate", s.gate ? gate : nullptr, map},
                          {"w_post", s.post ? w_post : nullptr, vec},
                          {"scale", s.post ? scale : nullptr, vec},
                          {"w_pre", s.pre ? w_pre : nullptr, vec},
                          {"dx_out", dx_out, map},
                          {"du", s.pre ? du : nullptr, map}});
        if (rc) return rc;
        char* ws = static_cast<char*>(workspace);
        const canvas::norm::Bwd a{x, z, gate, w_post, scale, w_pre, dx_out, du, dx, dz, dgate, dw_post, dscale, dw_pre, reinterpret_cast<float*>(ws),
                                  reinterpret_cast<float*>(ws + norm->r1_at), reinterpret_cast<float*>(ws + norm->partial_at)};
        (void)hipGetLastError();
        canvas::norm::backward(s, norm->plan, a, (hipStream_t)stream);
        return launched();
    });
}

void canvas_norm_destroy(canvas_norm* norm) { delete norm; }

}  // extern "C"
