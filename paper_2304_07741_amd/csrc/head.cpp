// C ABI of the head's log probabilities (include/canvas_head.h): checks, workspace, launches.
#include "../../include/canvas_head.h"

#include <cmath>
#include <memory>

#include "abi.hpp"
#include "head_kernels.hpp"
#include "launch.hpp"

struct canvas_head {
    canvas::head::Shape s;
    canvas::head::Plan plan;
    canvas_head_info info{};
};

namespace {
using canvas::set_last_error;
using namespace canvas::abi;

int check_call(const void* x, const void* weight, float it) {
    int rc;
    if ((rc = need(x, "x")) || (rc = need(weight, "weight"))) return rc;
    if (!(it > 0.f) || !std::isfinite(it)) return set_last_error(CANVAS_BAD_ARG, "inv_temperature must be finite and positive");
    return CANVAS_OK;
}
}  // namespace

extern "C" {

int canvas_head_compile(int64_t rows, int64_t features, int64_t classes, canvas_dtype dt, const canvas_options* opt, canvas_head** out) {
    return guarded([&]() -> int {
        if (!out) return set_last_error(CANVAS_BAD_ARG, "null output handle");
        *out = nullptr;
        if (dt != CANVAS_F32 && dt != CANVAS_BF16) return set_last_error(CANVAS_BAD_ARG, "unknown dtype");
        uint32_t flags = 0;
        if (int rc = check_options(opt, CANVAS_OPT_INFERENCE, flags)) return rc;
        if (rows < 1 || features < 1 || classes < 1) return set_last_error(CANVAS_BAD_ARG, "every size must be at least 1");
        if (rows > INT32_MAX || features > CANVAS_HEAD_MAX_FEATURES || classes > CANVAS_HEAD_MAX_CLASSES) return set_last_error(CANVAS_UNSUPPORTED, "too many rows, features or classes");
        auto h = std::make_unique<canvas_head>();
        canvas::head::Shape& s = h->s;
        s.rows = rows;
        s.features = features;
        s.classes = classes;
        s.f32 = dt == CANVAS_F32;
        s.inference = (flags & CANVAS_OPT_INFERENCE) != 0;
        h->plan = canvas::head::plan_of(s);
        if (h->plan.most_tiles > canvas::most_workgroups(512)) return set_last_error(CANVAS_UNSUPPORTED, "too many tiles of results for one launch");
        canvas_head_info& I = h->info;
        I.n_launches_fwd = h->plan.launches_fwd;
        I.n_launches_bwd = h->plan.launches_bwd;
        I.n_launches_bwd_mask = h->plan.launches_mask;
        I.pieces = s.inference ? 0 : h->plan.pieces;
        I.workspace_bytes = h->plan.workspace_bytes;
        const double t = (double)rows, c = (double)features, v = (double)classes, e = s.f32 ? 4 : 2;
        I.flops_fwd = 2 * t * c * v;
        I.min_bytes_fwd = e * (t * c + v * c) + 16 * t;
        if (!s.inference) {
            I.flops_bwd = 4 * t * c * v + 2 * t * c * (double)h->plan.again;
            I.min_bytes_bwd = 2 * e * (t * c + v * c) + 16 * t;
        }
        *out = h.release();
        return CANVAS_OK;
    });
}

int canvas_head_query(const canvas_head* head, canvas_head_info* info) {
    if (!head || !info) return set_last_error(CANVAS_BAD_ARG, "null argument");
    *info = head->info;
    return CANVAS_OK;
}

int canvas_head_forward(canvas_head* head, const void* x, const void* weight, float inv_temperature, const uint8_t* mask, const int64_t* tokens, float* logprob,
                        float* entropy, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!head) return set_last_error(CANVAS_BAD_ARG, "null head handle");
        int rc = check_call(x, weight, inv_temperature);
        if (rc) return rc;
        if (mask && (rc = need(mask, "mask"))) return rc;
        if ((tokens || logprob) && ((rc = need(tokens, "tokens")) || (rc = need(logprob, "logprob")))) return rc;
        if (entropy && (rc = need(entropy, "entropy"))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, head->plan.workspace_bytes))) return rc;
        const canvas::head::Shape& s = head->s;
        const uint64_t e = s.f32 ? 4 : 2, t = s.rows;
        rc = check_apart({{"logprob", logprob, 4 * t}, {"entropy", entropy, 4 * t}, {"workspace", workspace, head->plan.workspace_bytes}},
                         {{"x", x, e * t * s.features}, {"weight", weight, e * s.classes * s.features}, {"mask", mask, (uint64_t)s.classes}, {"tokens", tokens, 8 * t}});
        if (rc) return rc;
        const canvas::head::Fwd a{x, weight, inv_temperature, mask, tokens, logprob, entropy, static_cast<char*>(workspace)};
        (void)hipGetLastError();
        canvas::head::forward(s, head->plan, a, (hipStream_t)stream);
        return launched();
    });
}

int canvas_head_backward(canvas_head* head, const void* x, const void* weight, float inv_temperature, const uint8_t* mask, const int64_t* tokens,
                         const float* dlogprob, const float* dentropy, void* dx, void* dweight, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!head) return set_last_error(CANVAS_BAD_ARG, "null head handle");
        const canvas::head::Shape& s = head->s;
        if (s.inference) return set_last_error(CANVAS_UNSUPPORTED, "this plan was compiled for inference: it has no backward pass");
        int rc = check_call(x, weight, inv_temperature);
        if (rc) return rc;
        if (mask && (rc = need(mask, "mask"))) return rc;
        if ((tokens || dlogprob) && (rc = need(tokens, "tokens"))) return rc;
        if (dlogprob && (rc = need(dlogprob, "dlogprob"))) return rc;
        if (dentropy && (rc = need(dentropy, "dentropy"))) return rc;
        if ((rc = need(dx, "dx")) || (rc = need(dweight, "dweight"))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, head->plan.workspace_bytes))) return rc;
        const uint64_t e = s.f32 ? 4 : 2, t = s.rows, nx = e * t * s.features, nw = e * s.classes * s.features;
        rc = check_apart({{"dx", dx, nx}, {"dweight", dweight, nw}, {"workspace", workspace, head->plan.workspace_bytes}},
                         {{"x", x, nx}, {"weight", weight, nw}, {"mask", mask, (uint64_t)s.classes}, {"tokens", tokens, 8 * t}, {"dlogprob", dlogprob, 4 * t}, {"dentropy", dentropy, 4 * t}});
        if (rc) return rc;
        const canvas::head::Bwd a{x, weight, inv_temperature, mask, tokens, dlogprob, dentropy, dx, dweight, static_cast<char*>(workspace)};
        (void)hipGetLastError();
        canvas::head::backward(s, head->plan, a, (hipStream_t)stream);
        return launched();
    });
}

void canvas_head_destroy(canvas_head* head) { delete head; }

}  // extern "C"
