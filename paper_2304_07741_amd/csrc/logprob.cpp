// C ABI of the token log probabilities (include/canvas_logprob.h): checks, workspace, launches.
#include "../../include/canvas_logprob.h"

#include <cmath>
#include <memory>

#include "abi.hpp"
#include "logprob_kernels.hpp"

struct canvas_logprob {
    canvas::logprob::Shape s;
    canvas::logprob::Plan plan;
    bool inference = false;
    canvas_logprob_info info{};
};

namespace {
using canvas::set_last_error;
using namespace canvas::abi;

int check_rows(const canvas_logprob* h, const void* p, int64_t pitch, const char* name) {
    const uintptr_t e = h->s.bf16 ? 2 : 4;
    if (!p || (reinterpret_cast<uintptr_t>(p) & (e - 1)))
        return set_last_error(CANVAS_BAD_ARG, std::string(name) + " must be a non-null device pointer, aligned to its element");
    if (pitch < h->s.classes) return set_last_error(CANVAS_BAD_ARG, std::string("the pitch of ") + name + " is less than a row");
    if (pitch > INT64_MAX / 4 / h->s.rows) return set_last_error(CANVAS_BAD_ARG, std::string("the pitch of ") + name + " is out of range");
    return CANVAS_OK;
}

Region rows_of(const canvas_logprob* h, const char* name, const void* p, int64_t pitch) {
    const uint64_t e = h->s.bf16 ? 2 : 4;
    return Region{name, p, e * h->s.classes, (uint64_t)h->s.rows, e * pitch};
}
Region mask_of(const canvas_logprob* h, const uint8_t* mask, int64_t mask_pitch) {
    return Region{"mask", mask, (uint64_t)h->s.classes, mask_pitch ? (uint64_t)h->s.rows : 1, (uint64_t)mask_pitch};
}

int check_call(const canvas_logprob* h, const void* logits, int64_t pitch, float it, const uint8_t* mask, int64_t mask_pitch) {
    if (int rc = check_rows(h, logits, pitch, "logits")) return rc;
    if (!(it > 0.f) || !std::isfinite(it)) return set_last_error(CANVAS_BAD_ARG, "inv_temperature must be finite and positive");
    if (mask && mask_pitch != 0 && (mask_pitch < h->s.classes || mask_pitch > INT64_MAX / h->s.rows))
        return set_last_error(CANVAS_BAD_ARG, "mask_pitch must be 0 or at least a row");
    return CANVAS_OK;
}
}  // namespace

extern "C" {

int canvas_logprob_compile(int64_t rows, int64_t classes, canvas_dtype dt, int32_t top_k, const canvas_options* opt, canvas_logprob** out) {
    return guarded([&]() -> int {
        if (!out) return set_last_error(CANVAS_BAD_ARG, "null output handle");
        *out = nullptr;
        if (dt != CANVAS_F32 && dt != CANVAS_BF16) return set_last_error(CANVAS_BAD_ARG, "unknown dtype");
        uint32_t flags = 0;
        if (int rc = check_options(opt, CANVAS_OPT_INFERENCE, flags)) return rc;
        if (rows < 1 || classes < 1) return set_last_error(CANVAS_BAD_ARG, "rows and classes must be at least 1");
        if (rows > INT32_MAX || classes > CANVAS_LOGPROB_MAX_CLASSES) return set_last_error(CANVAS_UNSUPPORTED, "too many rows or classes");
        if (top_k < 0 || top_k > CANVAS_LOGPROB_MAX_TOP) return set_last_error(CANVAS_BAD_ARG, "top_k out of range");
        auto h = std::make_unique<canvas_logprob>();
        h->s.rows = rows;
        h->s.classes = classes;
        h->s.bf16 = dt == CANVAS_BF16;
        h->s.top = top_k;
        h->inference = (flags & CANVAS_OPT_INFERENCE) != 0;
        h->plan = canvas::logprob::plan_of(h->s);
        canvas_logprob_info& I = h->info;
        I.n_launches_fwd = h->plan.launches_fwd;
        I.n_launches_bwd = h->inference ? 0 : 1;
        I.workspace_bytes = h->plan.workspace_bytes;
        const double n = (h->s.bf16 ? 2.0 : 4.0) * rows * classes;
        I.min_bytes_fwd = n + rows * (16.0 + 8.0 * top_k);
        I.min_bytes_bwd = 2 * n + rows * 16.0;
        *out = h.release();
        return CANVAS_OK;
    });
}

int canvas_logprob_query(const canvas_logprob* lp, canvas_logprob_info* info) {
    if (!lp || !info) return set_last_error(CANVAS_BAD_ARG, "null argument");
    *info = lp->info;
    return CANVAS_OK;
}

int canvas_logprob_forward(canvas_logprob* lp, const void* logits, int64_t pitch, float inv_temperature, const uint8_t* mask, int64_t mask_pitch,
                           const int64_t* tokens, float* logprob, float* entropy, float* top_logprob, int32_t* top_index, void* workspace,
                           size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!lp) return set_last_error(CANVAS_BAD_ARG, "null logprob handle");
        int rc = check_call(lp, logits, pitch, inv_temperature, mask, mask_pitch);
        if (rc) return rc;
        if ((tokens || logprob) && ((rc = need(tokens, "tokens")) || (rc = need(logprob, "logprob")))) return rc;
        if (entropy && (rc = need(entropy, "entropy"))) return rc;
        if (lp->s.top > 0 && ((rc = need(top_logprob, "top_logprob")) || (rc = need(top_index, "top_index")))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, lp->plan.workspace_bytes))) return rc;
        const uint64_t n = lp->s.rows, top = lp->s.top;
        rc = check_apart({{"logprob", logprob, 4 * n},
                          {"entropy", entropy, 4 * n},
                          {"top_logprob", top ? top_logprob : nullptr, 4 * n * top},
                          {"top_index", top ? top_index : nullptr, 4 * n * top},
                          {"workspace", workspace, lp->plan.workspace_bytes}},
                         {rows_of(lp, "logits", logits, pitch), mask_of(lp, mask, mask_pitch), {"tokens", tokens, 8 * n}});
        if (rc) return rc;
        const canvas::logprob::Fwd a{logits, pitch, inv_temperature, mask, mask_pitch, tokens, logprob, entropy, top_logprob, top_index,
                                     static_cast<char*>(workspace)};
        (void)hipGetLastError();
        canvas::logprob::forward(lp->s, lp->plan, a, (hipStream_t)stream);
        return launched();
    });
}

int canvas_logprob_backward(canvas_logprob* lp, const void* logits, int64_t pitch, float inv_temperature, const uint8_t* mask, int64_t mask_pitch,
                            const int64_t* tokens, const float* dlogprob, const float* dentropy, void* dlogits, int64_t dpitch, void* workspace,
                            size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!lp) return set_last_error(CANVAS_BAD_ARG, "null logprob handle");
        if (lp->inference) return set_last_error(CANVAS_UNSUPPORTED, "this plan was compiled for inference: it has no backward pass");
        int rc = check_call(lp, logits, pitch, inv_temperature, mask, mask_pitch);
        if (rc || (rc = check_rows(lp, dlogits, dpitch, "dlogits"))) return rc;
        if (dlogits == logits && dpitch != pitch) return set_last_error(CANVAS_BAD_ARG, "dlogits in the place of logits needs the same pitch");
        if ((tokens || dlogprob) && (rc = need(tokens, "tokens"))) return rc;
        if (dlogprob && (rc = need(dlogprob, "dlogprob"))) return rc;
        if (dentropy && (rc = need(dentropy, "dentropy"))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, lp->plan.workspace_bytes))) return rc;
        const uint64_t n = lp->s.rows;
        rc = check_apart({rows_of(lp, "dlogits", dlogits, dpitch)},
                         {rows_of(lp, "logits", dlogits == logits ? nullptr : logits, pitch),
                          mask_of(lp, mask, mask_pitch),
                          {"tokens", tokens, 8 * n},
                          {"dlogprob", dlogprob, 4 * n},
                          {"dentropy", dentropy, 4 * n},
                          {"workspace", workspace, lp->plan.workspace_bytes}});
        if (rc) return rc;
        const canvas::logprob::Bwd a{logits, pitch, inv_temperature, mask, mask_pitch, tokens, dlogprob, dentropy, dlogits, dpitch,
                                     static_cast<const char*>(workspace)};
        (void)hipGetLastError();
        canvas::logprob::backward(lp->s, lp->plan, a, (hipStream_t)stream);
        return launched();
    });
}

void canvas_logprob_destroy(canvas_logprob* lp) { delete lp; }

}  // extern "C"
