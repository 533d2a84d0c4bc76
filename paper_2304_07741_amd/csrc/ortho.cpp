// C ABI of the orthogonalised update (include/canvas_ortho.h): checks, workspace, launches.
#include "../../include/canvas_ortho.h"

#include <algorithm>
#include <cmath>
#include <memory>

#include "abi.hpp"
#include "launch.hpp"
#include "ortho_kernels.hpp"

struct canvas_ortho {
    canvas::ortho::Shape s;
    canvas::ortho::Plan plan;
    canvas_ortho_info info{};
};

namespace {
using canvas::set_last_error;
using namespace canvas::abi;
}  // namespace

extern "C" {

int canvas_ortho_compile(const int64_t shape[3], canvas_dtype dt, int32_t steps, uint32_t flags, canvas_ortho** out) {
    return guarded([&]() -> int {
        if (!out) return set_last_error(CANVAS_BAD_ARG, "null output handle");
        *out = nullptr;
        if (!shape) return set_last_error(CANVAS_BAD_ARG, "null shape");
        if (dt != CANVAS_F32 && dt != CANVAS_BF16) return set_last_error(CANVAS_BAD_ARG, "unknown dtype");
        if (flags & ~CANVAS_ORTHO_NESTEROV) return set_last_error(CANVAS_BAD_ARG, "unknown option flag");
        if (steps < 0 || steps > CANVAS_ORTHO_MAX_STEPS) return set_last_error(CANVAS_BAD_ARG, "steps out of range");
        for (int i = 0; i < 3; i++)
            if (shape[i] < 1) return set_last_error(CANVAS_BAD_ARG, "every size must be at least 1");
        const int64_t most = INT32_MAX, G = shape[0], R = shape[1], K = shape[2];
        if (G > most || R > most || K > most || R * K > most / 2 || G > most / (R * K)) return set_last_error(CANVAS_UNSUPPORTED, "R * K must be below 2^30, G * R * K below 2^31");
        if (std::min(R, K) > CANVAS_ORTHO_MAX_SIDE || G > 65535) return set_last_error(CANVAS_UNSUPPORTED, "matrices too large or too many");
        auto h = std::make_unique<canvas_ortho>();
        canvas::ortho::Shape& s = h->s;
        s.G = G;
        s.R = R;
        s.K = K;
        s.m = std::min(R, K);
        s.n = std::max(R, K);
        s.tall = R > K;
        s.bf16 = dt == CANVAS_BF16;
        s.nesterov = (flags & CANVAS_ORTHO_NESTEROV) != 0;
        s.steps = steps;
        h->plan = canvas::ortho::plan_of(s);
        // (thin matrices with 2^30 elements and more in all, whose padded transposes would take 256 GB)
        if (h->plan.workgroups > canvas::most_workgroups(256)) return set_last_error(CANVAS_UNSUPPORTED, "matrices too large or too many for one launch");
        canvas_ortho_info& I = h->info;
        I.n_launches = h->plan.launches;
        I.workspace_bytes = h->plan.workspace_bytes;
        const double m = (double)s.m, n = (double)s.n;
        I.flops = G * (double)steps * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n);
        I.min_bytes = (double)G * R * K * (12 + (s.bf16 ? 2 : 4));
        *out = h.release();
        return CANVAS_OK;
    });
}

int canvas_ortho_query(const canvas_ortho* ortho, canvas_ortho_info* info) {
    if (!ortho || !info) return set_last_error(CANVAS_BAD_ARG, "null argument");
    *info = ortho->info;
    return CANVAS_OK;
}

int canvas_ortho_step(canvas_ortho* ortho, const float* grad, const float* momentum, float* momentum_out, double mu, const float* master,
                      float* master_out, double lr, double decay, void* weights, void* update, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!ortho) return set_last_error(CANVAS_BAD_ARG, "null ortho handle");
        int rc = need(grad, "grad");
        if (rc) return rc;
        if ((momentum || momentum_out) && ((rc = need(momentum, "momentum")) || (rc = need(momentum_out, "momentum_out")))) return rc;
        if ((master || master_out) && ((rc = need(master, "master")) || (rc = need(master_out, "master_out")))) return rc;
        if (momentum && !(mu >= 0.f && mu < 1.f)) return set_last_error(CANVAS_BAD_ARG, "mu must be in [0, 1)");
        if (master && !(std::isfinite(lr) && std::isfinite(decay))) return set_last_error(CANVAS_BAD_ARG, "lr and decay must be finite");
        if (weights && !master) return set_last_error(CANVAS_BAD_ARG, "weights need master weights");
        if (weights && (rc = need(weights, "weights"))) return rc;
        if ((update || !master) && (rc = need(update, "update"))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, ortho->plan.workspace_bytes))) return rc;
        const canvas::ortho::Shape& s = ortho->s;
        const uint64_t n = (uint64_t)(s.G * s.R * s.K), e = s.bf16 ? 2 : 4;
        rc = check_apart({{"momentum_out", momentum_out, 4 * n},
                          {"master_out", master_out, 4 * n},
                          {"weights", weights, e * n},
                          {"update", update, e * n},
                          {"workspace", workspace, ortho->plan.workspace_bytes}},
                         {{"grad", grad, 4 * n}, {"momentum", momentum == momentum_out ? nullptr : momentum, 4 * n}, {"master", master == master_out ? nullptr : master, 4 * n}});
        if (rc) return rc;
        const canvas::ortho::Args a{grad, momentum, momentum_out, mu, master, master_out, lr, decay, weights, update, static_cast<char*>(workspace)};
        (void)hipGetLastError();
        canvas::ortho::step(ortho->s, ortho->plan, a, (hipStream_t)stream);
        return launched();
    });
}

void canvas_ortho_destroy(canvas_ortho* ortho) { delete ortho; }

}  // extern "C"
