// C ABI of the clipping of gradients (include/canvas_clip.h): checks, workspace, launches.
#include "../../include/canvas_clip.h"

#include <algorithm>
#include <cmath>
#include <memory>
#include <vector>

#include "abi.hpp"
#include "clip_kernels.hpp"

struct canvas_clip {
    canvas::clip::Plan plan;
    canvas_clip_info info{};
};

namespace {
using canvas::set_last_error;
using namespace canvas::abi;

uint64_t size_of(bool bf16) { return bf16 ? 2 : 4; }

int check_tensor(const void* p, bool bf16, const char* what, size_t i) {
    if (p && (reinterpret_cast<uintptr_t>(p) & (size_of(bf16) - 1)) == 0) return CANVAS_OK;
    return set_last_error(CANVAS_BAD_ARG, std::string(what) + " " + std::to_string(i) + " must be a non-null device pointer, aligned to its element");
}

// Bytes that a call reads or writes.
struct Span {
    uint64_t from, to;
    bool written;
};
// BAD_ARG if bytes that are written are written or read as something else too: sorted by where they begin, a span shares bytes with what reaches
// beyond its beginning, of which the written one and the read one that reach furthest are kept.
int check_spans(std::vector<Span>& spans) {
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    uint64_t read_to = 0, written_to = 0;
    for (const Span& s : spans) {
        if (s.from == s.to) continue;
        if (s.from < written_to || (s.written && s.from < read_to)) return set_last_error(CANVAS_BAD_ARG, "what the call writes shares bytes with something else that it reads or writes");
        (s.written ? written_to : read_to) = std::max(s.written ? written_to : read_to, s.to);
    }
    return CANVAS_OK;
}
}  // namespace

extern "C" {

int canvas_clip_compile(int32_t tensors, const int64_t* counts, const canvas_dtype* types, const canvas_dtype* out_types, canvas_clip** out) {
    return guarded([&]() -> int {
        if (!out) return set_last_error(CANVAS_BAD_ARG, "null output handle");
        *out = nullptr;
        if (!counts || !types) return set_last_error(CANVAS_BAD_ARG, "null counts or types");
        if (tensors < 1) return set_last_error(CANVAS_BAD_ARG, "at least one tensor is needed");
        if (tensors > CANVAS_CLIP_MAX_TENSORS) return set_last_error(CANVAS_UNSUPPORTED, "too many tensors");
        auto h = std::make_unique<canvas_clip>();
        int64_t all = 0;
        double bytes = 0;
        for (int i = 0; i < tensors; i++) {
            const canvas_dtype o = out_types ? out_types[i] : types[i];
            for (canvas_dtype t : {types[i], o})
                if (t != CANVAS_F32 && t != CANVAS_BF16) return set_last_error(CANVAS_BAD_ARG, "unknown dtype");
            if (counts[i] < 0) return set_last_error(CANVAS_BAD_ARG, "a count must not be negative");
            if (counts[i] > (int64_t)1 << 40) return set_last_error(CANVAS_UNSUPPORTED, "too many elements");
            all += counts[i];
            canvas::clip::Tensor t;
            t.count = counts[i];
            t.bf16 = types[i] == CANVAS_BF16;
            t.out_bf16 = o == CANVAS_BF16;
            bytes += (double)t.count * (size_of(t.bf16) + size_of(t.out_bf16));
            h->plan.tensors.push_back(t);
        }
        if (all >= (int64_t)1 << 44) return set_last_error(CANVAS_UNSUPPORTED, "too many elements");
        canvas::clip::make_plan(h->plan);
        h->info.n_launches = h->plan.launches;
        h->info.n_launches_norm = h->plan.launches_norm;
        h->info.workspace_bytes = h->plan.workspace_bytes;
        h->info.min_bytes = bytes;
        *out = h.release();
        return CANVAS_OK;
    });
}

int canvas_clip_query(const canvas_clip* clip, canvas_clip_info* info) {
    if (!clip || !info) return set_last_error(CANVAS_BAD_ARG, "null argument");
    *info = clip->info;
    return CANVAS_OK;
}

int canvas_clip_step(canvas_clip* clip, const void* const* grads, void* const* outs, double max_norm, float* norm, float* scale, void* workspace,
                     size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (!clip) return set_last_error(CANVAS_BAD_ARG, "null clip handle");
        if (!grads) return set_last_error(CANVAS_BAD_ARG, "null grads");
        if (!(max_norm > 0)) return set_last_error(CANVAS_BAD_ARG, "max_norm must be positive");
        int rc = CANVAS_OK;
        auto place = [&](float* p, const char* name) {
            return p && (reinterpret_cast<uintptr_t>(p) & 3) == 0 ? CANVAS_OK : set_last_error(CANVAS_BAD_ARG, std::string(name) + " must be a non-null device pointer, aligned to its element");
        };
        if ((rc = place(norm, "norm")) || (scale && (rc = place(scale, "scale")))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, clip->plan.workspace_bytes))) return rc;
        auto at = [](const void* p) { return (uint64_t)reinterpret_cast<uintptr_t>(p); };
        std::vector<Span> spans;
        spans.push_back(Span{at(norm), at(norm) + 4, true});
        if (scale) spans.push_back(Span{at(scale), at(scale) + 4, true});
        spans.push_back(Span{at(workspace), at(workspace) + clip->plan.workspace_bytes, true});
        for (size_t i = 0; i < clip->plan.tensors.size(); i++) {
            const canvas::clip::Tensor& t = clip->plan.tensors[i];
            if (!t.count) continue;
            if ((rc = check_tensor(grads[i], t.bf16, "gradient", i))) return rc;
            if (outs && (rc = check_tensor(outs[i], t.out_bf16, "out", i))) return rc;
            const bool same = outs && outs[i] == grads[i];
            if (same && t.bf16 != t.out_bf16) return set_last_error(CANVAS_BAD_ARG, "out " + std::to_string(i) + " in the place of its gradient needs the same type");
            if (!same) spans.push_back(Span{at(grads[i]), at(grads[i]) + t.count * size_of(t.bf16), false});
            if (outs) spans.push_back(Span{at(outs[i]), at(outs[i]) + t.count * size_of(t.out_bf16), true});
        }
        if ((rc = check_spans(spans))) return rc;
        const canvas::clip::Args a{grads, outs, max_norm, norm, scale, static_cast<char*>(workspace)};
        (void)hipGetLastError();
        canvas::clip::step(clip->plan, a, (hipStream_t)stream);
        return launched();
    });
}

void canvas_clip_destroy(canvas_clip* clip) { delete clip; }

}  // extern "C"
