// What the entry points of the C ABI share: the error message, checks of pointers and options, the status of launches.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <exception>
#include <string>

#include "../../include/canvas_dag.h"

namespace canvas {

int set_last_error(int code, const std::string& msg);  // api.cpp

namespace abi {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// CANVAS_OK, or BAD_ARG with a message that names the pointer.
inline int need(const void* p, const char* name) {
    if (p && aligned16(p)) return CANVAS_OK;
    return set_last_error(CANVAS_BAD_ARG, std::string(name) + " must be a non-null, 16-byte aligned device pointer");
}

inline int check_options(const canvas_options* opt, uint32_t known, uint32_t& flags) {
    flags = 0;
    if (!opt) return CANVAS_OK;
    for (uint32_t r : opt->reserved)
        if (r) return set_last_error(CANVAS_BAD_ARG, "reserved option fields must be zero");
    if (opt->flags & ~known) return set_last_error(CANVAS_BAD_ARG, "unknown option flag");
    flags = opt->flags;
    return CANVAS_OK;
}

inline int check_workspace(const void* ws, size_t have, uint64_t want) {
    if (have < want) return set_last_error(CANVAS_WORKSPACE_TOO_SMALL, "workspace smaller than workspace_bytes");
    return want ? need(ws, "workspace") : CANVAS_OK;
}

inline int launched() {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_last_error(CANVAS_HIP_ERROR, std::string("kernel launch failed: ") + hipGetErrorString(e));
    return CANVAS_OK;
}

// The body of an entry point: no exception crosses the C boundary.
template <class F>
int guarded(F body) {
    try {
        return body();
    } catch (const std::exception& e) {
        return set_last_error(CANVAS_UNSUPPORTED, std::string("call failed: ") + e.what());
    }
}

}  // namespace abi
}  // namespace canvas
