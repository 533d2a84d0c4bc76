// What the entry points of the C ABI share: the error message, checks of pointers and options, the status of launches.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <exception>
#include <initializer_list>
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

// A tensor of a call: rows of `bytes` bytes, `pitch` bytes from one to the next.  Null: not part of the call.
struct Region {
    const char* name;
    const void* p;
    uint64_t bytes, rows = 1, pitch = 0;
};
inline bool share_bytes(const Region& a, const Region& b) {
    if (!a.p || !b.p) return false;
    if (a.rows < b.rows) return share_bytes(b, a);
    // (unsigned: an address and 2^63 bytes behind it are below 2^64)
    const uint64_t a0 = (uint64_t)(uintptr_t)a.p, b0 = (uint64_t)(uintptr_t)b.p;
    if (a0 >= b0 + (b.rows - 1) * b.pitch + b.bytes || b0 >= a0 + (a.rows - 1) * a.pitch + a.bytes) return false;
    if (a.rows == 1) return true;
    if (b.rows > 1 && a.pitch == b.pitch) {
        // rows i of a and j of b lie as i - j says: the first difference with which a's row ends behind the beginning of b's
        const int64_t pitch = (int64_t)a.pitch, d = (int64_t)(b0 - a0), n = d - (int64_t)a.bytes;
        int64_t k = (n >= 0 ? n / pitch : -((-n + pitch - 1) / pitch)) + 1;
        if (k < 1 - (int64_t)b.rows) k = 1 - (int64_t)b.rows;
        return k < (int64_t)a.rows && k * pitch < d + (int64_t)b.bytes;
    }
    // each row of b against the first of a's rows that ends behind its beginning
    for (uint64_t r = 0; r < b.rows; r++) {
        const uint64_t from = b0 + r * b.pitch, i = a0 + a.bytes > from ? 0 : (from - a0 - a.bytes) / a.pitch + 1;
        if (i < a.rows && a0 + i * a.pitch < from + b.bytes) return true;
    }
    return false;
}
// CANVAS_OK, or BAD_ARG if what a call writes shares bytes with anything else that it writes or reads.
inline int check_apart(std::initializer_list<Region> written, std::initializer_list<Region> read) {
    auto clash = [](const Region& a, const Region& b) {
        return set_last_error(CANVAS_BAD_ARG, std::string(a.name) + " is written and shares bytes with " + b.name);
    };
    for (const Region* a = written.begin(); a != written.end(); a++) {
        for (const Region* b = a + 1; b != written.end(); b++)
            if (share_bytes(*a, *b)) return clash(*a, *b);
        for (const Region& b : read)
            if (share_bytes(*a, b)) return clash(*a, b);
    }
    return CANVAS_OK;
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
