// Argument checks that the C entry points of the recurrences, the linear layer and the block operators share.
#pragma once
#include "sdm_internal.h"

#include <limits.h>
#include <stdarg.h>
#include <stdio.h>

namespace {

sdm_status fail(sdm_status st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return sdm::api_error(st, buf);
}

#define SDM_TRY(expr)                  \
    do {                               \
        sdm_status _st = (expr);       \
        if (_st != SDM_OK) return _st; \
    } while (0)

struct Buf {
    const char* name;
    const void* p;
    size_t bytes;
    size_t align;
    bool optional;
    bool written;
};

// Presence, alignment, and that nothing written overlaps anything else (but b[in] and b[out], unless negative, may be
// one buffer).
sdm_status check_bufs(const char* who, const Buf* b, int n, int in = -1, int out = -1) {
    for (int i = 0; i < n; ++i) {
        if (b[i].p == nullptr && !b[i].optional && b[i].bytes > 0) return fail(SDM_ERR_INVALID_ARG, "%s: %s is NULL", who, b[i].name);
        if (reinterpret_cast<uintptr_t>(b[i].p) % b[i].align != 0)
            return fail(SDM_ERR_INVALID_ARG, "%s: %s is not %zu-byte aligned", who, b[i].name, b[i].align);
    }
    for (int i = 0; i < n; ++i) {
        if (!b[i].written || b[i].p == nullptr || b[i].bytes == 0) continue;
        for (int j = 0; j < n; ++j) {
            if (j == i || b[j].p == nullptr || b[j].bytes == 0) continue;
            const uintptr_t x = reinterpret_cast<uintptr_t>(b[i].p), y = reinterpret_cast<uintptr_t>(b[j].p);
            if (i == out && j == in && b[i].p == b[j].p && b[i].bytes == b[j].bytes) continue;
            if (x < y + b[j].bytes && y < x + b[i].bytes)
                return fail(SDM_ERR_INVALID_ARG, "%s: %s overlaps %s", who, b[i].name, b[j].name);
        }
    }
    return SDM_OK;
}

sdm_status check_ws(const char* who, const void* ws, size_t have, size_t need) {
    if (need == 0) return SDM_OK;
    if (ws == nullptr) return fail(SDM_ERR_INVALID_ARG, "%s: workspace is NULL (need %zu bytes)", who, need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return fail(SDM_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
    if (have < need) return fail(SDM_ERR_INVALID_ARG, "%s: workspace too small (%zu < %zu bytes)", who, have, need);
    return SDM_OK;
}

sdm_status done(cudaError_t e, const char* who) {
    if (e == cudaErrorInvalidConfiguration)
        return fail(SDM_ERR_CUDA, "%s: %s (%s): a launch is out of range, or a kernel was compiled to another number of registers than the split "
                    "among its warps needs", who, cudaGetErrorString(e), cudaGetErrorName(e));
    if (e != cudaSuccess) return fail(SDM_ERR_CUDA, "%s: %s (%s)", who, cudaGetErrorString(e), cudaGetErrorName(e));
    return sdm::api_ok();
}

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
size_t esize(int dtype) { return dtype == SDM_F32 ? 4 : 2; }

}  // namespace
