// Status codes, error texts and argument checks that the C ABI's translation
// units share.
#pragma once

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <string>

#include "rsc.h"

namespace rsc {
namespace api {

inline thread_local std::string g_err;

inline rsc_status_t fail(rsc_status_t s, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    g_err = buf;
    return s;
}

inline rsc_status_t hip_fail(hipError_t e, const char *what) {
    return fail(RSC_ERR_HIP, "%s: %s (%s)", what, hipGetErrorName(e), hipGetErrorString(e));
}

#define RSC_TRY(expr)                     \
    do {                                  \
        rsc_status_t _s = (expr);         \
        if (_s != RSC_OK) return _s;      \
    } while (0)

#define RSC_HIP(expr, what)                         \
    do {                                            \
        hipError_t _e = (expr);                     \
        if (_e != hipSuccess) return hip_fail(_e, what); \
    } while (0)

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline rsc_status_t check_device() {
    static const int count = [] {  // counted once, thread-safe initialisation
        int c = 0;
        if (hipGetDeviceCount(&c) != hipSuccess) c = 0;
        return c;
    }();
    if (count <= 0) return fail(RSC_ERR_NO_DEVICE, "no HIP device visible");
    return RSC_OK;
}

inline rsc_status_t check_ws(const void *ws, size_t ws_bytes, size_t need, const char *what) {
    if (ws_bytes < need)
        return fail(RSC_ERR_CAPACITY, "%s workspace: %zu bytes given, %zu needed", what, ws_bytes, need);
    if (need > 0 && !ws) return fail(RSC_ERR_INVALID_ARGUMENT, "%s workspace is NULL", what);
    if (!aligned(ws, 256)) return fail(RSC_ERR_UNSUPPORTED, "%s workspace is not 256-byte aligned", what);
    return RSC_OK;
}

}  // namespace api
}  // namespace rsc
