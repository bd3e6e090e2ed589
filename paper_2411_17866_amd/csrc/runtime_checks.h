// What the operators' host runtimes check alike: errors by status and message,
// alignment, the caller's workspace.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "dsm.h"
#include "thread_error.h"

namespace dsm {

__attribute__((format(printf, 2, 3))) inline dsm_status bad(dsm_status st, const char* fmt, ...) {
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    return set_thread_error(st, msg);
}

inline dsm_status invalid(const char* what) { return bad(DSM_ERR_INVALID_ARG, "%s", what); }

inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

inline dsm_status check_device() {
    int n = 0;
    if (hipGetDeviceCount(&n) != hipSuccess || n < 1) return bad(DSM_ERR_HIP, "no HIP device");
    return DSM_OK;
}

inline dsm_status launched(const char* what, hipError_t e) {
    if (e == hipSuccess) return DSM_OK;
    return bad(DSM_ERR_HIP, "%s: %s (%d)", what, hipGetErrorString(e), static_cast<int>(e));
}

inline dsm_status check_workspace(const void* ws, int64_t bytes, int64_t need) {
    if (!ws) return invalid("workspace is NULL");
    if (!aligned(ws, 256)) return invalid("workspace is not 256-byte aligned");
    if (bytes < need)
        return bad(DSM_ERR_INVALID_ARG, "workspace_bytes %lld < %lld", static_cast<long long>(bytes),
                   static_cast<long long>(need));
    return DSM_OK;
}

}  // namespace dsm
