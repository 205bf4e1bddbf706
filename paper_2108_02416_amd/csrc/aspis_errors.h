// aspis_errors.h -- status codes and messages of the entry points that check
// their arguments and launch (aspis_clip.cpp, aspis_tokens.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/aspis.h"

namespace aspis {
aspis_status host_fail(aspis_status st, const char *msg);   // aspis_host.cpp
void host_clear_error();

constexpr int64_t kMaxElements = int64_t(1) << 60;

__attribute__((format(printf, 2, 3))) inline aspis_status fail(aspis_status st, const char *fmt,
                                                               ...) {
    char msg[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    return host_fail(st, msg);
}

inline aspis_status launched(hipError_t e, const char *what) {
    if (e != hipSuccess)
        return fail(ASPIS_ERR_DEVICE, "%s failed: %s", what, hipGetErrorString(e));
    host_clear_error();
    return ASPIS_OK;
}

inline int elem_bytes(int dtype) {
    return dtype == ASPIS_F32 ? 4 : dtype == ASPIS_BF16 || dtype == ASPIS_F16 ? 2 : 0;
}
}  // namespace aspis
