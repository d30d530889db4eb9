// The context behind the C ABI and how its entry points fail.
#pragma once

#include <stdarg.h>
#include <stdio.h>

#include "harp_internal.h"

struct harp_ctx {
    int device;
    int n_cu;
    int plan_path;
    harp::BuildHeader *pinned;   // host, pinned
    unsigned char *scratch;   // this device's copy of the library's static scratch array
    char err[512];
};

namespace harp {

inline int fail(harp_ctx *ctx, int code, const char *fmt, ...) {
    if (ctx) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap);
        va_end(ap);
    }
    return code;
}

inline int hip_fail(harp_ctx *ctx, hipError_t e, const char *what) {
    return fail(ctx, HARP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace harp
