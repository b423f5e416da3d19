// What the entry points share: the text of a failing call and checks of arguments.
#pragma once

#include <cstdarg>
#include <cstdio>

#include "common.h"

namespace uncomp {

inline uncomp_status fail(uncomp_ctx* ctx, uncomp_status st, const char* fmt, ...) {
    if (ctx != nullptr) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap);
        va_end(ap);
    }
    return st;
}

inline uncomp_status hip_fail(uncomp_ctx* ctx, hipError_t e, const char* what) {
    return fail(ctx, UNCOMP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace uncomp
