// Error reporting and argument checks shared by the entry points.
#pragma once

#include <hip/hip_runtime.h>

#include "internal.h"
#include "proxyattn.h"

namespace pa {

// Sets the calling thread's error text and returns code.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char* where);
void clear_error();

// A device pointer that a call needs: not NULL, 16-byte aligned.
int check_ptr(const void* p, const char* name);

// Validates the descriptor and resolves it into a Shape.
int resolve(const proxyattn_problem* p, Shape* sh);

#define PA_TRY(expr)                         \
    do {                                     \
        const int rc_ = (expr);              \
        if (rc_ != PROXYATTN_OK) return rc_; \
    } while (0)

#define PA_LAUNCH(expr, where)                        \
    do {                                              \
        const hipError_t e_ = (expr);                 \
        if (e_ != hipSuccess) return hip_fail(e_, where); \
    } while (0)

}  // namespace pa
