// Host-side helpers of the C entry points (defined in qnn_api.cpp).
#pragma once

#include "qnn.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qnn {

// Records the message of a status other than QNN_OK and returns it.
qnn_status fail(qnn_status s, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
qnn_status hip_fail(hipError_t e, const char *what);

#define HIP_TRY(expr)                                 \
    do {                                              \
        hipError_t e_ = (expr);                       \
        if (e_ != hipSuccess)                         \
            return hip_fail(e_, #expr);               \
    } while (0)

struct Range {
    int64_t lo, hi;
};
bool dtype_range(qnn_dtype t, Range *r);   // false: not an integer dtype
const char *dtype_name(qnn_dtype t);
qnn_status check_qparams(const qnn_qparams &q, const char *what, int32_t n_allowed, qnn_dtype zp_dtype,
                         bool allow_zero_scale);
qnn_status out_bounds(qnn_dtype yt, qnn_clamp act, int32_t *lo, int32_t *hi);
int device_cus();

}  // namespace qnn
