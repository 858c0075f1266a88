// The host side of the library in one translation unit: the k-means entry
// points (km_capi.hip) and, for those of km_ops.hip, their error text and device
// checks.  These stand apart because km_capi.hip configures every k-means
// kernel: counters that were measured of a kernel hold while it is unchanged.
#include "km_capi.hip"

#include <stdarg.h>

#include "km_ops.h"

namespace km {

int ops_hip_error(hipError_t e, const char* what) { return hip_fail(e, what); }

int ops_error(int status, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_hip, sizeof g_last_hip, fmt, ap);
    va_end(ap);
    return status;
}

int ops_check_range(const void* p, size_t bytes, int device, const char* what) {
    return check_device_range(p, bytes, device, what);
}

}  // namespace km
