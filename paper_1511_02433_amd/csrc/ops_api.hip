// Errors and the device check of the operators of ccdpp_ops.h.
#include <cstdio>
#include <cstring>

#include "ops_internal.hpp"

namespace ccdops {
namespace {
thread_local char g_error[256] = "";  // fixed, so that nothing can throw here
}

int fail(int code, const char* msg) {
    std::snprintf(g_error, sizeof g_error, "%s", msg);
    return code;
}

int hip_fail(hipError_t e, const char* what) {
    std::snprintf(g_error, sizeof g_error, "%s: %s", what, hipGetErrorString(e));
    return CCDPP_EDEVICE;
}

int check_device() {
    thread_local int checked = -1;  // the last device found to be usable by this thread
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return hip_fail(e, "no device");
    }
    if (dev == checked) return CCDPP_OK;
    hipDeviceProp_t prop;
    e = hipGetDeviceProperties(&prop, dev);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return hip_fail(e, "device properties");
    }
    if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0) return fail(CCDPP_EDEVICE, "the current device is not gfx950");
    checked = dev;
    return CCDPP_OK;
}

}  // namespace ccdops

extern "C" const char* ccdpp_ops_last_error(void) { return ccdops::g_error; }
