// Shared by the sources of the operators of ccdpp_ops.h (gfx950).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "ccdpp_ops.h"

namespace ccdops {

// Sets the message that ccdpp_ops_last_error() returns on this thread; returns `code`.
int fail(int code, const char* msg);
int hip_fail(hipError_t e, const char* what);

// CCDPP_OK where the current device is a gfx950 one.
int check_device();

// N values in one access that need not be aligned beyond their type: global memory takes 16 bytes at any address.
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Run {
    T v[N];
};

inline int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

}  // namespace ccdops
