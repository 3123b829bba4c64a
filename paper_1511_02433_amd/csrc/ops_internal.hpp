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

// N values in one access (two of 16 bytes at most) that need not be aligned beyond their type: global memory takes 16
// bytes at any address.  The accesses are of whole vectors: of a structure's values the compiler would make an
// access each.
template <class T, int N>
struct Run {
    T v[N];
};
typedef uint32_t words2 __attribute__((ext_vector_type(2), may_alias));
typedef uint32_t words4 __attribute__((ext_vector_type(4), may_alias));
template <int A> struct Loose;
template <> struct Loose<2> {
    typedef words2 two __attribute__((aligned(2)));
    typedef words4 four __attribute__((aligned(2)));
};
template <> struct Loose<4> {
    typedef words2 two __attribute__((aligned(4)));
    typedef words4 four __attribute__((aligned(4)));
};

template <int N, class T>
__device__ __forceinline__ Run<T, N> load_run(const T* at) {
    typedef Loose<sizeof(T)> L;
    constexpr int B = N * sizeof(T);
    typedef Run<T, N> R;
    static_assert(B == 8 || B == 16 || B == 32, "");
    if constexpr (B == 8) {
        return __builtin_bit_cast(R, (words2)*(const typename L::two*)at);
    } else if constexpr (B == 16) {
        return __builtin_bit_cast(R, (words4)*(const typename L::four*)at);
    } else {
        struct Both { words4 a, b; };
        const Both both = {*(const typename L::four*)at, *((const typename L::four*)at + 1)};
        return __builtin_bit_cast(R, both);
    }
}

template <int N, class T>
__device__ __forceinline__ void store_run(T* at, Run<T, N> r) {
    typedef Loose<sizeof(T)> L;
    constexpr int B = N * sizeof(T);
    static_assert(B == 8 || B == 16, "");
    if constexpr (B == 8) *(typename L::two*)at = __builtin_bit_cast(words2, r);
    else *(typename L::four*)at = __builtin_bit_cast(words4, r);
}

// The N values of a row from column c on, those past its d columns 0.  One access as well where the memory goes on for
// `room` values from the row's start (the rows after it).
template <int N, class T>
__device__ __forceinline__ Run<T, N> load_tail(const T* row, int c, int d, int64_t room) {
    if (c + N <= d) return load_run<N>(row + c);
    Run<T, N> r = {};
    if (c >= d) return r;
    if (c + N <= room) {
        r = load_run<N>(row + c);
#pragma unroll
        for (int j = 0; j < N; ++j) r.v[j] = c + j < d ? r.v[j] : (T)0.f;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c + j < d) r.v[j] = row[c + j];
    }
    return r;
}

// Stores those of N values from column c on that lie within d columns.
template <int N, class T>
__device__ __forceinline__ void store_tail(T* row, int c, int d, Run<T, N> r) {
    if (c + N <= d) {
        store_run<N>(row + c, r);
    } else {
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (c + j < d) row[c + j] = r.v[j];
    }
}

inline int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

}  // namespace ccdops
