// Shared by the kernels of ccdpp_seq.h that take values side by side (gfx950).
#pragma once

#include "ops_internal.hpp"

namespace ccdops {

// N values of a row from column c on, in accesses of 16 bytes (of 8 for four of 16 bits); `whole`: all of them lie within its d columns.
template <class T, int N>
struct Values {
    static constexpr int W = N < (int)(16 / sizeof(T)) ? N : 16 / sizeof(T);
    Run<T, W> r[N / W];
    __device__ __forceinline__ void load(const T* row, int64_t c, int64_t d, bool whole) {
        if (whole) {
#pragma unroll
            for (int k = 0; k < N / W; ++k) r[k] = load_run<W>(row + c + k * W);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) r[j / W].v[j % W] = c + j < d ? row[c + j] : (T)0.f;
        }
    }
    __device__ __forceinline__ void store(T* row, int64_t c, int64_t d, bool whole) const {
        if (whole) {
#pragma unroll
            for (int k = 0; k < N / W; ++k) store_run<W>(row + c + k * W, r[k]);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (c + j < d) row[c + j] = r[j / W].v[j % W];
        }
    }
    __device__ __forceinline__ float get(int j) const { return (float)r[j / W].v[j % W]; }
    __device__ __forceinline__ void set(int j, float v) { r[j / W].v[j % W] = (T)v; }
};

}  // namespace ccdops
