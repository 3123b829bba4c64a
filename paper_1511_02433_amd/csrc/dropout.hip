// Dropout whose mask is drawn again wherever it is needed (gfx950).
//
//   y_ij = [residual_ij +] x_ij [r_ij >= p 2^32] / (1 - p)
//
// r is a word of Philox4x32 with 7 rounds, the fewest that pass the tests of its authors: four columns share a counter.
//
// Bound by memory: 32,768 x 4,096 bfloat16 onto a residual 146 us (5.5 TB/s; the first kernel, with four columns a thread and every word from its
// first round on, 336).  A product of 32 by 32 bits takes as long as four other instructions, so those that a column's rows share are left out of the loop: 11
// of 14 for four words are left.
#include <algorithm>
#include <cmath>

#include "ccdpp_seq.h"
#include "seq_device.hpp"

namespace ccdops {
namespace {

struct Drop {
    int64_t n, d, ldx, ldr, ldy, first_row;
    const void *x, *residual;
    void* y;
    uint64_t seed;
    const uint64_t* seed_at;
    uint32_t least;   // words from here on are kept
    int none;         // 1: nothing is kept
    float scale;
    int64_t groups, step;  // of columns; rows that are at work at once
};

struct Words { uint32_t w[4]; };

__device__ __forceinline__ Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t k0, uint32_t k1) {
    uint32_t c3 = 0;
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0, c1 = (uint32_t)q;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1, c3 = (uint32_t)p;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// A thread keeps its kColumns columns and goes down the rows, `step` at a time, so the words' first round and half of their second are
// computed once for the rows that share the upper half of their number.  (10,007 x 777 half precision: 7.6 to 8.6 us, unaligned rows; 1,024 x 40
// floats 3.2.)
constexpr int kColumns = 8;
constexpr int64_t kThreads = 1 << 19;  // of a launch: eight blocks of 256 for each CU

template <class T, bool RESIDUAL>
__global__ __launch_bounds__(256) void k_drop(Drop a) {
    const uint64_t seed = a.seed_at ? *a.seed_at : a.seed;
    const uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
    const int64_t thread = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
    int64_t row = thread / a.groups;
    if (row >= a.step) return;
    const int64_t c = (thread - row * a.groups) * kColumns;
    const bool whole = c + kColumns <= a.d;
    while (row < a.n) {
        const uint64_t first = (uint64_t)(a.first_row + row);
        const uint32_t high = (uint32_t)(first >> 32);
        const int64_t same = (int64_t)(0x100000000ull - (uint32_t)first);  // rows from here on with this upper half
        const int64_t end = min(a.n, row + same);
        for (; row < end; row += a.step) {
            Values<T, kColumns> x, res, y;
            x.load((const T*)a.x + row * a.ldx, c, a.d, whole);
            if constexpr (RESIDUAL) res.load((const T*)a.residual + row * a.ldr, c, a.d, whole);
            const uint32_t low = (uint32_t)(a.first_row + row);
#pragma unroll
            for (int q = 0; q < kColumns / 4; ++q) {
                const Words w = philox((uint32_t)(c / 4) + q, low, high, k0, k1);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float v = !a.none && w.w[j] >= a.least ? x.get(4 * q + j) * a.scale : 0.f;
                    y.set(4 * q + j, RESIDUAL ? res.get(4 * q + j) + v : v);
                }
            }
            y.store((T*)a.y + row * a.ldy, c, a.d, whole);
        }
    }
}

template <class F>
void typed(int dtype, F&& body) {
    if (dtype == CCDPP_F32) body(float());
    else if (dtype == CCDPP_BF16) body((__bf16)0.f);
    else body((_Float16)0.f);
}

}  // namespace
}  // namespace ccdops

extern "C" int ccdpp_dropout(int64_t n, int64_t d, int32_t dtype, const void* x, int64_t ldx, const void* residual, int64_t ldr, void* y,
                             int64_t ldy, double p, uint64_t seed, const uint64_t* seed_at, int64_t first_row, void* stream) {
    using namespace ccdops;
    if (n < 0 || n >= (int64_t)1 << 31 || d < 1 || d >= (int64_t)1 << 31) return fail(CCDPP_EINVAL, "n must be in [0, 2^31) and d in [1, 2^31)");
    if (dtype < CCDPP_F32 || dtype > CCDPP_F16) return fail(CCDPP_EINVAL, "dtype must be CCDPP_F32, CCDPP_BF16 or CCDPP_F16");
    if (!(p >= 0.0 && p <= 1.0)) return fail(CCDPP_EINVAL, "p must be in [0, 1]");
    if (first_row < 0 || first_row > INT64_MAX - n) return fail(CCDPP_EINVAL, "first_row must be >= 0, and no row beyond 2^63");
    if (ldx < d || ldy < d || (residual && ldr < d)) return fail(CCDPP_EINVAL, "row strides must be at least d");
    if (n > 0 && (!x || !y)) return fail(CCDPP_EINVAL, "x and y must be non-NULL");
    const uintptr_t es = dtype == CCDPP_F32 ? 4 : 2;
    if ((uintptr_t)x % es || (uintptr_t)y % es || (uintptr_t)residual % es || (uintptr_t)seed_at % 8)
        return fail(CCDPP_EINVAL, "pointers must be aligned to their types");
    if ((y == x && ldy != ldx) || (residual && y == residual && ldy != ldr)) return fail(CCDPP_EINVAL, "y in place must have the same row stride");
    if (int rc = check_device()) return rc;
    if (n == 0) return CCDPP_OK;
    const double least = std::rint(p * 4294967296.0);
    Drop a = {n, d, ldx, ldr, ldy, first_row, x, residual, y, seed, seed_at, 0, least >= 4294967296.0, 0.f, 0, 0};
    if (!a.none) a.least = (uint32_t)least, a.scale = (float)(1.0 / (1.0 - p));
    a.groups = (d + kColumns - 1) / kColumns;
    a.step = std::min<int64_t>(n, std::max<int64_t>(1, kThreads / a.groups));
    const unsigned blocks = (unsigned)((a.groups * a.step + 255) / 256);
    typed(dtype, [&](auto z) {
        typedef decltype(z) T;
        if (residual) k_drop<T, true><<<blocks, 256, 0, (hipStream_t)stream>>>(a);
        else k_drop<T, false><<<blocks, 256, 0, (hipStream_t)stream>>>(a);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CCDPP_OK : hip_fail(e, "dropout");
}
