// Device code that the softmax loss's kernels share (gfx950).
#pragma once

#include <type_traits>

#include "ops_internal.hpp"

namespace ccdops {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kExcluded = -1e38f;  // offsets below this exclude an item
constexpr int kBlk = 1024;           // bytes of one operand fragment

// The 16-bit type that the matrix instructions read.
struct BF {
    typedef __bf16 elem;
    typedef bf16x8 vec;
    static __device__ f32x16 mfma(vec a, vec b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
struct HF {
    typedef _Float16 elem;
    typedef f16x8 vec;
    static __device__ f32x16 mfma(vec a, vec b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// Input type -> operand type and number of planes.  `turned`: what many factors' gradients take, half precision, whose 11
// bits keep the terms G of bfloat16 problems from costing as much as the rounding of the result does; the
// turned matrices then get a power of two of their own.
template <int DT> struct Types;
template <> struct Types<CCDPP_F32> { typedef float in; typedef HF op; typedef HF turned; static constexpr int planes = 2; };
template <> struct Types<CCDPP_BF16> { typedef __bf16 in; typedef BF op; typedef HF turned; static constexpr int planes = 1; };
template <> struct Types<CCDPP_F16> { typedef _Float16 in; typedef HF op; typedef HF turned; static constexpr int planes = 1; };

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// Power of two that brings values up to `top` below 2^15 (the result's exponent).
__device__ __forceinline__ int scale_exp(float top) {
    if (!(top > 0.f)) return 0;
    const int e = (int)(__float_as_uint(top) >> 23) - 127;  // subnormals: -127
    return min(126, 14 - e);
}

// Power of two that brings the table to [4, 8) for the logits.
__device__ __forceinline__ int unit_exp(float top) {
    if (!(top > 0.f)) return 0;
    return max(-126, min(126, 129 - (int)(__float_as_uint(top) >> 23)));
}

// Two half-precision planes hold a value to 22 bits of itself, or to 2^-25.  With the whole table under one power of two
// (unit_exp) and x under its inverse the products are logits as they are, and what the table's and x's values lack of 22 bits
// costs a logit some 2^-26 |x'| and 2^-26 |e'|, x' and e' being the rows as they are multiplied.  Up to kUnitNorm that is
// 5e-7 each (|e'| is 12 for 40 factors and 22 for 128, if the largest is five deviations).  Beyond it a large value of the table could cost other items their digits: rows of x get powers of two of their own, so that the table's
// can be 2^14 higher (a factor for each row of x), which is as good up to kFactorNorm, and from there on the table's rows have
// their own, too.  (1,500 x 624,961 x 40 floats, the three ways: 330, 384 and 429 us.)
constexpr float kUnitNorm = 32.f, kFactorNorm = 32.f * 16384.f;
enum { kUnit = 0, kFactor = 1, kOwn = 2 };

// Value in planes: hi + lo, 22 bits; lo stays 0 where hi is not finite.
template <class P, int NPL>
__device__ __forceinline__ void to_planes(float v, typename P::elem* out) {
    out[0] = (typename P::elem)v;
    if constexpr (NPL == 2) {
        const float hi = (float)out[0];
        out[1] = (typename P::elem)(finite(hi) ? v - hi : 0.f);
    }
}

// The terms G of one lane, in planes of operand fragments, rounded to nearest (pairs of half-precision values share an
// instruction): 22 bits of each term in two planes down to 2^-3, 2^-25 below it.
template <class P, int NPL>
__device__ __forceinline__ void split_terms(const float* g, typename P::vec (*pl)[2]) {
    if constexpr (NPL == 2 && std::is_same<P, HF>::value) {
        typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
        typedef float float2_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            const half2_t hi = __builtin_convertvector((float2_t){g[r], g[r + 1]}, half2_t);
            const half2_t lo = __builtin_convertvector((float2_t){g[r] - (float)hi[0], g[r + 1] - (float)hi[1]}, half2_t);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                pl[0][r >> 3][(r & 7) + k] = (typename P::elem)hi[k];
                pl[1][r >> 3][(r & 7) + k] = (typename P::elem)lo[k];
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            pl[0][r >> 3][r & 7] = (typename P::elem)g[r];
            if constexpr (NPL == 2) pl[1][r >> 3][r & 7] = (typename P::elem)(g[r] - (float)pl[0][r >> 3][r & 7]);
        }
    }
}

__device__ __forceinline__ int64_t load_target(const void* y, int bits, int64_t t) {
    return bits == 64 ? ((const int64_t*)y)[t] : (int64_t)((const int32_t*)y)[t];
}

// Whether row t takes part in the gradients: its target is neither negative nor an excluded item.
__device__ __forceinline__ bool row_counts(int64_t y, int64_t v, const float* offset) {
    if (y < 0) return false;
    return !(y < v && offset && offset[y] < kExcluded);
}

// Largest value of a wave, by moves between lanes that do not go through LDS: within rows of 16 lanes, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_from(float m) {
    const int i = __builtin_bit_cast(int, m);
    return fmaxf(m, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float m) {
    m = max_from<0x111, 0xf>(m), m = max_from<0x112, 0xf>(m), m = max_from<0x114, 0xf>(m), m = max_from<0x118, 0xf>(m);  // row_shr
    m = max_from<0x142, 0xa>(m), m = max_from<0x143, 0xc>(m);  // row_bcast:15, row_bcast:31
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, m), 63));
}

// The larger of a lane's value and that of the lane 32 places away.
__device__ __forceinline__ float halves_max(float m) {
    const uint32_t i = __float_as_uint(m);
    const auto both = __builtin_amdgcn_permlane32_swap(i, i, false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// 1 KB from global memory into LDS, 16 bytes per lane, without passing through registers.
__device__ __forceinline__ void fetch(const char* from, char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// ---- few factors (d <= kSmallD) ------------------------------------------------------------
// Everything about 32 rows of x or of the table in one piece of memory, in blocks of 1 KB: the operand fragments of the
// rows [plane][step of 16 over d]; the rows' numbers, 32 floats each; the fragments of the turned rows
// [plane][32 columns][2 steps of 16 rows].
enum {
    kNumFactor = 0,   // x: factor of the accumulated logits, or (kOwn) an exponent, as int32
    kNumOffset = 0,   // table: offset in base 2, -inf for excluded and missing entries
    kNumExp = 1,      // table: (kOwn) the exponent of its row
    kNumTerm = 1,     // x: log2 |weight| - lse in base 2, G's exponent: G = exp2(logit + term)
    kNumWeight = 2,   // x: |weight| with G's power of two
    kNumTarget = 3,   // x: target, as int32
    kNumLse = 4,      // x: minus lse in base 2; -inf in rows that do not count
    kNumRaw = 5       // x: weight as it is
};
constexpr int kTermExp = 13;  // of dx's terms, which leave the row's weight to the end: at most 2^13 each

// Up to here the kernels of few factors; above it the products of k_gemm.  Loss and gradients of 1,024 x 20,000 rows,
// this way and by k_gemm: 100 floats 114 and 174 us, 128 floats 122 and 191, 128 in bfloat16 75 and 132.
constexpr int kSmallD = 128;

// A product of few factors is cut by tiles: kept blocks of 128 rows times streamed tiles of 32, in that order, in shares
// of `len` tiles, a block each, so that all blocks work equally long.  A share may end in one kept block and go on in the
// next; every kept block sums the shares that touch it, in order.
struct Shares {
    int64_t tiles;   // streamed tiles of each kept block
    int64_t len;     // tiles of a share
    int64_t blocks;  // shares
    __host__ __device__ int64_t first(int64_t kept) const { return kept * tiles / len; }
    __host__ __device__ int count(int64_t kept) const { return (int)(((kept + 1) * tiles - 1) / len - first(kept) + 1); }
    __host__ __device__ bool whole() const { return len > 0 && tiles > 0 && len % tiles == 0; }  // a share per kept block
    __host__ __device__ int64_t most() const { return whole() ? 1 : tiles > 0 ? (tiles + len - 2) / len + 1 : 0; }  // of count()
};

struct SmallOut {
    void* to;     // a gradient
    int64_t ld;
};

struct SmallArgs {
    const char *x, *xlive, *e;          // bundles: x without turned rows; x with them, rows that do not count zeroed; the table
    int64_t x_tile, xlive_tile, e_tile; // bytes of one bundle
    int64_t tt, vt;                     // bundles
    int64_t t, v;
    int offsets;                        // whether the table has offsets
    Shares lse, dx, de;                 // dx.blocks or de.blocks 0: not asked for
    float2* part;                       // [share of the kept block][t]
    float *dxp, *dep;                   // [share of the kept block][rows, in tiles][d, in blocks of 32]
    SmallOut dx_out, de_out;            // of kept blocks that have one share
    int d, scaled;                      // scaled: fin holds exponents of x and the table
    const int32_t* fin;                 // or NULL
    float scale;
};

// ksd: steps of 16 over d that the kernels were built for (small_steps).  Return launch errors.
int small_steps(int d);
// Blocks that a CU holds, by registers and LDS.
constexpr int small_lse_per_cu(int planes, int ks) { return planes * ks > 12 ? 3 : 4; }
constexpr int small_grads_per_cu(int planes, int ks) { return ks > 4 || planes * ks > 8 ? 2 : 3; }
template <class P, int NPL> hipError_t launch_small_lse(int ksd, const SmallArgs& a, hipStream_t st);
template <class P, int NPL> hipError_t launch_small_grads(int ksd, const SmallArgs& a, hipStream_t st);

// ---- few rows --------------------------------------------------------------------------------
// Rows whose logits are computed from the table as it lies.  The loss of 200,000 entries, this way and by k_gemm from a
// packed table: 64 x 256 floats 88 and 217 us, 128 x 256 floats 182 and 219, 128 x 1,024 in bfloat16 195 and 296: the time
// of the former grows with the rows, that of packing the table does not.
constexpr int kDirectT = 128;
// Rows whose gradients are, too.  Loss and gradients of 200,000 x 256, this way and the other: 16 rows of floats 136 and 399
// us, 32 rows 177 and 415, 32 in bfloat16 107 and 217; more rows do not fit the registers of two blocks on a CU.
constexpr int kFewT = 32;

struct FewArgs {
    int t, d, dp;             // dp: columns of partial sums, a multiple of 4
    int64_t v;
    const void *x, *table, *target;
    int64_t ldx, ldt;
    int target_bits;
    float scale;
    const float* offset;
    int share, chunk;         // see FewShape
    float2* part;             // [block][t] (max, sum), base 2, or NULL
    float* z;                 // logits in base 2 [t][z_row], or NULL
    int64_t z_row;            // a multiple of 32
    const float *lse, *grad;
    void* de;                 // or NULL
    int64_t ldde;
    float* dxp;               // [part][t][dp], or NULL
    int parts;                // blocks along the table
    int across;               // waves along a row
};

struct FewShape {
    int share;    // waves that share the columns of 16 table rows
    int rows;     // groups of 16 table rows of a wave
    int chunk;    // steps of 64 bytes of x's rows in LDS at a time
    int blocks;
    int64_t lds;
};

FewShape few_shape(int64_t t, int64_t v, int d, int bytes);
int few_across(int d, int columns);
template <class T> hipError_t launch_few_logits(const FewArgs& a, const FewShape& s, hipStream_t st);
template <class T> hipError_t launch_few_grads(const FewArgs& a, T* dx, int64_t lddx, hipStream_t st);

}  // namespace ccdops
