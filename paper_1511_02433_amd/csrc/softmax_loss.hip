// Softmax cross entropy of rows against a whole table, and its gradients, without keeping the logits (gfx950).
//
//   z_tv = s x_t.e_v + o_v     lse_t = log sum_v exp z_tv     loss_t = lse_t - z_{t,y_t}
//   G_tv = g_t (exp(z_tv - lse_t) - [v = y_t])     dx = s G E     de = s G^T X
//
// Three matrix products: logits (v x t, contracted over d), dx (t x d, over v) and de (v x d, over t).  All of
// them run on one kernel, k_gemm, that takes its two operands in fragment order: a matrix of R rows contracted over
// K is stored as blocks of 32 rows x 16 columns, block (r, s) being the 64 lanes' 8 values of one
// v_mfma_f32_32x32x16 operand in lane order (lane l: row l % 32, columns 8 (l / 32) .. + 7), 1 KB in one piece.  k_pack
// brings x and the table into that order once per call, zero-padded, both as they are and turned (for the
// contraction over their rows), whatever their strides, alignment and type.  32-bit values become two half-precision
// planes, hi + lo, under a common power of two; a product of such matrices is the three products hi hi + hi lo +
// lo hi, summed in the same accumulator (lo lo is below 2^-22 of the result).
//
// The accumulator of the logits holds, per lane, one row t and 16 table entries v = 8 q + 4 h + r (h = lane / 32): those
// are what two fragments of G need for a contraction over v in the order
//   slot (h, j) of a fragment of 16  <->  v = 4 h + j (j < 4), 8 + 4 h + j - 4 (j >= 4),
// so G is written as operand fragments straight from the accumulators, and k_pack turns the table in the same order.
// G^T for de comes from the same fragments by one more product, with the identity: its accumulator holds the turned
// block, exact since every sum has one term.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops_internal.hpp"

namespace ccdops {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kExcluded = -1e38f;  // offsets below this exclude an item
constexpr int kParts = 256;          // partial maxima of k_scales per quantity
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

// Input type -> operand type and number of planes.
template <int DT> struct Types;
template <> struct Types<CCDPP_F32> { typedef float in; typedef HF op; static constexpr int planes = 2; };
template <> struct Types<CCDPP_BF16> { typedef __bf16 in; typedef BF op; static constexpr int planes = 1; };
template <> struct Types<CCDPP_F16> { typedef _Float16 in; typedef HF op; static constexpr int planes = 1; };

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// Power of two that brings values up to `top` below 2^15 (the result's exponent).
__device__ __forceinline__ int scale_exp(float top) {
    if (!(top > 0.f)) return 0;
    const int e = (int)(__float_as_uint(top) >> 23) - 127;  // subnormals: -127
    return min(126, 14 - e);
}

// Value in planes: hi + lo, 22 bits; lo stays 0 where hi is not finite.
template <class P, int NPL>
__device__ __forceinline__ void to_planes(float v, typename P::elem* out) {
    out[0] = (typename P::elem)v;
    if constexpr (NPL == 2) {
        const float hi = (float)out[0];
        out[1] = (typename P::elem)(finite(hi) ? v - hi : 0.f);
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

__device__ __forceinline__ float wave_max(float m) {
    for (int k = 32; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    return m;
}

// ---- scales of 32-bit inputs ----------------------------------------------------------
// Exponents of the powers of two that x's rows (their own, for the logits; one for all rows that count, for de), the
// table and the rows' weights are multiplied with.  Only finite values count.
struct Scales {
    float* e_part;   // [kParts] largest |table| value (items that are not excluded)
    float* x_part;   // [kParts] largest |x| value of rows that count
    float* g_part;   // [kParts] largest |grad|
    int32_t* x_row;  // [t] exponent of each row of x
    int32_t* fin;    // [3] exponents: table, x, G
};

// Blocks 0 .. kParts - 1 take the table's rows in turn (a wave per row), blocks kParts .. the rows of x.
template <class T>
__global__ __launch_bounds__(256) void k_scales(ccdpp_softmax_t p, const float* grad, Scales sc, int with_mats, int grads) {
    __shared__ float red[4][3];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float em = 0.f, xm = 0.f, gm = 0.f;
    const int b = blockIdx.x < kParts ? blockIdx.x : blockIdx.x - kParts;
    if (blockIdx.x < kParts) {
        if (with_mats)
            for (int64_t v = b * 4 + wave; v < p.v; v += kParts * 4) {
                if (p.offset && p.offset[v] < kExcluded) continue;
                const T* row = (const T*)p.table + v * p.ldt;
                for (int d = lane; d < p.d; d += 64) {
                    const float a = fabsf((float)row[d]);
                    if (finite(a)) em = fmaxf(em, a);
                }
            }
    } else {
        for (int64_t t = b * 4 + wave; t < p.t; t += kParts * 4) {
            const bool counts = row_counts(load_target(p.target, p.target_bits, t), p.v, p.offset);
            if (with_mats) {
                const T* row = (const T*)p.x + t * p.ldx;
                float m = 0.f;
                for (int d = lane; d < p.d; d += 64) {
                    const float a = fabsf((float)row[d]);
                    if (finite(a)) m = fmaxf(m, a);
                }
                m = wave_max(m);
                if (lane == 0) sc.x_row[t] = scale_exp(m);
                if (counts) xm = fmaxf(xm, m);
            }
            if (grads && counts) {
                const float g = grad ? fabsf(grad[t]) : 1.f;
                if (finite(g)) gm = fmaxf(gm, g);
            }
        }
    }
    em = wave_max(em), xm = wave_max(xm), gm = wave_max(gm);
    if (lane == 0) red[wave][0] = em, red[wave][1] = xm, red[wave][2] = gm;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w) {
            em = fmaxf(em, red[w][0]), xm = fmaxf(xm, red[w][1]), gm = fmaxf(gm, red[w][2]);
        }
        if (blockIdx.x < kParts) sc.e_part[b] = em;
        else sc.x_part[b] = xm, sc.g_part[b] = gm;
    }
}

// G lies within its row's weight, or a few times that where lse is the caller's own: two bits are left for it.
__global__ __launch_bounds__(64) void k_scales_final(Scales sc) {
    float em = 0.f, xm = 0.f, gm = 0.f;
    for (int i = threadIdx.x; i < kParts; i += 64) em = fmaxf(em, sc.e_part[i]), xm = fmaxf(xm, sc.x_part[i]), gm = fmaxf(gm, sc.g_part[i]);
    em = wave_max(em), xm = wave_max(xm), gm = wave_max(gm);
    if (threadIdx.x == 0) sc.fin[0] = scale_exp(em), sc.fin[1] = scale_exp(xm), sc.fin[2] = scale_exp(gm) - 2;
}

// ---- operands in fragment order ----------------------------------------------------------
struct PackArgs {
    const void* src;
    int64_t ld, rows;
    int d;
    int ksd;              // 16-wide steps over d (even)
    int64_t ksr;          // 16-wide steps over rows (even)
    char* nat;            // [plane][rows/32][ksd] fragments of the matrix, or NULL
    char* turned;         // [plane][d/32][ksr] fragments of its transpose, or NULL
    int64_t nat_plane, turned_plane;  // bytes
    const int32_t* row_exp;           // exponent per row for `nat` (x), or NULL
    const int32_t* fin;               // exponents of k_scales_final, or NULL: no scaling
    int which;                        // 0: the table, 1: x
    const void* target;
    int target_bits;
    int64_t v;
    const float* offset;
    float* o2;                        // of the table: offsets in base 2, padded with -inf
};

// One block: 32 rows x 128 columns through LDS.
template <int DT>
__global__ __launch_bounds__(256) void k_pack(PackArgs a) {
    typedef typename Types<DT>::in T;
    typedef typename Types<DT>::op P;
    constexpr int NPL = Types<DT>::planes;
    __shared__ float tile[32][129];
    __shared__ float mul[32];   // natural
    __shared__ float mult[32];  // turned
    const int64_t r0 = (int64_t)blockIdx.x * 32;
    const int c0 = blockIdx.y * 128;
    if (threadIdx.x < 32) {
        const int64_t r = r0 + threadIdx.x;
        float m = 1.f, mt = 1.f;
        if (r < a.rows) {
            if (a.fin) {
                m = pow2i(a.row_exp ? a.row_exp[r] : a.fin[a.which]);
                mt = pow2i(a.fin[a.which]);
            }
            if (a.which == 0) {
                if (a.offset && a.offset[r] < kExcluded) m = mt = 0.f;
            } else if (a.turned && !row_counts(load_target(a.target, a.target_bits, r), a.v, a.offset)) {
                mt = 0.f;
            }
        }
        mul[threadIdx.x] = m, mult[threadIdx.x] = mt;
        if (a.o2 && blockIdx.y == 0) {
            const float o = r < a.rows && a.offset ? a.offset[r] : 0.f;
            a.o2[r] = r >= a.rows || o < kExcluded ? -INFINITY : o * kLog2e;
        }
    }
    for (int i = threadIdx.x; i < 32 * 128; i += 256) {
        const int r = i >> 7, c = i & 127;
        float v = 0.f;
        if (r0 + r < a.rows && c0 + c < a.d) v = (float)((const T*)a.src)[(r0 + r) * a.ld + c0 + c];
        tile[r][c] = v;
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 31, h = lane >> 5;
    if (a.nat)
        for (int s = wave; s < 8; s += 4) {
            const int ks = c0 / 16 + s;
            if (ks >= a.ksd) break;
            typename P::elem o[8][2];
            const float f = mul[m];
            for (int j = 0; j < 8; ++j) {
                const float v = f == 0.f ? 0.f : tile[m][s * 16 + 8 * h + j] * f;
                to_planes<P, NPL>(v, o[j]);
            }
            for (int pl = 0; pl < NPL; ++pl) {
                typename P::vec w;
                for (int j = 0; j < 8; ++j) w[j] = o[j][pl];
                *(typename P::vec*)(a.nat + pl * a.nat_plane + ((int64_t)blockIdx.x * a.ksd + ks) * kBlk + lane * 16) = w;
            }
        }
    if (a.turned)
        for (int i = wave; i < 8; i += 4) {  // 4 blocks of 32 columns x 2 steps of 16 rows
            const int dt = i >> 1, s = i & 1;
            if (c0 + dt * 32 >= a.d) break;
            typename P::elem o[8][2];
            for (int j = 0; j < 8; ++j) {
                const int r = 16 * s + (j < 4 ? 4 * h + j : 8 + 4 * h + j - 4);
                const float f = mult[r];
                const float v = f == 0.f ? 0.f : tile[r][dt * 32 + m] * f;
                to_planes<P, NPL>(v, o[j]);
            }
            for (int pl = 0; pl < NPL; ++pl) {
                typename P::vec w;
                for (int j = 0; j < 8; ++j) w[j] = o[j][pl];
                *(typename P::vec*)(a.turned + pl * a.turned_plane +
                                    ((int64_t)(c0 / 32 + dt) * a.ksr + (int64_t)blockIdx.x * 2 + s) * kBlk + lane * 16) = w;
            }
        }
}

// ---- the product -----------------------------------------------------------------------------
// C (M x N) = A (M x K) B (N x K)^T from fragments: 256 x 256 of C per block, 8 waves of 128 x 64 each.
enum { EPI_LSE = 0, EPI_G = 1, EPI_OUT = 2 };

struct GemmArgs {
    const char *a, *b;
    int64_t a_plane, b_plane;    // bytes between planes
    int64_t a_tile, b_tile;      // bytes between blocks of 32 rows
    int64_t m_tiles, n_tiles;    // blocks of 32 rows that exist
    int64_t kb;                  // steps of 32 over K, in one plane
    int splits;                  // shares of kb
    // logits
    int64_t v0;                  // table entry of row 0 of A
    int64_t t, v;
    int scaled;                  // 32-bit inputs: x_row, fin[0] hold
    const int32_t *x_row, *fin;  // exponents; fin is NULL where nothing is scaled
    float scale;
    const float* offset;
    const float* o2;             // offsets of A's rows in base 2, -inf for excluded and missing ones
    float2* part;                // [blocks of 256 table entries][t] (max, sum), base 2
    const void* target;
    int target_bits;
    const float *lse, *grad;
    char *g, *gt;                // G [plane][t/32][ksv], G^T [plane][v/32][kst] fragments
    int64_t g_plane, gt_plane;
    int64_t ksv, kst;
    // other products
    float* out;                  // [split][M][ldo]
    void* last;                  // or the result itself
    int64_t out_split, rows, cols, ldo;
    int add, which;              // which: the exponent in fin of the other operand, or -1
};

constexpr int kStages = 4;          // of LDS, each a step of 32 over K of both operands
constexpr int kStage = 32 * kBlk;

// 1 KB from global memory into LDS, 16 bytes per lane, without passing through registers.
__device__ __forceinline__ void fetch(const char* from, char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

template <class P, int NPL, int EPI, class T>
__global__ __launch_bounds__(512) void k_gemm(GemmArgs a) {
    constexpr int NSEG = NPL == 2 ? 3 : 1;
    __shared__ __align__(16) char lds[kStages * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 2, wn = wave & 3;
    const int split = blockIdx.y;
    // Blocks b, b + 8, .. share an XCD and its L2: each gets a contiguous run of tiles, eight rows of tiles at a time.
    const int64_t mb = (a.m_tiles + 7) / 8, nb = (a.n_tiles + 7) / 8;
    int64_t bm, bn;
    {
        const int64_t all = mb * nb, x = blockIdx.x & 7, per = all >> 3, more = all & 7;
        const int64_t id = x * per + min(x, more) + (blockIdx.x >> 3);
        const int64_t band = id / (8 * nb), first = band * 8, height = min((int64_t)8, mb - first);
        const int64_t in = id - band * 8 * nb;
        bm = first + in % height, bn = in / height;
    }
    const int64_t k0 = a.kb * split / a.splits, k1 = a.kb * (split + 1) / a.splits;
    f32x16 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // A wave brings one block of 32 rows of either operand, 2 KB a stage each.
    const int64_t steps = k1 - k0, total = steps * NSEG;
    if (total > 0) {
        const char* const a0 = a.a + min(bm * 8 + wave, a.m_tiles - 1) * a.a_tile + k0 * 2 * kBlk + lane * 16;
        const char* const b0 = a.b + min(bn * 8 + wave, a.n_tiles - 1) * a.b_tile + k0 * 2 * kBlk + lane * 16;
        const char *pa = a0, *pb = b0;
        int64_t left = steps;
        int seg = 0;
        char* const to = lds + wave * 2 * kBlk;
        int slot = 0;
        // Past the last step the last one is fetched again, so that the count of loads in flight stays the same.
        const auto next = [&]() {
            char* const s = to + slot * kStage;
            fetch(pa, s);
            fetch(pa + kBlk, s + kBlk);
            fetch(pb, s + 16 * kBlk);
            fetch(pb + kBlk, s + 17 * kBlk);
            slot = (slot + 1) & (kStages - 1);
            if (--left > 0) {
                pa += 2 * kBlk, pb += 2 * kBlk;
            } else if (seg < NSEG - 1) {
                ++seg;
                pa = a0 + (seg == 2 ? a.a_plane : 0), pb = b0 + (seg == 1 ? a.b_plane : 0);
                left = steps;
            } else {
                left = 1;
            }
        };
        typename P::vec fa[2][4], fb[2][2];
        const char* const ra = lds + wm * 8 * kBlk + lane * 16;
        const char* const rb = lds + (16 + wn * 4) * kBlk + lane * 16;
        const auto read = [&](int s, int at, int buf) {
#pragma unroll
            for (int i = 0; i < 4; ++i) fa[buf][i] = *(const typename P::vec*)(ra + at * kStage + (2 * i + s) * kBlk);
#pragma unroll
            for (int j = 0; j < 2; ++j) fb[buf][j] = *(const typename P::vec*)(rb + at * kStage + (2 * j + s) * kBlk);
        };
        // Eight products; the reads (and fetches) issued with them go in between, one after each.
        const auto multiply = [&](int buf, bool fetched) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = P::mfma(fa[buf][i], fb[buf][j], acc[i][j]);
#pragma unroll
            for (int i = 0; i < 6; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (fetched && i < 4) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" ::: "memory");
        };
        next(), next(), next(), next();
        asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(0, 0, 0);
        int at = 0;
        for (int64_t k = total; k > 0; --k) {
            read(1, at, 1);
            multiply(0, false);
            // Everybody is done with this stage and has the next one: fetch into this one, read on in the next.
            asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            next();
            at = (at + 1) & (kStages - 1);
            read(0, at, 0);
            multiply(1, true);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    const int n = lane & 31, h = lane >> 5;
    if constexpr (EPI == EPI_OUT) {
        // Last piece and only share: the caller's type.  Else 32 bits, added to what earlier pieces left.
        const float fg = a.fin ? ldexpf(1.f, -a.fin[2]) : 1.f, f = a.fin && a.which >= 0 ? ldexpf(a.scale, -a.fin[a.which]) : a.scale;
        float* const part = a.out + split * a.out_split;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t col = (bn * 8 + wn * 2 + j) * 32 + n;
                const int64_t row0 = (bm * 8 + wm * 4 + i) * 32 + 4 * h;
                if (col >= a.cols) continue;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int64_t row = row0 + 8 * (r >> 2) + (r & 3);
                    if (row >= a.rows) continue;
                    if (a.last) {
                        ((T*)a.last)[row * a.ldo + col] = (T)(acc[i][j][r] * fg * f);
                    } else {
                        float* o = part + row * a.ldo + col;
                        *o = a.add ? *o + acc[i][j][r] : acc[i][j][r];
                    }
                }
            }
        return;
    }
    // Logits in base 2: accumulator times the row's factor, plus offset.
    const int ee = a.scaled ? a.fin[0] : 0;
    const auto factor = [&](int64_t t) {
        const int xe = a.scaled ? a.x_row[min(t, a.t - 1)] : 0;
        return ldexpf(a.scale * kLog2e, -(xe + ee));
    };
    const auto offsets = [&](int64_t tile, f32x4* o) {  // of a block of 32 entries, those of this lane's rows
        const float* at = a.o2 + tile * 32 + 4 * h;
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = *(const f32x4*)(at + 8 * q);
    };
    if constexpr (EPI == EPI_LSE) {
        float2(*share)[256] = (float2(*)[256])lds;
        float f[2], top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j) f[j] = factor((bn * 8 + wn * 2 + j) * 32 + n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t tile = bm * 8 + wm * 4 + i;
            f32x4 o[4];
            if (tile < a.m_tiles) {
                offsets(tile, o);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) o[q] = -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    acc[i][j][r] = fmaf(acc[i][j][r], f[j], o[r >> 2][r & 3]);
                    top[j] = fmaxf(top[j], acc[i][j][r]);
                }
        }
        __syncthreads();  // LDS is free
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            top[j] = fmaxf(top[j], __shfl_xor(top[j], 32));
            const float ref = top[j] == -INFINITY ? 0.f : top[j];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[j] += exp2_fast(acc[i][j][r] - ref);
            sum[j] += __shfl_xor(sum[j], 32);
            if (h == 0) share[wm][(wn * 2 + j) * 32 + n] = make_float2(top[j], sum[j]);
        }
        __syncthreads();
        if (threadIdx.x < 256) {
            const int64_t t = bn * 256 + threadIdx.x;
            const float2 p = share[0][threadIdx.x], q = share[1][threadIdx.x];
            const float m = fmaxf(p.x, q.x);
            const float mr = m == -INFINITY ? 0.f : m;
            if (t < a.t) a.part[bm * a.t + t] = make_float2(m, p.y * exp2_fast(p.x - mr) + q.y * exp2_fast(q.x - mr));
        }
        return;
    }
    if constexpr (EPI == EPI_G) {
        // identity in B-operand order for the two steps of 16 entries
        typename P::vec eye[2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < 8; ++k) eye[s][k] = (typename P::elem)(16 * s + (k < 4 ? 4 * h + k : 8 + 4 * h + k - 4) == n ? 1.f : 0.f);
        float w[2], l2[2], f[2];
        int64_t y[2];        // target, from the piece's first entry
        uint32_t keep[2];    // all ones in rows that count: others are cut off as bits, whatever they hold
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t t = (bn * 8 + wn * 2 + j) * 32 + n;
            w[j] = 0.f, l2[j] = 0.f, f[j] = 0.f, y[j] = -1, keep[j] = 0;
            if (t < a.t) {
                const int64_t yt = load_target(a.target, a.target_bits, t);
                f[j] = factor(t);
                if (row_counts(yt, a.v, a.offset)) {
                    keep[j] = ~0u;
                    w[j] = a.grad ? a.grad[t] : 1.f;
                    if (a.fin) w[j] = ldexpf(w[j], a.fin[2]);
                    if (yt >= a.v) w[j] = NAN;
                    l2[j] = a.lse[t] * kLog2e;
                    y[j] = yt - a.v0;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t vt = bm * 8 + wm * 4 + i;
            if (vt >= a.m_tiles) continue;
            f32x4 o[4];
            offsets(vt, o);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t tt = bn * 8 + wn * 2 + j;
                if (tt >= a.n_tiles) continue;
                float g[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) g[r] = w[j] * exp2_fast(fmaf(acc[i][j][r], f[j], o[r >> 2][r & 3]) - l2[j]);
                const int64_t at = y[j] - vt * 32;
                if (__any(at >= 0 && at < 32)) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (at == 8 * (r >> 2) + 4 * h + (r & 3)) g[r] -= w[j];
                }
                typename P::vec pl[NPL][2];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    typename P::elem e2[2];
                    to_planes<P, NPL>(g[r], e2);
#pragma unroll
                    for (int k = 0; k < NPL; ++k) pl[k][r >> 3][r & 7] = e2[k];
                }
#pragma unroll
                for (int k = 0; k < NPL; ++k) {
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        u32x4 bits = __builtin_bit_cast(u32x4, pl[k][s]);
                        bits &= keep[j];
                        pl[k][s] = __builtin_bit_cast(typename P::vec, bits);
                        *(u32x4*)(a.g + k * a.g_plane + (tt * a.ksv + vt * 2 + s) * kBlk + lane * 16) = bits;
                    }
                    f32x16 tr = {};
                    tr = P::mfma(pl[k][0], eye[0], tr);
                    tr = P::mfma(pl[k][1], eye[1], tr);
                    typename P::vec to[2];
#pragma unroll
                    for (int r = 0; r < 16; ++r) to[r >> 3][r & 7] = (typename P::elem)tr[r];
#pragma unroll
                    for (int s = 0; s < 2; ++s) *(typename P::vec*)(a.gt + k * a.gt_plane + (vt * a.kst + tt * 2 + s) * kBlk + lane * 16) = to[s];
                }
            }
        }
    }
}

// ---- ends ------------------------------------------------------------------------------------
// A wave per row: joins the (max, sum) pairs of its pieces, and takes the target's logit from x and the table.
template <class T>
__global__ __launch_bounds__(256) void k_loss(ccdpp_softmax_t p, const float2* part, int64_t pieces, float* loss, float* lse) {
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= p.t) return;
    const int lane = threadIdx.x & 63;
    float m = -INFINITY, s = 0.f;
    bool nan = false;
    for (int64_t i = lane; i < pieces; i += 64) {
        const float2 q = part[i * p.t + t];
        const float top = fmaxf(m, q.x), ref = top == -INFINITY ? 0.f : top;
        nan |= q.x != q.x || q.y != q.y;
        s = s * exp2_fast(m - ref) + q.y * exp2_fast(q.x - ref);
        m = top;
    }
    const float top = wave_max(m), ref = top == -INFINITY ? 0.f : top;
    s *= exp2_fast(m - ref);
    for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k);
    float l = top == -INFINITY ? -INFINITY : (top + log2f(s)) * kLn2;
    if (__any(nan)) l = NAN;
    const int64_t y = load_target(p.target, p.target_bits, t);
    float out = 0.f;
    if (y >= p.v) {
        out = NAN;
    } else if (y >= 0) {
        const float o = p.offset ? p.offset[y] : 0.f;
        if (o < kExcluded) {
            out = INFINITY;
        } else {
            const T *x = (const T*)p.x + t * p.ldx, *e = (const T*)p.table + y * p.ldt;
            float dot = 0.f;
            for (int d = lane; d < p.d; d += 64) dot = fmaf((float)x[d], (float)e[d], dot);
            for (int k = 32; k > 0; k >>= 1) dot += __shfl_xor(dot, k);
            out = l - fmaf(dot, p.scale, o);
        }
    }
    if (lane == 0) loss[t] = out, lse[t] = l;
}

// out = factor * sum over splits, in the caller's type and strides.
template <class T>
__global__ __launch_bounds__(256) void k_finish(const float* part, int splits, int64_t split, int64_t rows, int cols, int64_t ldp,
                                                T* out, int64_t ldo, float scale, const int32_t* fin, int which) {
    // G's power of two and the other operand's are taken off one after the other: their product may be below any float
    const float fg = fin ? ldexpf(1.f, -fin[2]) : 1.f, f = fin && which >= 0 ? ldexpf(scale, -fin[which]) : scale;
    const int64_t n = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / cols;
        const int c = (int)(i - r * cols);
        float v = 0.f;
        for (int s = 0; s < splits; ++s) v += part[s * split + r * ldp + c];
        out[r * ldo + c] = (T)(v * fg * f);
    }
}

// ---- host --------------------------------------------------------------------------------------
struct Plan {
    int planes = 1;
    bool scaled = false, scale_g = false;
    bool grads = false, forward = false;
    int64_t tt, vt, dt;      // blocks of 32
    int ksd;                 // steps of 16 over d
    int64_t kst, ksv;        // over rows, over the whole table
    int64_t vc;              // table entries per piece of the gradients (a multiple of 256)
    int sx, se;              // splits of the two gradients' contractions
    // offsets into the workspace
    int64_t o_scale, o_xrow, o_fin, o_xf, o_ef, o_o2, o_xt, o_et, o_g, o_gt, o_part, o_dx, o_de, o_lse, bytes;
};

constexpr int64_t kPieceBytes = int64_t(128) << 20;  // of G

Plan make_plan(const ccdpp_softmax_t& p, int call) {
    Plan w;
    w.grads = call != CCDPP_SOFTMAX_LOSS;
    w.forward = call != CCDPP_SOFTMAX_GRAD;
    w.planes = p.dtype == CCDPP_F32 ? 2 : 1;
    w.scaled = p.dtype == CCDPP_F32;
    w.scale_g = w.grads && p.dtype != CCDPP_BF16;
    w.tt = (p.t + 31) / 32, w.vt = (p.v + 31) / 32, w.dt = (p.d + 31) / 32;
    w.ksd = (int)w.dt * 2;
    w.kst = w.tt * 2, w.ksv = w.vt * 2;
    const int64_t row_bytes = w.tt * 32 * 2 * w.planes;
    w.vc = std::max<int64_t>(2048, kPieceBytes / std::max<int64_t>(row_bytes, 1) / 256 * 256);
    w.vc = std::min(w.vc, round_up(p.v, 256));
    const auto splits = [](int64_t m, int64_t n, int64_t kb) {
        const int64_t blocks = std::max<int64_t>(1, (m + 7) / 8 * ((n + 7) / 8));
        return (int)std::max<int64_t>(1, std::min<int64_t>({256 / blocks, kb / 8, 64}));
    };
    w.sx = splits(w.tt, w.dt, w.vc / 32);
    w.se = splits(w.vc / 32, w.dt, w.tt);
    int64_t at = 0;
    const auto take = [&](int64_t n) {
        const int64_t o = at;
        at += round_up(std::max<int64_t>(n, 0), 256);
        return o;
    };
    w.o_scale = take(3 * kParts * 4);
    w.o_fin = take(64);
    w.o_xrow = take(w.scaled ? p.t * 4 : 0);
    w.o_xf = take(w.planes * w.tt * w.ksd * kBlk);
    w.o_ef = take(w.planes * w.vt * w.ksd * kBlk);
    w.o_o2 = take(w.vt * 32 * 4);
    w.o_part = take(w.forward ? (w.vt + 7) / 8 * p.t * 8 : 0);
    if (w.grads) {
        w.o_xt = take(w.planes * w.dt * w.kst * kBlk);
        w.o_et = take(w.planes * w.dt * w.ksv * kBlk);
        w.o_g = take(w.planes * w.tt * (w.vc / 16) * kBlk);
        w.o_gt = take(w.planes * (w.vc / 32) * w.kst * kBlk);
        w.o_dx = take(p.v <= w.vc && w.sx == 1 ? 0 : w.sx * p.t * p.d * 4);
        w.o_de = take(w.se == 1 ? 0 : w.se * w.vc * p.d * 4);
    } else {
        w.o_xt = w.o_et = w.o_g = w.o_gt = w.o_dx = w.o_de = 0;
    }
    w.bytes = at;
    return w;
}

#define OPS_LAUNCH(what)                                              \
    do {                                                              \
        const hipError_t e_ = hipGetLastError();                      \
        if (e_ != hipSuccess) return hip_fail(e_, what);              \
    } while (0)

template <int DT>
int run(const ccdpp_softmax_t& p, int call, float* loss, float* lse, const float* lse_in, const float* grad, void* dx, int64_t lddx,
        void* de, int64_t ldde, char* ws, hipStream_t st) {
    typedef typename Types<DT>::in T;
    typedef typename Types<DT>::op P;
    constexpr int NPL = Types<DT>::planes;
    const Plan w = make_plan(p, call);
    Scales sc;
    sc.e_part = (float*)(ws + w.o_scale), sc.x_part = sc.e_part + kParts, sc.g_part = sc.x_part + kParts;
    sc.fin = (int32_t*)(ws + w.o_fin), sc.x_row = (int32_t*)(ws + w.o_xrow);
    const int32_t* fin = w.scaled || w.scale_g ? sc.fin : nullptr;
    if (w.scaled || w.scale_g) {
        k_scales<T><<<2 * kParts, 256, 0, st>>>(p, grad, sc, w.scaled, w.grads);
        OPS_LAUNCH("scales");
        k_scales_final<<<1, 64, 0, st>>>(sc);
        OPS_LAUNCH("scales");
    }
    PackArgs pk = {};
    pk.d = p.d, pk.ksd = w.ksd, pk.target = p.target, pk.target_bits = p.target_bits, pk.v = p.v, pk.offset = p.offset;
    pk.fin = w.scaled ? sc.fin : nullptr;
    pk.src = p.x, pk.ld = p.ldx, pk.rows = p.t, pk.ksr = w.kst, pk.which = 1;
    pk.row_exp = w.scaled ? sc.x_row : nullptr;
    pk.nat = ws + w.o_xf, pk.nat_plane = w.tt * w.ksd * kBlk;
    pk.turned = w.grads ? ws + w.o_xt : nullptr, pk.turned_plane = w.dt * w.kst * kBlk;
    k_pack<DT><<<dim3((unsigned)w.tt, (p.d + 127) / 128), 256, 0, st>>>(pk);
    OPS_LAUNCH("pack x");
    pk.src = p.table, pk.ld = p.ldt, pk.rows = p.v, pk.ksr = w.ksv, pk.which = 0, pk.row_exp = nullptr;
    pk.nat = ws + w.o_ef, pk.nat_plane = w.vt * w.ksd * kBlk;
    pk.turned = w.grads ? ws + w.o_et : nullptr, pk.turned_plane = w.dt * w.ksv * kBlk;
    pk.o2 = (float*)(ws + w.o_o2);
    k_pack<DT><<<dim3((unsigned)w.vt, (p.d + 127) / 128), 256, 0, st>>>(pk);
    OPS_LAUNCH("pack table");

    GemmArgs z = {};
    z.a = ws + w.o_ef, z.b = ws + w.o_xf;
    z.a_plane = w.vt * w.ksd * kBlk, z.b_plane = w.tt * w.ksd * kBlk;
    z.a_tile = z.b_tile = (int64_t)w.ksd * kBlk;
    z.m_tiles = w.vt, z.n_tiles = w.tt, z.kb = w.ksd / 2, z.splits = 1;
    z.t = p.t, z.v = p.v, z.scaled = w.scaled, z.x_row = sc.x_row, z.fin = fin, z.o2 = (const float*)(ws + w.o_o2);
    z.scale = p.scale, z.offset = p.offset, z.target = p.target, z.target_bits = p.target_bits;
    if (w.forward) {
        z.part = (float2*)(ws + w.o_part);
        const int64_t blocks = (w.vt + 7) / 8 * ((w.tt + 7) / 8);
        k_gemm<P, NPL, EPI_LSE, T><<<(unsigned)blocks, 512, 0, st>>>(z);
        OPS_LAUNCH("logits");
        k_loss<T><<<(unsigned)((p.t + 3) / 4), 256, 0, st>>>(p, z.part, (w.vt + 7) / 8, loss, lse);
        OPS_LAUNCH("loss");
    }
    if (!w.grads) return CCDPP_OK;
    z.lse = w.forward ? lse : lse_in, z.grad = grad;
    z.g = ws + w.o_g, z.gt = ws + w.o_gt;
    z.kst = w.kst;
    for (int64_t v0 = 0; v0 < p.v; v0 += w.vc) {
        const int64_t n = std::min(w.vc, p.v - v0), nt = (n + 31) / 32;
        GemmArgs q = z;
        q.v0 = v0, q.a = z.a + v0 / 32 * z.a_tile, q.o2 = z.o2 + v0, q.m_tiles = nt;
        q.ksv = nt * 2, q.g_plane = w.tt * q.ksv * kBlk, q.gt_plane = nt * w.kst * kBlk;
        k_gemm<P, NPL, EPI_G, T><<<(unsigned)((nt + 7) / 8 * ((w.tt + 7) / 8)), 512, 0, st>>>(q);
        OPS_LAUNCH("G");
        GemmArgs o = {};
        o.n_tiles = w.dt, o.cols = p.d, o.scale = p.scale, o.fin = fin;
        if (dx) {
            o.a = z.g, o.a_plane = q.g_plane, o.a_tile = q.ksv * kBlk, o.m_tiles = w.tt, o.rows = p.t;
            o.b = ws + w.o_et + v0 / 16 * kBlk, o.b_plane = w.dt * w.ksv * kBlk, o.b_tile = w.ksv * kBlk;
            o.kb = nt, o.splits = w.sx, o.out = (float*)(ws + w.o_dx), o.out_split = p.t * p.d, o.add = v0 > 0;
            o.which = w.scaled ? 0 : -1;
            o.last = p.v <= w.vc && w.sx == 1 ? dx : nullptr, o.ldo = o.last ? lddx : p.d;
            k_gemm<P, NPL, EPI_OUT, T><<<dim3((unsigned)((w.tt + 7) / 8 * ((w.dt + 7) / 8)), w.sx), 512, 0, st>>>(o);
            OPS_LAUNCH("dx");
        }
        if (de) {
            o.a = z.gt, o.a_plane = q.gt_plane, o.a_tile = w.kst * kBlk, o.m_tiles = nt, o.rows = n;
            o.b = ws + w.o_xt, o.b_plane = w.dt * w.kst * kBlk, o.b_tile = w.kst * kBlk;
            o.kb = w.tt, o.splits = w.se, o.out = (float*)(ws + w.o_de), o.out_split = w.vc * p.d, o.add = 0;
            o.which = w.scaled ? 1 : -1;
            o.last = w.se == 1 ? (T*)de + v0 * ldde : nullptr, o.ldo = o.last ? ldde : p.d;
            k_gemm<P, NPL, EPI_OUT, T><<<dim3((unsigned)((nt + 7) / 8 * ((w.dt + 7) / 8)), w.se), 512, 0, st>>>(o);
            OPS_LAUNCH("dtable");
            if (!o.last) {
                k_finish<T><<<2048, 256, 0, st>>>(o.out, w.se, o.out_split, n, p.d, p.d, (T*)de + v0 * ldde, ldde, p.scale, fin, o.which);
                OPS_LAUNCH("dtable");
            }
        }
    }
    if (dx && !(p.v <= w.vc && w.sx == 1)) {
        k_finish<T><<<2048, 256, 0, st>>>((const float*)(ws + w.o_dx), w.sx, p.t * p.d, p.t, p.d, p.d, (T*)dx, lddx, p.scale, fin, w.scaled ? 0 : -1);
        OPS_LAUNCH("dx");
    }
    return CCDPP_OK;
}

int check(const ccdpp_softmax_t* p, bool pointers) {
    constexpr int64_t kMax = (int64_t(1) << 31) - 256;
    if (!p) return fail(CCDPP_EINVAL, "the problem is NULL");
    if (p->t < 0 || p->t >= kMax) return fail(CCDPP_EINVAL, "t must be in [0, 2^31 - 256)");
    if (p->v < 1 || p->v >= kMax) return fail(CCDPP_EINVAL, "v must be in [1, 2^31 - 256)");
    if (p->d < 1 || p->d > 65536) return fail(CCDPP_EINVAL, "d must be in [1, 65536]");
    if (p->dtype < CCDPP_F32 || p->dtype > CCDPP_F16) return fail(CCDPP_EINVAL, "dtype must be CCDPP_F32, CCDPP_BF16 or CCDPP_F16");
    if (p->ldx < p->d || p->ldt < p->d) return fail(CCDPP_EINVAL, "ldx and ldt must be at least d");
    if ((double)p->t * (double)p->v >= 549755813888.0) return fail(CCDPP_EINVAL, "t * v must be below 2^39: take fewer rows at a time");
    if (p->target_bits != 32 && p->target_bits != 64) return fail(CCDPP_EINVAL, "target_bits must be 32 or 64");
    if (!std::isfinite(p->scale)) return fail(CCDPP_EINVAL, "scale must be finite");
    if (pointers && (!p->table || (p->t > 0 && (!p->x || !p->target)))) return fail(CCDPP_EINVAL, "x, table and target must be non-NULL");
    return CCDPP_OK;
}

int call(const ccdpp_softmax_t* p, int what, float* loss, float* lse, const float* lse_in, const float* grad, void* dx, int64_t lddx,
         void* de, int64_t ldde, void* ws, int64_t ws_bytes, void* stream) {
    if (int rc = check(p, true)) return rc;
    if (what != CCDPP_SOFTMAX_GRAD && p->t > 0 && (!loss || !lse)) return fail(CCDPP_EINVAL, "loss and lse must be non-NULL");
    if (what == CCDPP_SOFTMAX_GRAD && p->t > 0 && !lse_in) return fail(CCDPP_EINVAL, "lse must be non-NULL");
    if (what != CCDPP_SOFTMAX_LOSS && ((dx && lddx < p->d) || (de && ldde < p->d))) return fail(CCDPP_EINVAL, "lddx and lddt must be at least d");
    const Plan w = make_plan(*p, what);
    if (ws_bytes < w.bytes || (!ws && w.bytes > 0)) return fail(CCDPP_EINVAL, "the workspace is too small");
    if ((uintptr_t)ws % 256) return fail(CCDPP_EINVAL, "the workspace must be aligned to 256 bytes");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    if (p->t == 0) {
        if (what != CCDPP_SOFTMAX_LOSS && de) {  // no rows: the table's gradient is zero
            const int es = p->dtype == CCDPP_F32 ? 4 : 2;
            if (es == 4) k_finish<float><<<2048, 256, 0, st>>>(nullptr, 0, 0, p->v, p->d, p->d, (float*)de, ldde, 0.f, nullptr, -1);
            else k_finish<_Float16><<<2048, 256, 0, st>>>(nullptr, 0, 0, p->v, p->d, p->d, (_Float16*)de, ldde, 0.f, nullptr, -1);
            OPS_LAUNCH("dtable");
        }
        return CCDPP_OK;
    }
    switch (p->dtype) {
        case CCDPP_F32: return run<CCDPP_F32>(*p, what, loss, lse, lse_in, grad, dx, lddx, de, ldde, (char*)ws, st);
        case CCDPP_BF16: return run<CCDPP_BF16>(*p, what, loss, lse, lse_in, grad, dx, lddx, de, ldde, (char*)ws, st);
        default: return run<CCDPP_F16>(*p, what, loss, lse, lse_in, grad, dx, lddx, de, ldde, (char*)ws, st);
    }
}

}  // namespace
}  // namespace ccdops

extern "C" {

int ccdpp_softmax_workspace(const ccdpp_softmax_t* p, int32_t call, int64_t* bytes) {
    using namespace ccdops;
    if (int rc = check(p, false)) return rc;
    if (call < CCDPP_SOFTMAX_LOSS || call > CCDPP_SOFTMAX_TRAIN) return fail(CCDPP_EINVAL, "call must be one of enum ccdpp_softmax_call");
    if (!bytes) return fail(CCDPP_EINVAL, "bytes is NULL");
    *bytes = make_plan(*p, call).bytes;
    return CCDPP_OK;
}

int ccdpp_softmax_loss(const ccdpp_softmax_t* p, float* loss, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    return ccdops::call(p, CCDPP_SOFTMAX_LOSS, loss, lse, nullptr, nullptr, nullptr, 0, nullptr, 0, workspace, workspace_bytes, stream);
}

int ccdpp_softmax_loss_grad(const ccdpp_softmax_t* p, const float* lse, const float* grad, void* dx, int64_t lddx, void* dtable,
                            int64_t lddt, void* workspace, int64_t workspace_bytes, void* stream) {
    return ccdops::call(p, CCDPP_SOFTMAX_GRAD, nullptr, nullptr, lse, grad, dx, lddx, dtable, lddt, workspace, workspace_bytes, stream);
}

int ccdpp_softmax_loss_train(const ccdpp_softmax_t* p, float* loss, float* lse, const float* grad, void* dx, int64_t lddx, void* dtable,
                             int64_t lddt, void* workspace, int64_t workspace_bytes, void* stream) {
    return ccdops::call(p, CCDPP_SOFTMAX_TRAIN, loss, lse, nullptr, grad, dx, lddx, dtable, lddt, workspace, workspace_bytes, stream);
}

}  // extern "C"
