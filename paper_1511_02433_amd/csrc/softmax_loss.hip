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
    const int32_t *x_row, *fin;  // exponents (32-bit inputs), or NULL
    float scale;
    const float* offset;
    float2* part;                // [blocks of 256 table entries][t] (max, sum), base 2
    const void* target;
    int target_bits;
    const float *lse, *grad;
    char *g, *gt;                // G [plane][t/32][ksv], G^T [plane][v/32][kst] fragments
    int64_t g_plane, gt_plane;
    int64_t ksv, kst;
    // other products
    float* out;                  // [split][M][ldo]
    int64_t out_split, rows, cols, ldo;
    int add;
};

template <class P, int NPL, int EPI>
__global__ __launch_bounds__(512) void k_gemm(GemmArgs a) {
    constexpr int NSEG = NPL == 2 ? 3 : 1;
    __shared__ __align__(16) char lds[2][16][kBlk];  // A, B: 8 blocks of 32 rows x 2 steps
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave >> 2, wn = wave & 3;
    const int64_t mb = (a.m_tiles + 7) / 8;
    const int64_t bm = blockIdx.x % mb, bn = blockIdx.x / mb;
    const int split = blockIdx.y;
    const int64_t k0 = a.kb * split / a.splits, k1 = a.kb * (split + 1) / a.splits;
    f32x16 acc[4][2];
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 2; ++j)
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    const int64_t am = min(bm * 8 + wave, a.m_tiles - 1), bt = min(bn * 8 + wave, a.n_tiles - 1);
    for (int seg = 0; seg < NSEG; ++seg) {
        const char* pa = a.a + (seg == 2 ? a.a_plane : 0) + am * a.a_tile + lane * 16;
        const char* pb = a.b + (seg == 1 ? a.b_plane : 0) + bt * a.b_tile + lane * 16;
        for (int64_t k = k0; k < k1; ++k) {
            const u32x4 a0 = *(const u32x4*)(pa + k * 2 * kBlk), a1 = *(const u32x4*)(pa + k * 2 * kBlk + kBlk);
            const u32x4 b0 = *(const u32x4*)(pb + k * 2 * kBlk), b1 = *(const u32x4*)(pb + k * 2 * kBlk + kBlk);
            __syncthreads();
            *(u32x4*)&lds[0][wave * 2][lane * 16] = a0;
            *(u32x4*)&lds[0][wave * 2 + 1][lane * 16] = a1;
            *(u32x4*)&lds[1][wave * 2][lane * 16] = b0;
            *(u32x4*)&lds[1][wave * 2 + 1][lane * 16] = b1;
            __syncthreads();
            for (int s = 0; s < 2; ++s) {
                typename P::vec fa[4], fb[2];
                for (int i = 0; i < 4; ++i) fa[i] = *(const typename P::vec*)&lds[0][(wm * 4 + i) * 2 + s][lane * 16];
                for (int j = 0; j < 2; ++j) fb[j] = *(const typename P::vec*)&lds[1][(wn * 2 + j) * 2 + s][lane * 16];
                for (int i = 0; i < 4; ++i)
                    for (int j = 0; j < 2; ++j) acc[i][j] = P::mfma(fa[i], fb[j], acc[i][j]);
            }
        }
    }
    const int n = lane & 31, h = lane >> 5;
    if constexpr (EPI == EPI_OUT) {
        float* out = a.out + split * a.out_split;
        for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 2; ++j) {
                const int64_t col = (bn * 8 + wn * 2 + j) * 32 + n;
                if (col >= a.cols) continue;
                for (int r = 0; r < 16; ++r) {
                    const int64_t row = (bm * 8 + wm * 4 + i) * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                    if (row >= a.rows) continue;
                    float* o = out + row * a.ldo + col;
                    *o = a.add ? *o + acc[i][j][r] : acc[i][j][r];
                }
            }
        return;
    }
    // Logits in base 2; excluded and missing entries are -inf.
    const int ee = a.fin ? a.fin[0] : 0;
    if constexpr (EPI == EPI_LSE) {
        __shared__ float2 share[2][256];
        for (int j = 0; j < 2; ++j) {
            const int64_t t = (bn * 8 + wn * 2 + j) * 32 + n;
            const int xe = a.x_row && t < a.t ? a.x_row[t] : 0;
            const float f = ldexpf(a.scale * kLog2e, -(xe + ee));
            float top = -INFINITY;
            for (int i = 0; i < 4; ++i)
                for (int r = 0; r < 16; ++r) {
                    const int64_t v = a.v0 + (bm * 8 + wm * 4 + i) * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                    float z = -INFINITY;
                    if (v < a.v) {
                        const float o = a.offset ? a.offset[v] : 0.f;
                        if (!(o < kExcluded)) z = fmaf(acc[i][j][r], f, o * kLog2e);
                    }
                    acc[i][j][r] = z;
                    top = fmaxf(top, z);
                }
            float sum = 0.f;
            const float ref = top == -INFINITY ? 0.f : top;
            for (int i = 0; i < 4; ++i)
                for (int r = 0; r < 16; ++r) sum += exp2_fast(acc[i][j][r] - ref);
            const float top2 = __shfl_xor(top, 32), sum2 = __shfl_xor(sum, 32);
            const float m = fmaxf(top, top2);
            const float mr = m == -INFINITY ? 0.f : m;
            sum = sum * exp2_fast(top - mr) + sum2 * exp2_fast(top2 - mr);
            if (h == 0) share[wm][(wn * 2 + j) * 32 + n] = make_float2(m, sum);
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
        for (int s = 0; s < 2; ++s)
            for (int k = 0; k < 8; ++k) {
                const int v = 16 * s + (k < 4 ? 4 * h + k : 8 + 4 * h + k - 4);
                eye[s][k] = (typename P::elem)(v == n ? 1.f : 0.f);
            }
        for (int j = 0; j < 2; ++j) {
            const int64_t tt = bn * 8 + wn * 2 + j, t = tt * 32 + n;
            if (tt >= a.n_tiles) continue;
            float w = 0.f, l2 = 0.f, f = 0.f;
            int64_t y = -1;
            if (t < a.t) {
                y = load_target(a.target, a.target_bits, t);
                const int xe = a.x_row ? a.x_row[t] : 0;
                f = ldexpf(a.scale * kLog2e, -(xe + ee));
                if (row_counts(y, a.v, a.offset)) {
                    w = a.grad ? a.grad[t] : 1.f;
                    if (a.fin) w = ldexpf(w, a.fin[2]);
                    if (y >= a.v) w = NAN;
                    l2 = a.lse[t] * kLog2e;
                }
            }
            const bool dead = t >= a.t || !row_counts(y, a.v, a.offset);
            for (int i = 0; i < 4; ++i) {
                const int64_t vt = bm * 8 + wm * 4 + i;
                if (vt >= a.m_tiles) continue;
                typename P::vec hi[NPL][2];
                for (int r = 0; r < 16; ++r) {
                    const int64_t v = a.v0 + vt * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                    float g = 0.f;
                    if (v < a.v && !dead) {
                        const float o = a.offset ? a.offset[v] : 0.f;
                        const float pr = o < kExcluded ? 0.f : exp2_fast(fmaf(acc[i][j][r], f, o * kLog2e) - l2);
                        g = w * (pr - (v == y ? 1.f : 0.f));
                    }
                    typename P::elem o2[2];
                    to_planes<P, NPL>(g, o2);
                    for (int pl = 0; pl < NPL; ++pl) hi[pl][r >> 3][r & 7] = o2[pl];
                }
                for (int pl = 0; pl < NPL; ++pl) {
                    char* g = a.g + pl * a.g_plane + (tt * a.ksv + vt * 2) * kBlk + lane * 16;
                    *(typename P::vec*)g = hi[pl][0];
                    *(typename P::vec*)(g + kBlk) = hi[pl][1];
                    f32x16 tr;
                    for (int r = 0; r < 16; ++r) tr[r] = 0.f;
                    tr = P::mfma(hi[pl][0], eye[0], tr);
                    tr = P::mfma(hi[pl][1], eye[1], tr);
                    typename P::vec o[2];
                    for (int r = 0; r < 16; ++r) o[r >> 3][r & 7] = (typename P::elem)tr[r];
                    char* gt = a.gt + pl * a.gt_plane + (vt * a.kst + tt * 2) * kBlk + lane * 16;
                    *(typename P::vec*)gt = o[0];
                    *(typename P::vec*)(gt + kBlk) = o[1];
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
    int64_t o_scale, o_xrow, o_fin, o_xf, o_ef, o_xt, o_et, o_g, o_gt, o_part, o_dx, o_de, o_lse, bytes;
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
    w.o_part = take(w.forward ? (w.vt + 7) / 8 * p.t * 8 : 0);
    if (w.grads) {
        w.o_xt = take(w.planes * w.dt * w.kst * kBlk);
        w.o_et = take(w.planes * w.dt * w.ksv * kBlk);
        w.o_g = take(w.planes * w.tt * (w.vc / 16) * kBlk);
        w.o_gt = take(w.planes * (w.vc / 32) * w.kst * kBlk);
        w.o_dx = take(w.sx * p.t * p.d * 4);
        w.o_de = take(w.se * w.vc * p.d * 4);
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
    k_pack<DT><<<dim3((unsigned)w.vt, (p.d + 127) / 128), 256, 0, st>>>(pk);
    OPS_LAUNCH("pack table");

    GemmArgs z = {};
    z.a = ws + w.o_ef, z.b = ws + w.o_xf;
    z.a_plane = w.vt * w.ksd * kBlk, z.b_plane = w.tt * w.ksd * kBlk;
    z.a_tile = z.b_tile = (int64_t)w.ksd * kBlk;
    z.m_tiles = w.vt, z.n_tiles = w.tt, z.kb = w.ksd / 2, z.splits = 1;
    z.t = p.t, z.v = p.v, z.x_row = w.scaled ? sc.x_row : nullptr, z.fin = fin;
    z.scale = p.scale, z.offset = p.offset, z.target = p.target, z.target_bits = p.target_bits;
    // the table's exponent is part of the logits' factor for 32-bit inputs alone
    if (w.forward) {
        z.part = (float2*)(ws + w.o_part);
        GemmArgs f = z;
        if (!w.scaled) f.fin = nullptr;
        const int64_t blocks = (w.vt + 7) / 8 * ((w.tt + 7) / 8);
        k_gemm<P, NPL, EPI_LSE><<<(unsigned)blocks, 512, 0, st>>>(f);
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
        q.v0 = v0, q.a = z.a + v0 / 32 * z.a_tile, q.m_tiles = nt;
        q.ksv = nt * 2, q.g_plane = w.tt * q.ksv * kBlk, q.gt_plane = nt * w.kst * kBlk;
        k_gemm<P, NPL, EPI_G><<<(unsigned)((nt + 7) / 8 * ((w.tt + 7) / 8)), 512, 0, st>>>(q);
        OPS_LAUNCH("G");
        GemmArgs o = {};
        o.n_tiles = w.dt, o.cols = o.ldo = p.d;
        if (dx) {
            o.a = z.g, o.a_plane = q.g_plane, o.a_tile = q.ksv * kBlk, o.m_tiles = w.tt, o.rows = p.t;
            o.b = ws + w.o_et + v0 / 16 * kBlk, o.b_plane = w.dt * w.ksv * kBlk, o.b_tile = w.ksv * kBlk;
            o.kb = nt, o.splits = w.sx, o.out = (float*)(ws + w.o_dx), o.out_split = p.t * p.d, o.add = v0 > 0;
            k_gemm<P, NPL, EPI_OUT><<<dim3((unsigned)((w.tt + 7) / 8 * ((w.dt + 7) / 8)), w.sx), 512, 0, st>>>(o);
            OPS_LAUNCH("dx");
        }
        if (de) {
            o.a = z.gt, o.a_plane = q.gt_plane, o.a_tile = w.kst * kBlk, o.m_tiles = nt, o.rows = n;
            o.b = ws + w.o_xt, o.b_plane = w.dt * w.kst * kBlk, o.b_tile = w.kst * kBlk;
            o.kb = w.tt, o.splits = w.se, o.out = (float*)(ws + w.o_de), o.out_split = w.vc * p.d, o.add = 0;
            k_gemm<P, NPL, EPI_OUT><<<dim3((unsigned)((nt + 7) / 8 * ((w.dt + 7) / 8)), w.se), 512, 0, st>>>(o);
            OPS_LAUNCH("dtable");
            k_finish<T><<<2048, 256, 0, st>>>(o.out, w.se, o.out_split, n, p.d, p.d, (T*)de + v0 * ldde, ldde, p.scale, fin, w.scaled ? 1 : -1);
            OPS_LAUNCH("dtable");
        }
    }
    if (dx) {
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
