// Softmax cross entropy of rows against a whole table, and its gradients, without keeping all logits (gfx950).
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
// planes, hi + lo, under powers of two (each row's own for the logits, the matrix's for the gradients); a product of such matrices is the three products hi hi + hi lo +
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

#include "softmax_device.hpp"

namespace ccdops {
namespace {

// ---- scales of 32-bit inputs ----------------------------------------------------------
// Exponents of the powers of two that x's rows and the table's (their own, for the logits; one for all that count, for the
// gradients) and the rows' weights are multiplied with.  Only finite values count.
constexpr int kParts = 256;  // blocks of k_scales, and partial maxima of each quantity

struct Scales {
    float *e_part, *x_part, *g_part;  // [kParts] largest |table| (excluded items apart), |x| of rows that count, |grad|
    float* n_part;                    // [kParts] largest 2-norm of a row of x (few factors)
    float *x_row, *e_row;             // [t], [v] largest |value| of each row; e_row: NULL where it is not asked for
    int32_t* fin;                     // [4] exponents: table, x, G; kUnit, kFactor or kOwn (few factors)
};

template <class T>
__device__ __forceinline__ float abs_finite(T v) {
    const float a = fabsf((float)v);
    return finite(a) ? a : 0.f;
}

// Largest finite |value| of `n` values from `lane` of `lanes` threads, eight reads in flight.
template <class T>
__device__ __forceinline__ float run_max(const T* at, int64_t n, int64_t lane, int64_t lanes) {
    constexpr int N = 16 / sizeof(T), U = 4;
    float m = 0.f;
    const int64_t whole = n / N;
    for (int64_t i = lane; i < whole; i += lanes * U) {
        Run<T, N> q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = load_run<N>(at + min(i + u * lanes, whole - 1) * N);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < N; ++j) m = fmaxf(m, abs_finite(q[u].v[j]));
    }
    for (int64_t i = whole * N + lane; i < n; i += lanes) m = fmaxf(m, abs_finite(at[i]));
    return m;
}

// Largest value over the lanes (16 or 64) that share a row.
__device__ __forceinline__ float lanes_max(float m, int lanes) {
    for (int k = lanes / 2; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    return m;
}

// The table and x (where `mats` is set), 16 lanes a row or 64 where it is long (the table in one run where its rows are not
// asked for, no items are excluded and rows follow one another), and the rows' weights (`grads`).  Bound by reading both
// once (131,072 x 4,096 in bfloat16 and 8,192 rows: 211 us, 5.4 TB/s).  The logits of wide 32-bit rows take a power of two
// from each row; what is contracted over rows (the turned matrices) one from the whole matrix.
template <class T>
__global__ __launch_bounds__(1024) void k_scales(ccdpp_softmax_t p, const float* grad, Scales sc, int mats, int norms, int grads) {
    __shared__ float red[16][4];
    float em = 0.f, xm = 0.f, gm = 0.f, nm = 0.f;
    if (mats) {
        const int lanes = p.d > (sc.e_row ? 1024 : 256) ? 64 : 16, l = threadIdx.x & (lanes - 1), per = 1024 / lanes;
        const int64_t first = (int64_t)blockIdx.x * per + threadIdx.x / lanes, stride = (int64_t)kParts * per;
        if (!sc.e_row && !p.offset && p.ldt == p.d) {
            em = run_max((const T*)p.table, p.v * p.d, (int64_t)blockIdx.x * 1024 + threadIdx.x, (int64_t)kParts * 1024);
        } else {
            for (int64_t v = first; v < p.v; v += stride) {
                float m = 0.f;
                if (!p.offset || !(p.offset[v] < kExcluded)) m = run_max((const T*)p.table + v * p.ldt, p.d, l, lanes);
                em = fmaxf(em, m);
                if (sc.e_row) {
                    m = lanes_max(m, lanes);
                    if (l == 0) sc.e_row[v] = m;
                }
            }
        }
        for (int64_t t = first; t < p.t; t += stride) {
            const T* const row = (const T*)p.x + t * p.ldx;
            const float m = lanes_max(run_max(row, p.d, l, lanes), lanes);
            if (norms) {
                double s = 0.0;
                for (int i = l; i < p.d; i += lanes) s += (double)abs_finite(row[i]) * (double)abs_finite(row[i]);
                for (int k = lanes / 2; k > 0; k >>= 1) s += __shfl_xor(s, k);
                nm = fmaxf(nm, (float)sqrt(s));
            }
            if (l == 0) sc.x_row[t] = m;
            if (row_counts(load_target(p.target, p.target_bits, t), p.v, p.offset)) xm = fmaxf(xm, m);
        }
    }
    if (grads)
        for (int64_t t = (int64_t)blockIdx.x * 1024 + threadIdx.x; t < p.t; t += (int64_t)kParts * 1024)
            if (row_counts(load_target(p.target, p.target_bits, t), p.v, p.offset)) gm = fmaxf(gm, grad ? abs_finite(grad[t]) : 1.f);
    em = wave_max(em), xm = wave_max(xm), gm = wave_max(gm), nm = wave_max(nm);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) red[wave][0] = em, red[wave][1] = xm, red[wave][2] = gm, red[wave][3] = nm;
    __syncthreads();
    if (wave < 4) {  // a wave each
        const float m = wave_max(lane < 16 ? red[lane][wave] : 0.f);
        if (lane == 0) (wave == 0 ? sc.e_part : wave == 1 ? sc.x_part : wave == 2 ? sc.g_part : sc.n_part)[blockIdx.x] = m;
    }
}

// Largest of kParts partial maxima of each quantity that is asked for (0 for the others), by 256 threads, with one round
// trip to memory.
struct Tops {
    float e, x, g, n;
};
__device__ __forceinline__ Tops parts_max(const Scales& sc, bool want_e, bool want_x, bool want_g, bool want_n, float (*red)[4]) {
    const int i = threadIdx.x, wave = i >> 6;
    Tops top = {want_e ? sc.e_part[i] : 0.f, want_x ? sc.x_part[i] : 0.f, want_g ? sc.g_part[i] : 0.f, want_n ? sc.n_part[i] : 0.f};
    if (want_e) top.e = wave_max(top.e);
    if (want_x) top.x = wave_max(top.x);
    if (want_g) top.g = wave_max(top.g);
    if (want_n) top.n = wave_max(top.n);
    if ((i & 63) == 0) red[wave][0] = top.e, red[wave][1] = top.x, red[wave][2] = top.g, red[wave][3] = top.n;
    __syncthreads();
    const auto of = [&](int k) { return fmaxf(fmaxf(red[0][k], red[1][k]), fmaxf(red[2][k], red[3][k])); };
    if (want_e) top.e = of(0);
    if (want_x) top.x = of(1);
    if (want_g) top.g = of(2);
    if (want_n) top.n = of(3);
    return top;
}

// ---- operands in fragment order ----------------------------------------------------------
// Where the fragments of one matrix go; pointers that are NULL are not written.
struct PackSide {
    const void* src;
    int64_t ld, rows, tiles;                  // tiles: blocks of 32 rows
    char* nat;                                // the matrix as it is
    int64_t nat_row, nat_plane;               // bytes per block of 32 rows, per plane
    char* live;                               // the same with rows that do not count zeroed (x)
    int64_t live_row;
    char* turned;                             // its transpose, without the rows that do not count
    int64_t turned_row, turned_d, turned_plane;  // per block of 32 rows, per block of 32 columns, per plane
    char *num, *live_num;                     // numbers of the first 32 rows (see softmax_device.hpp; `num`: the first one only)
    int64_t num_row, live_num_row;
    char* exps;                               // the table's kNumExp, num_row apart (32-bit values)
};
struct PackArgs {
    PackSide x, e;
    Scales sc;
    int scaled;    // e_part and x_part hold: the turned matrices (and 32-bit ones as they are) get powers of two
    int weights;   // g_part holds
    int d, ksd;    // ksd: steps of 16 over d
    const void* target;
    int target_bits;
    int64_t v;
    float scale;
    const float* offset;
    const float* grad;
};

// One block: 32 rows x 128 columns, blocks of x first.  A wave takes 16 columns at a time: a lane's 8 values of a
// fragment are 8 neighbours in memory; the turned ones are picked out of LDS.  Bound by memory: it reads a matrix once
// and writes it twice (131,072 x 4,096 in bfloat16 and 8,192 rows: 709 us, 4.9 TB/s), so that every later access is a
// whole fragment of 1 KB, whatever the inputs' strides and alignment are.
template <int DT, bool SMALL>
__global__ __launch_bounds__(256) void k_pack(PackArgs a) {
    typedef typename Types<DT>::in T;
    typedef typename Types<DT>::op P;
    typedef typename std::conditional<SMALL, P, typename Types<DT>::turned>::type PT;
    constexpr int NPL = Types<DT>::planes;
    constexpr int kPitch = 128 + 16 / sizeof(T);
    __shared__ __align__(16) T tile[32][kPitch];
    __shared__ float live[32], red[4][4], tops[4][32];
    __shared__ int exps[32];
    const bool is_x = blockIdx.x < a.x.tiles;
    const PackSide& side = is_x ? a.x : a.e;
    const int64_t rt = is_x ? blockIdx.x : blockIdx.x - a.x.tiles, r0 = rt * 32;
    const int c0 = blockIdx.y * 128;
    // All that is read, before the first wait.
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 31, h = lane >> 5;
    const int64_t row = r0 + m;
    const bool in = row < side.rows;
    const T* const src = (const T*)side.src + row * side.ld;
    Run<T, 8> held[2] = {};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int s = wave + 4 * k;
        if (in && c0 / 16 + s < a.ksd) held[k] = load_tail<8>(src, c0 + 16 * s + 8 * h, a.d, (side.rows - 1 - row) * side.ld + a.d);
    }
    const int64_t r = r0 + threadIdx.x;  // of the first 32 threads
    bool row_in = threadIdx.x < 32 && r < side.rows, row_live = row_in, negative = false;
    float row_top = 0.f, row_offset = 0.f;
    if (NPL == 2 && row_in && (is_x || a.sc.e_row)) row_top = (is_x ? a.sc.x_row : a.sc.e_row)[r];
    if (row_in && is_x) {
        if (side.live && a.grad) negative = a.grad[r] < 0.f;
        row_live = row_counts(load_target(a.target, a.target_bits, r), a.v, a.offset);
    } else if (row_in && a.offset) {
        row_offset = a.offset[r];
        row_live = !(row_offset < kExcluded);
    }
    // 32-bit rows of x are multiplied with scale and log2 e before they are split.
    const float before = NPL == 2 ? a.scale * kLog2e : 1.f;
    int exp = 0, unit = 0;  // powers of two of the turned matrix, and of the table as it is
    int way = kOwn;         // of 32-bit rows
    const bool leaves = blockIdx.x == 0 && blockIdx.y == 0;  // the exponents
    if (a.scaled || (leaves && a.weights)) {
        const Tops top = parts_max(a.sc, a.scaled, a.scaled && (is_x || leaves), leaves && a.weights, SMALL && NPL == 2, red);
        if constexpr (SMALL && NPL == 2) {
            unit = unit_exp(top.e);
            const float norm = top.n * fabsf(before) * pow2i(-unit);
            way = norm <= kUnitNorm ? kUnit : norm <= kFactorNorm ? kFactor : kOwn;
            if (way == kFactor) unit = scale_exp(top.e);
            if (leaves && threadIdx.x == 0) a.sc.fin[3] = way;
            if (way == kOwn && !is_x) {  // (all columns are here)
                float most = 0.f;
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) most = fmaxf(most, abs_finite(held[k].v[j]));
                most = fmaxf(most, __shfl_xor(most, 32));
                if (h == 0) tops[wave][m] = most;
                __syncthreads();
                if (threadIdx.x < 32) row_top = fmaxf(fmaxf(tops[0][threadIdx.x], tops[1][threadIdx.x]), fmaxf(tops[2][threadIdx.x], tops[3][threadIdx.x]));
            }
        }
        exp = a.scaled ? scale_exp(is_x ? top.x : top.e) : 0;
        // G lies within its row's weight, or a few times that where lse is the caller's own: two bits are left for it.
        if (leaves && threadIdx.x == 0) a.sc.fin[0] = scale_exp(top.e), a.sc.fin[1] = scale_exp(top.x), a.sc.fin[2] = scale_exp(top.g) - 2;
    }
    if (threadIdx.x < 32) {
        if (is_x) {
            const int e = way == kUnit ? -unit : scale_exp(row_top * fabsf(before));
            float f = row_in ? a.scale * kLog2e : 0.f;
            if (NPL == 2) f = way == kOwn ? __int_as_float(-e) : way == kFactor ? ldexpf(1.f, -(e + unit)) : 1.f;
            exps[threadIdx.x] = e;
            if (blockIdx.y == 0) {
                if (side.num) *(float*)(side.num + rt * side.num_row + (kNumFactor * 32 + threadIdx.x) * 4) = f;
                if (side.live_num) {  // rows that count get the rest once their lse is there
                    float* o = (float*)(side.live_num + rt * side.live_num_row) + threadIdx.x;
                    o[kNumFactor * 32] = row_live ? f : 0.f;
                    o[kNumTerm * 32] = o[kNumLse * 32] = -INFINITY;
                    o[kNumWeight * 32] = o[kNumRaw * 32] = 0.f;
                    o[kNumTarget * 32] = __int_as_float(-1);
                }
            }
        } else {
            const int e = way == kOwn ? scale_exp(row_top) : unit;
            exps[threadIdx.x] = e;
            if (blockIdx.y == 0 && side.num) *(float*)(side.num + rt * side.num_row + (kNumOffset * 32 + threadIdx.x) * 4) = row_live ? row_offset * kLog2e : -INFINITY;
            if (NPL == 2 && way == kOwn && blockIdx.y == 0 && side.exps) *(int*)(side.exps + rt * side.num_row + threadIdx.x * 4) = -e;
        }
        // Terms of few factors are exponentials, with no sign: a negative weight's is taken into the turned row.
        live[threadIdx.x] = !row_live ? 0.f : negative ? -1.f : 1.f;
    }
    __syncthreads();
    const float mul = NPL == 2 ? pow2i(exps[m]) : 1.f, mul_t = pow2i(exp);
    const bool counts = live[m] != 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int s = wave + 4 * k, ks = c0 / 16 + s;
        if (ks >= a.ksd) break;
        T* const v = held[k].v;
        if (!is_x && !counts)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (T)0.f;
        if (side.turned) {
            struct alignas(16) Eight { T v[8]; } to;
#pragma unroll
            for (int j = 0; j < 8; ++j) to.v[j] = counts ? (live[m] < 0.f ? (T)(-(float)v[j]) : v[j]) : (T)0.f;
            *(Eight*)&tile[m][16 * s + 8 * h] = to;
        }
        typename P::elem o[8][2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (NPL == 2) to_planes<P, NPL>((is_x ? (float)v[j] * before : (float)v[j]) * mul, o[j]);
            else o[j][0] = (typename P::elem)v[j];
        }
#pragma unroll
        for (int pl = 0; pl < NPL; ++pl) {
            typename P::vec w;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = o[j][pl];
            const int64_t at = pl * side.nat_plane + (int64_t)ks * kBlk + lane * 16;
            if (side.nat) *(typename P::vec*)(side.nat + rt * side.nat_row + at) = w;
            if (side.live) {
                const typename P::vec none = {};
                *(typename P::vec*)(side.live + rt * side.live_row + at) = counts ? w : none;
            }
        }
    }
    if (!side.turned) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = wave + 4 * k, dt = i >> 1, s = i & 1;  // 4 blocks of 32 columns x 2 steps of 16 rows
        if (c0 + dt * 32 >= a.d) break;
        typename PT::elem o[8][2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = 16 * s + (j < 4 ? 4 * h + j : 8 + 4 * h + j - 4);
            // columns past d were not written by a fragment if they start a new one
            const T v = c0 + dt * 32 + m < a.d ? tile[r][dt * 32 + m] : (T)0.f;
            if constexpr (std::is_same<T, typename PT::elem>::value) o[j][0] = v;
            else to_planes<PT, NPL>((float)v * mul_t, o[j]);
        }
#pragma unroll
        for (int pl = 0; pl < NPL; ++pl) {
            typename PT::vec w;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = o[j][pl];
            *(typename PT::vec*)(side.turned + pl * side.turned_plane + (int64_t)(c0 / 32 + dt) * side.turned_d + rt * side.turned_row +
                                 s * kBlk + lane * 16) = w;
        }
    }
}

// ---- the product -----------------------------------------------------------------------------
// C (M x N) = A (M x K) B (N x K)^T from fragments: 256 x 256 of C per block, eight waves of 128 x 64, since a wave then
// needs 6 KB of fragments for 8 products (a square of 64 x 64 4 KB for 4: LDS would bound it).  Four stages of LDS
// (128 KB) are filled directly, three ahead.  Bound by the matrix cores at the clock that their power leaves (1.5 to
// 2.1 GHz): logits of 8,192 x 131,072 x 4,096 in bfloat16 7.3 ms (1.21 PFLOP/s), their G 1.84 ms and either gradient
// 1.78 ms per 32,768 entries (1.19 and 1.24 PFLOP/s; a large library product reaches 1.35); 2,000 x 32,003 x 1,024 in 32
// bits (three products) 358 us, 1.10 PFLOP/s.
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
    const int32_t* fin;          // exponents; NULL where nothing is scaled
    const float* xf;             // factor of each row's accumulated logits (32-bit values: an exponent)
    const int* ek;               // exponents of A's rows (32-bit values)
    float scale;
    const float* offset;
    const float* o2;             // offsets of A's rows in base 2, -inf for excluded and missing ones
    float2* part;                // [blocks of 256 table entries][t] (max, sum), base 2
    float* kept;                 // logits of the first kept_tiles blocks of 32 entries [t/32][block][32 x 32, as in an accumulator]
    int64_t kept_tiles;
    const void* target;
    int target_bits;
    const float *lse, *grad;
    char *g, *gt;                // G [plane][t/32][ksv], G^T [plane][v/32][kst] fragments, or NULL
    int64_t g_plane, gt_plane;
    int64_t ksv, kst;
    uint8_t* lev;                // powers of two of G^T's items, of 64 rows each: [v/32][t/64][32]
    int* item_e;                 // those of all rows, [v/32][32]
    // other products
    float* out;                  // [split][N][ldo]: of a gradient's rows; M are its columns
    void* last;                  // or the result itself
    int wide;                    // its rows are aligned to four values
    int64_t out_split, rows, cols, ldo;
    int add, which;              // which: the exponent in fin of the other operand, or -1
    int own;                     // whether the rows' terms have powers of two of their own: kRowsOwn (from grad), kItemsOwn (item_e)
};
enum { kNoneOwn = 0, kRowsOwn = 1, kItemsOwn = 2 };

constexpr int kStages = 4;          // of LDS
constexpr int kStage = 32 * kBlk;

// Terms are held in half precision (one plane or two), largest weight at 2^12 .. 2^13, and what they are multiplied with has
// a power of two of its own for all its rows.  So that neither a row that weighs little nor an item that is unlikely for every
// row loses its digits to the others: terms of a row whose weight is below kLight of that scale are taken times 2^light_exp
// (in G, for dx); and those of an item whose largest one is below kItemLow among 64 rows times a power of its own (in G^T,
// for dtable: k_levels brings an item's groups of 64 rows to one power).  Both come off the gradients' rows.  Above these
// limits a term's last place, 2^-24, is 2^-18 of its item's largest term or better.
constexpr float kLight = 16.f, kItemLow = 0.015625f;
constexpr int kNoTerms = 255;   // in lev: no terms in these rows
__device__ __forceinline__ int light_exp(float w) {  // w: weight in G's scale
    const float a = fabsf(w);
    return a < kLight && a > 0.f ? min(12 + 127 - (int)(__float_as_uint(a) >> 23), 120) : 0;
}

// What a row's terms G = w (2^(logit - l2) - [target]) take.
struct TermRow {
    float w = 0.f, l2 = 0.f, f = 0.f;
    int light = 0;       // w has this power of two of its own
    int64_t y = -1;      // target, from the first table entry of the piece
    uint32_t keep = 0;   // all ones in rows that count: others are cut off as bits, whatever they hold
    __device__ __forceinline__ void load(const GemmArgs& a, int64_t t) {
        if (t >= a.t) return;
        const int64_t yt = load_target(a.target, a.target_bits, t);
        f = a.xf[t];
        if (!row_counts(yt, a.v, a.offset)) return;
        keep = ~0u;
        w = a.grad ? a.grad[t] : 1.f;
        w = ldexpf(w, a.fin[2]);
        light = light_exp(w);
        w = ldexpf(w, light);
        if (yt >= a.v) w = NAN;
        l2 = a.lse[t] * kLog2e;
        y = yt - a.v0;
    }
};

// Writes 32 x 32 terms as operand fragments, of G and (by a product with the identity) of G^T.
template <class PG, int NPL>
struct TermBlocks {
    typename PG::vec eye[2];  // the identity in B-operand order for the two steps of 16 entries
    __device__ __forceinline__ explicit TermBlocks(int lane) {
        const int n = lane & 31, h = lane >> 5;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < 8; ++k) eye[s][k] = (typename PG::elem)(16 * s + (k < 4 ? 4 * h + k : 8 + 4 * h + k - 4) == n ? 1.f : 0.f);
    }
    // z: logits in base 2, lane (n, h): row n, entries 8 q + 4 h + r.  Returns the largest term of the lane's item n among
    // its 16 rows of G^T (0 where that is not asked for).
    __device__ __forceinline__ float put(const GemmArgs& a, int64_t vt, int64_t tt, int lane, const f32x16& z, const TermRow& row) const {
        const int h = lane >> 5;
        float g[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) g[r] = row.w * exp2_fast(z[r] - row.l2);
        const int64_t at = row.y - vt * 32;
        if (__any(at >= 0 && at < 32)) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (at == 8 * (r >> 2) + 4 * h + (r & 3)) g[r] -= row.w;
        }
        return write(a, vt, tt, lane, g, row.keep, a.g);
    }

    // The terms of 64 rows (two tiles; the second one may not be there), and their items' power of two.
    __device__ __forceinline__ void put_pair(const GemmArgs& a, int64_t vt, int64_t tt, int lane, const f32x16& z0, const f32x16& z1, bool two,
                                             const TermRow& row0, const TermRow& row1) const {
        float top = put(a, vt, tt, lane, z0, row0);
        if (two) top = fmaxf(top, put(a, vt, tt + 1, lane, z1, row1));
        if (!a.gt) return;
        top = halves_max(top);
        int own = 0;
        if (__any((row0.light | row1.light) != 0) || __any(top < kItemLow && a.o2[vt * 32 + (lane & 31)] != -INFINITY))
            own = put_again(a, vt, tt, lane, z0, z1, two, row0, row1);
        if (lane < 32) {
            if (a.lev) a.lev[(vt * ((a.n_tiles + 1) / 2) + tt / 2) * 32 + lane] = (uint8_t)own;
            else a.item_e[vt * 32 + lane] = own == kNoTerms ? 0 : own;
        }
    }

    // G^T once more, each item's terms by the power of two that brings its largest one above 1; returns that of item `lane`.
    __device__ int put_again(const GemmArgs& a, int64_t vt, int64_t tt, int lane, const f32x16& z0, const f32x16& z1, bool two, const TermRow& row0,
                             const TermRow& row1) const {
        const int h = lane >> 5;
        const float w0 = row0.keep ? log2f(fabsf(row0.w)) - (float)row0.light : -INFINITY;
        const float w1 = row1.keep && two ? log2f(fabsf(row1.w)) - (float)row1.light : -INFINITY;
        const int64_t y0 = row0.y - vt * 32, y1 = row1.y - vt * 32;
        int own[16], mine = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int item = 8 * (r >> 2) + 4 * h + (r & 3);
            float c = w0 == -INFINITY ? -INFINITY : fmaxf(z0[r] - row0.l2 + w0, y0 == item ? w0 : -INFINITY);
            if (w1 != -INFINITY) c = fmaxf(c, fmaxf(z1[r] - row1.l2 + w1, y1 == item ? w1 : -INFINITY));
            // the largest among the 32 lanes of either half
            c = max_from<0x111, 0xf>(c), c = max_from<0x112, 0xf>(c), c = max_from<0x114, 0xf>(c), c = max_from<0x118, 0xf>(c);
            c = max_from<0x142, 0xa>(c);
            const int i = __builtin_bit_cast(int, c);
            const float low = __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 31)), high = __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 63));
            const auto power = [](float top) {  // multiples of 8, so that neighbouring groups of rows mostly agree
                if (top == -INFINITY) return kNoTerms;
                return top < -6.f ? (int)fminf(8.f * ceilf((4.f - top) * 0.125f), 112.f) : 0;
            };
            const int p0 = power(low), p1 = power(high);
            own[r] = h ? p1 : p0;
            const int first = 8 * (r >> 2) + (r & 3);
            if (lane == first) mine = p0;
            if (lane == first + 4) mine = p1;
        }
        const auto tile = [&](int64_t tt, const f32x16& z, const TermRow& row, int64_t y) {
            float g[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int up = (own[r] == kNoTerms ? 0 : own[r]) - row.light;
                g[r] = row.w * exp2_fast(z[r] - row.l2 + (float)up);
                if (y == 8 * (r >> 2) + 4 * h + (r & 3)) g[r] -= __builtin_amdgcn_ldexpf(row.w, up);
            }
            write(a, vt, tt, lane, g, row.keep, nullptr);
        };
        tile(tt, z0, row0, y0);
        if (two) tile(tt + 1, z1, row1, y1);
        return mine;
    }

    __device__ __forceinline__ float write(const GemmArgs& a, int64_t vt, int64_t tt, int lane, const float* g, uint32_t keep, char* to_g) const {
        typename PG::vec pl[NPL][2];
        float top = 0.f;
        split_terms<PG, NPL>(g, pl);
#pragma unroll
        for (int k = 0; k < NPL; ++k) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 bits = __builtin_bit_cast(u32x4, pl[k][s]);
                bits &= keep;
                pl[k][s] = __builtin_bit_cast(typename PG::vec, bits);
                if (to_g) *(u32x4*)(to_g + k * a.g_plane + (tt * a.ksv + vt * 2 + s) * kBlk + lane * 16) = bits;
            }
            if (!a.gt) continue;
            f32x16 tr = {};
            tr = PG::mfma(pl[k][0], eye[0], tr);
            tr = PG::mfma(pl[k][1], eye[1], tr);
            typename PG::vec to[2];
#pragma unroll
            for (int r = 0; r < 16; ++r) to[r >> 3][r & 7] = (typename PG::elem)tr[r];
            if (k == 0)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(tr[r]));
#pragma unroll
            for (int s = 0; s < 2; ++s) *(typename PG::vec*)(a.gt + k * a.gt_plane + (vt * a.kst + tt * 2 + s) * kBlk + lane * 16) = to[s];
        }
        return top;
    }
};

// P: operands; PG: terms G.
constexpr int kNf = 2;                  // blocks of 32 columns of a wave
constexpr int kWaveCols = 8 / kNf;      // waves beside each other
constexpr int kWaves = 2 * kWaveCols, kGemmThreads = 64 * kWaves;
constexpr int kEach = 8 / kWaves;       // blocks of 32 rows of each operand that a wave fetches

template <class P, class PG, int NPL, int EPI, class T>
__global__ __launch_bounds__(kGemmThreads) void k_gemm(GemmArgs a) {
    __shared__ __align__(16) char lds[kStages * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / kWaveCols, wn = wave % kWaveCols;
    const int split = blockIdx.y;
    // Blocks b, b + 8, .. share an XCD and its L2: each gets a contiguous run of tiles, eight rows of tiles at a time.
    // (Places are the same for all lanes, which the compiler does not see through the divisions.)
    const int64_t mb = (a.m_tiles + 7) / 8, nb = (a.n_tiles + 7) / 8;
    int bm, bn;
    {
        const int64_t all = mb * nb, x = blockIdx.x & 7, per = all >> 3, more = all & 7;
        const int64_t id = x * per + min(x, more) + (blockIdx.x >> 3);
        const int64_t band = id / (8 * nb), first = band * 8, height = min((int64_t)8, mb - first);
        const int64_t in = id - band * 8 * nb;
        bm = __builtin_amdgcn_readfirstlane((int)(first + in % height));
        bn = __builtin_amdgcn_readfirstlane((int)(in / height));
    }
    const int k0 = __builtin_amdgcn_readfirstlane((int)(a.kb * split / a.splits));
    const int steps = __builtin_amdgcn_readfirstlane((int)(a.kb * (split + 1) / a.splits)) - k0;
    f32x16 acc[4][kNf];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kNf; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // A stage of LDS is 32 KB.  One plane: 32 columns of K, two steps of 16.  Two planes: 16 columns, hi and lo.  A wave
    // brings kEach blocks of 32 rows of either operand.
    if (steps > 0) {
        const char *a0[kEach], *b0[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            a0[i] = a.a + min((int64_t)bm * 8 + wave * kEach + i, a.m_tiles - 1) * a.a_tile + (int64_t)k0 * 2 * kBlk;
            b0[i] = a.b + min((int64_t)bn * 8 + wave * kEach + i, a.n_tiles - 1) * a.b_tile + (int64_t)k0 * 2 * kBlk;
        }
        const int total = NPL == 2 ? 2 * steps : steps;  // stages
        constexpr int kStep = NPL == 2 ? kBlk : 2 * kBlk;
        const int64_t beside_a = NPL == 2 ? a.a_plane : kBlk, beside_b = NPL == 2 ? a.b_plane : kBlk;
        char* const to = lds + wave * kEach * 2 * kBlk;
        const uint32_t mine = lane * 16;
        int slot = 0, k_next = 0;
        // Past the last stage the last one is fetched again, so that the count of loads in flight stays the same.
        const auto next = [&]() {
            const int64_t at_k = (int64_t)k_next * kStep;
            k_next = __builtin_amdgcn_readfirstlane(min(k_next + 1, total - 1));
            char* const s = to + slot * kStage;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const char *pa = a0[i] + at_k, *pb = b0[i] + at_k;
                fetch(pa + mine, s + i * 2 * kBlk);
                fetch(pa + beside_a + mine, s + (i * 2 + 1) * kBlk);
                fetch(pb + mine, s + (16 + i * 2) * kBlk);
                fetch(pb + beside_b + mine, s + (16 + i * 2 + 1) * kBlk);
            }
            slot = (slot + 1) & (kStages - 1);
        };
        const char* const ra = lds + wm * 8 * kBlk + lane * 16;
        const char* const rb = lds + (16 + wn * kNf * 2) * kBlk + lane * 16;
        // What a stage holds for this wave, the half `s` of it (step or plane).
        const auto read = [&](int s, int at, typename P::vec* fa, typename P::vec* fb) {
#pragma unroll
            for (int i = 0; i < 4; ++i) fa[i] = *(const typename P::vec*)(ra + at * kStage + (2 * i + s) * kBlk);
#pragma unroll
            for (int j = 0; j < kNf; ++j) fb[j] = *(const typename P::vec*)(rb + at * kStage + (2 * j + s) * kBlk);
        };
        const auto multiply = [&](const typename P::vec* fa, const typename P::vec* fb) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kNf; ++j) acc[i][j] = P::mfma(fa[i], fb[j], acc[i][j]);
        };
        // The order of a run of `products`: a read from LDS after each of the first ones, then the fetches.
        const auto order = [](auto products, auto reads, auto fetches) {
            constexpr int p = decltype(products)::value, r = decltype(reads)::value, f = decltype(fetches)::value;
#pragma unroll
            for (int i = 0; i < p; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (i < r) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                else if (f && i < r + f) __builtin_amdgcn_sched_group_barrier(0x020, (f + p - r - 1) / (p - r), 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" ::: "memory");
        };
        // Everybody has read this stage into registers and brought what the next one holds.
        const auto meet = [&]() {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(8 * kEach) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        constexpr std::integral_constant<int, 4 * kNf> kRun = {};
        constexpr std::integral_constant<int, 4 + kNf> kReads = {};
        constexpr std::integral_constant<int, 4 * kEach> kFetches = {};
        constexpr std::integral_constant<int, 0> kNone = {};
        next(), next(), next(), next();
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(12 * kEach) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        int at = 0;
        typename P::vec fa[4][4], fb[4][kNf];
        if constexpr (NPL == 1) {
            read(0, at, fa[0], fb[0]);
            for (int k = total; k > 0; --k) {
                read(1, at, fa[1], fb[1]);
                multiply(fa[0], fb[0]);
                order(kRun, kReads, kNone);
                meet();
                at = (at + 1) & (kStages - 1);
                read(0, at, fa[0], fb[0]);
                next();
                multiply(fa[1], fb[1]);
                order(kRun, kReads, kFetches);
            }
        } else {
            // hi hi + hi lo + lo hi; a stage's operands come while the one before is multiplied
            constexpr std::integral_constant<int, 3 * kRun> kRun3 = {};
            constexpr std::integral_constant<int, 2 * kReads> kReads2 = {};
            read(0, at, fa[0], fb[0]), read(1, at, fa[1], fb[1]);
            for (int k = total; k > 0; k -= 2)
#pragma unroll
                for (int u = 0; u < 4; u += 2) {
                    meet();
                    at = (at + 1) & (kStages - 1);
                    read(0, at, fa[2 - u], fb[2 - u]), read(1, at, fa[3 - u], fb[3 - u]);
                    next();
                    multiply(fa[u], fb[u]), multiply(fa[u], fb[u + 1]), multiply(fa[u + 1], fb[u]);
                    order(kRun3, kReads2, kFetches);
                }
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    }
    const int n = lane & 31, h = lane >> 5;
    if constexpr (EPI == EPI_OUT) {
        // The product is the gradient turned: a lane has four neighbouring columns of a row at a time.
        // Last piece and only share: the caller's type.  Else 32 bits, added to what earlier pieces left.
        // The terms' powers of two and the other operand's are taken off one after the other.
        const int eg = a.fin ? a.fin[2] : 0;
        const float f = a.fin && a.which >= 0 ? ldexpf(a.scale, -a.fin[a.which]) : a.scale;
        const auto row_exp = [&](int64_t row) {
            if (a.own == kItemsOwn) return a.item_e[row];
            return a.own == kRowsOwn && a.grad ? light_exp(ldexpf(a.grad[row], eg)) : 0;
        };
        if (a.last && !a.wide) {
            // Rows that are not aligned to four values (stores across them take longer: 50,021 x 777 in half
            // precision 161 us against 142): 32 rows of the wave's 128 columns at a time through LDS (quads of columns swapped
            // about by the row, so that neither side meets a bank twice), and out 64 neighbours at a time.
            __syncthreads();
            float* const mine = (float*)(lds + wave * (32 * 128 * 4));
            const int64_t col0 = ((int64_t)bm * 8 + wm * 4) * 32;
#pragma unroll
            for (int j = 0; j < kNf; ++j) {
                const int64_t row0 = ((int64_t)bn * 8 + wn * kNf + j) * 32;
                const int e = eg + row_exp(min(row0 + n, a.rows - 1));
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        f32x4 v;
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = __builtin_amdgcn_ldexpf(acc[i][j][4 * q + r], -e) * f;
                        *(f32x4*)(mine + n * 128 + ((i * 8 + 2 * q + h) ^ n) * 4) = v;
                    }
                __builtin_amdgcn_wave_barrier();
                const int rows = (int)min((int64_t)32, a.rows - row0);
#pragma unroll 4
                for (int r = 0; r < rows; ++r)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int c = lane + 64 * k;
                        if (col0 + c < a.cols) ((T*)a.last)[(row0 + r) * a.ldo + col0 + c] = (T)mine[r * 128 + ((c >> 2) ^ r) * 4 + (c & 3)];
                    }
                __builtin_amdgcn_wave_barrier();
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < kNf; ++j) {
            const int64_t row = ((int64_t)bn * 8 + wn * kNf + j) * 32 + n;
            if (row >= a.rows) continue;
            const int e = row_exp(row) + (a.last ? eg : 0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t col = ((int64_t)bm * 8 + wm * 4 + i) * 32 + 8 * q + 4 * h;
                    if (col >= a.cols) continue;
                    f32x4 v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = __builtin_amdgcn_ldexpf(acc[i][j][4 * q + r], -e);
                    if (!a.last) {  // columns of partial sums are a multiple of four
                        f32x4* const o = (f32x4*)(a.out + split * a.out_split + row * a.ldo + col);
                        *o = a.add ? *o + v : v;
                        continue;
                    }
                    Run<T, 4> t;
#pragma unroll
                    for (int r = 0; r < 4; ++r) t.v[r] = (T)(v[r] * f);
                    T* const o = (T*)a.last + row * a.ldo + col;
                    if (col + 4 <= a.cols) {
                        store_run<4>(o, t);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (col + r < a.cols) o[r] = t.v[r];
                    }
                }
        }
        return;
    }
    // Logits in base 2: accumulator times the row's factor, plus offset; of 32-bit values both rows' powers of two are taken off.
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const auto logit = [](float acc, float f, int k, float o) {
        if constexpr (NPL == 2) return __builtin_amdgcn_ldexpf(acc, __float_as_int(f) + k) + o;
        else return fmaf(acc, f, o);
    };
    const auto exponents = [&](int64_t tile, i32x4* k) {  // of a block of 32 entries, like their offsets
#pragma unroll
        for (int q = 0; q < 4; ++q) k[q] = NPL == 2 ? *(const i32x4*)(a.ek + tile * 32 + 4 * h + 8 * q) : i32x4{};
    };
    const auto offsets = [&](int64_t tile, f32x4* o) {  // of a block of 32 entries, those of this lane's rows
        const float* at = a.o2 + tile * 32 + 4 * h;
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = *(const f32x4*)(at + 8 * q);
    };
    if constexpr (EPI == EPI_LSE) {
        float2(*share)[256] = (float2(*)[256])lds;
        float f[kNf], top[kNf], sum[kNf];
#pragma unroll
        for (int j = 0; j < kNf; ++j) top[j] = -INFINITY, sum[j] = 0.f, f[j] = a.xf[min(((int64_t)bn * 8 + wn * kNf + j) * 32 + n, a.t - 1)];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t tile = (int64_t)bm * 8 + wm * 4 + i;
            f32x4 o[4];
            i32x4 k[4] = {};
            if (tile < a.m_tiles) {
                offsets(tile, o);
                exponents(tile, k);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) o[q] = -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < kNf; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    acc[i][j][r] = logit(acc[i][j][r], f[j], k[r >> 2][r & 3], o[r >> 2][r & 3]);
                    top[j] = fmaxf(top[j], acc[i][j][r]);
                }
            if (tile >= a.kept_tiles) continue;
#pragma unroll
            for (int j = 0; j < kNf; ++j) {
                const int64_t tt = (int64_t)bn * 8 + wn * kNf + j;
                if (tt >= a.n_tiles) continue;
                f32x4* const to = (f32x4*)(a.kept + (tt * a.kept_tiles + tile) * 1024) + lane;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f32x4 four;
#pragma unroll
                    for (int r = 0; r < 4; ++r) four[r] = acc[i][j][4 * q + r];
                    to[q * 64] = four;
                }
            }
        }
        __syncthreads();  // LDS is free
#pragma unroll
        for (int j = 0; j < kNf; ++j) {
            top[j] = fmaxf(top[j], __shfl_xor(top[j], 32));
            const float ref = top[j] == -INFINITY ? 0.f : top[j];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[j] += exp2_fast(acc[i][j][r] - ref);
            sum[j] += __shfl_xor(sum[j], 32);
            if (h == 0) share[wm][(wn * kNf + j) * 32 + n] = make_float2(top[j], sum[j]);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += kGemmThreads) {
            const int64_t t = (int64_t)bn * 256 + i;
            const float2 p = share[0][i], q = share[1][i];
            const float m = fmaxf(p.x, q.x);
            const float mr = m == -INFINITY ? 0.f : m;
            if (t < a.t) a.part[bm * a.t + t] = make_float2(m, p.y * exp2_fast(p.x - mr) + q.y * exp2_fast(q.x - mr));
        }
        return;
    }
    if constexpr (EPI == EPI_G) {
        __syncthreads();  // LDS is free
        const TermBlocks<PG, NPL> terms(lane);
        TermRow row[kNf];
#pragma unroll
        for (int j = 0; j < kNf; ++j) row[j].load(a, ((int64_t)bn * 8 + wn * kNf + j) * 32 + n);
        const int64_t tt = (int64_t)bn * 8 + wn * kNf;  // (even)
        if (tt >= a.n_tiles) return;
        // Logits go through LDS, half of the wave's at a time, and the terms' code is there once: unrolled, what rare groups
        // take would not fit the registers.
        f32x4* const mine = (f32x4*)(lds + wave * (16 * kBlk)) + lane;
#pragma unroll
        for (int i0 = 0; i0 < 4; i0 += 2) {
#pragma unroll
            for (int i = i0; i < i0 + 2; ++i) {
                const int64_t vt = min((int64_t)bm * 8 + wm * 4 + i, a.m_tiles - 1);
                f32x4 o[4];
                i32x4 k[4];
                offsets(vt, o);
                exponents(vt, k);
#pragma unroll
                for (int j = 0; j < kNf; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        f32x4 four;
#pragma unroll
                        for (int r = 0; r < 4; ++r) four[r] = logit(acc[i][j][4 * q + r], row[j].f, k[q][r], o[q][r]);
                        mine[(((i - i0) * kNf + j) * 4 + q) * 64] = four;
                    }
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (int i = i0; i < i0 + 2; ++i) {
                const int64_t vt = (int64_t)bm * 8 + wm * 4 + i;
                if (vt >= a.m_tiles) break;
                f32x16 z[kNf];
#pragma unroll
                for (int j = 0; j < kNf; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4 four = mine[(((i - i0) * kNf + j) * 4 + q) * 64];
#pragma unroll
                        for (int r = 0; r < 4; ++r) z[j][4 * q + r] = four[r];
                    }
                terms.put_pair(a, vt, tt, lane, z[0], z[1], tt + 1 < a.n_tiles, row[0], row[1]);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// ---- logits of small products ----------------------------------------------------------------
// Where blocks of 256 x 256 logits are fewer than CUs, their contraction is cut as well: the shares' partial logits
// (64 MB at most in all) are joined here, and stay for the gradients' terms.  (200 x 2,372 in shares: 6 us.)
struct JoinArgs {
    float* z;            // [share][t][pitch]; the first one receives the logits in base 2
    int shares;
    int64_t share, pitch, t;
    const float *xf, *o2;
    const int* ek;       // (32-bit values: xf and ek are exponents) or NULL
    float2* part;        // [blocks of 1024 entries][t], or NULL
};

__global__ __launch_bounds__(256) void k_join(JoinArgs a) {
    __shared__ float red[4][2];
    const int64_t t = blockIdx.y, v = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    float top = -INFINITY, sum = 0.f;
    f32x4 z = {};
    if (v < a.pitch) {
        float* const at = a.z + t * a.pitch + v;
        int s = 0;
        for (; s + 8 <= a.shares; s += 8) {  // eight reads in flight
            f32x4 q[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) q[k] = *(const f32x4*)(at + (s + k) * a.share);
#pragma unroll
            for (int k = 0; k < 8; ++k) z += q[k];
        }
        for (; s < a.shares; ++s) z += *(const f32x4*)(at + s * a.share);
        const f32x4 o = *(const f32x4*)(a.o2 + v);
        const float f = a.xf[t];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            z[r] = a.ek ? __builtin_amdgcn_ldexpf(z[r], __float_as_int(f) + a.ek[v + r]) + o[r] : fmaf(z[r], f, o[r]);
            top = fmaxf(top, z[r]);
        }
        *(f32x4*)at = z;
    }
    if (!a.part) return;
    top = wave_max(top);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) red[wave][0] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0][0], red[1][0]), fmaxf(red[2][0], red[3][0]));
    const float ref = top == -INFINITY ? 0.f : top;
    if (v < a.pitch)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += exp2_fast(z[r] - ref);
    for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
    if (lane == 0) red[wave][1] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.part[blockIdx.x * a.t + t] = make_float2(top, red[0][1] + red[1][1] + red[2][1] + red[3][1]);
}

// The terms of 64 rows x 32 entries a wave: from rows (pitch), or from what k_gemm kept (pitch 0; v0 is the piece's first
// entry).  Bound by memory (2,000 x 32,003 in two planes: 145 us, 5.3 TB/s).
template <class PG, int NPL>
__global__ __launch_bounds__(256) void k_terms(GemmArgs a, const float* z, int64_t pitch) {
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const uint32_t across = (uint32_t)((a.m_tiles + 3) / 4);
    const int64_t vt = (int64_t)(blockIdx.x % across) * 4 + (threadIdx.x >> 6), tt = blockIdx.x / across * 2;
    if (vt >= a.m_tiles) return;
    const bool two = tt + 1 < a.n_tiles;
    const int step = pitch ? 8 : 256;
    f32x16 q[2];
    TermRow row[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t at = two ? tt + j : tt;
        const float* const from = pitch ? z + min(at * 32 + n, a.t - 1) * pitch + vt * 32 + 4 * h : a.kept + (at * a.kept_tiles + a.v0 / 32 + vt) * 1024 + lane * 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const f32x4 four = *(const f32x4*)(from + step * k);
#pragma unroll
            for (int r = 0; r < 4; ++r) q[j][4 * k + r] = four[r];
        }
    }
    row[0].load(a, tt * 32 + n);
    if (two) row[1].load(a, tt * 32 + 32 + n);
    const TermBlocks<PG, NPL> terms(lane);
    terms.put_pair(a, vt, tt, lane, q[0], q[1], two, row[0], row[1]);
}

// One power of two for each item over all groups of 64 rows, the lowest of theirs: fragments of G^T that have another one are
// brought to it (most have none of their own, and nothing is moved: 1,003 x 50,021 then take 5 us).  A block per 32 items.
template <int NPL>
__global__ __launch_bounds__(256) void k_levels(GemmArgs a) {
    __shared__ int low[8][32];
    const int item = threadIdx.x & 31, part = threadIdx.x >> 5, groups = (int)((a.n_tiles + 1) / 2);
    const uint8_t* const lev = a.lev + (int64_t)blockIdx.x * groups * 32;
    int least = kNoTerms;
    for (int g = part; g < groups; g += 8) least = min(least, (int)lev[g * 32 + item]);
    low[part][item] = least;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) least = min(least, low[k][item]);
    if (part == 0) a.item_e[(int64_t)blockIdx.x * 32 + item] = least == kNoTerms ? 0 : least;
    const int lane = threadIdx.x & 63;
    for (int g = threadIdx.x >> 6; g < groups; g += 4) {
        const int own = lev[g * 32 + item], down = own == kNoTerms ? 0 : own - least;
        if (!__any(down != 0)) continue;
        for (int tt = 2 * g; tt < min(2 * g + 2, (int)a.n_tiles); ++tt)
#pragma unroll
            for (int i = 0; i < 2 * NPL; ++i) {
                f16x8* const at = (f16x8*)(a.gt + (i >> 1) * a.gt_plane + (blockIdx.x * a.kst + tt * 2 + (i & 1)) * kBlk + lane * 16);
                f16x8 v = *at;
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = (_Float16)__builtin_amdgcn_ldexpf((float)v[k], -down);
                *at = v;
            }
    }
}

// ---- ends ------------------------------------------------------------------------------------
// The numbers of row t that the gradients of few factors need (see softmax_device.hpp).
struct RowNumbers {
    char* first;      // of the first 32 rows, or NULL
    int64_t step;     // bytes per 32 rows
    const float* grad;
    const int32_t* fin;
};

__device__ __forceinline__ void put_numbers(const RowNumbers& n, int64_t t, int64_t y, int64_t v, const float* offset, float lse) {
    if (!row_counts(y, v, offset)) return;
    float w = n.grad ? n.grad[t] : 1.f;
    if (n.fin) w = ldexpf(w, n.fin[2]);
    float* o = (float*)(n.first + t / 32 * n.step) + t % 32;
    const float l2 = lse * kLog2e;
    o[kNumLse * 32] = y < v ? -l2 : NAN;
    o[kNumRaw * 32] = n.grad ? n.grad[t] : 1.f;
    o[kNumTerm * 32] = y < v ? log2f(fabsf(w)) - l2 : NAN;
    o[kNumWeight * 32] = fabsf(w);
    o[kNumTarget * 32] = __int_as_float(y < v ? (int)y : -1);
}

__global__ __launch_bounds__(256) void k_rows(ccdpp_softmax_t p, const float* lse, RowNumbers n) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < p.t) put_numbers(n, t, load_target(p.target, p.target_bits, t), p.v, p.offset, lse[t]);
}

// Joins the (max, sum) pairs of a row's pieces (0: of its shares), and takes the target's logit from x and the table: a
// wave a row, or a block of 256 threads where rows are long or few.  (Latency: 5 us for 1,024 or 4,096 rows; 59 us for 8,192
// rows of 512 pieces and 4,096 columns.)
template <class T, int THREADS>
__global__ __launch_bounds__(256) void k_loss(ccdpp_softmax_t p, const float2* part, int64_t pieces, Shares shares, float* loss, float* lse, RowNumbers num) {
    constexpr int kRows = 256 / THREADS;
    __shared__ float red[4][4];
    const int i0 = threadIdx.x % THREADS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS; t < p.t; t += (int64_t)gridDim.x * kRows) {
        // the target's products first: their reads are under way while the pieces come
        const int64_t y = load_target(p.target, p.target_bits, t);
        const float o = p.offset && y >= 0 && y < p.v ? p.offset[y] : 0.f;
        float dot = 0.f;
        if (y >= 0 && y < p.v && !(o < kExcluded)) {
            const T *x = (const T*)p.x + t * p.ldx, *e = (const T*)p.table + y * p.ldt;
            constexpr int N = 16 / sizeof(T);
#pragma unroll 4
            for (int d = i0 * N; d + N <= p.d; d += THREADS * N) {
                const Run<T, N> a = load_run<N>(x + d), b = load_run<N>(e + d);
#pragma unroll
                for (int j = 0; j < N; ++j) dot = fmaf((float)a.v[j], (float)b.v[j], dot);
            }
            for (int d = p.d / N * N + i0; d < p.d; d += THREADS) dot = fmaf((float)x[d], (float)e[d], dot);
        }
        float m = -INFINITY, s = 0.f;
        bool nan = false;
        const int64_t n = pieces ? pieces : shares.count(t / 128);
        for (int64_t i = i0; i < n; i += THREADS) {
            const float2 q = part[i * p.t + t];
            const float top = fmaxf(m, q.x), ref = top == -INFINITY ? 0.f : top;
            nan |= q.x != q.x || q.y != q.y;
            s = s * exp2_fast(m - ref) + q.y * exp2_fast(q.x - ref);
            m = top;
        }
        float top = wave_max(m), ref = top == -INFINITY ? 0.f : top;
        s *= exp2_fast(m - ref);
        for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k), dot += __shfl_xor(dot, k);
        nan = __any(nan);
        if constexpr (THREADS == 256) {
            if (lane == 0) red[wave][0] = top, red[wave][1] = s, red[wave][2] = dot, red[wave][3] = nan ? 1.f : 0.f;
            __syncthreads();
            for (int w = 0; w < 4; ++w) top = fmaxf(top, red[w][0]);
            ref = top == -INFINITY ? 0.f : top;
            s = 0.f, dot = 0.f;
            for (int w = 0; w < 4; ++w) {
                s += red[w][1] * exp2_fast(red[w][0] - ref);
                dot += red[w][2];
                nan |= red[w][3] != 0.f;
            }
        }
        float l = top == -INFINITY ? -INFINITY : (top + log2f(s)) * kLn2;
        if (nan) l = NAN;
        float out = 0.f;
        if (y >= p.v) out = NAN;
        else if (y >= 0) out = o < kExcluded ? INFINITY : l - fmaf(dot, p.scale, o);
        if (i0 == 0) {
            loss[t] = out, lse[t] = l;
            if (num.first) put_numbers(num, t, y, p.v, p.offset, l);
        }
        if (THREADS == 256 && t + gridDim.x < p.t) __syncthreads();  // `red` is free again
    }
}

// One gradient from the partial sums of its shares, in the caller's type and strides.
struct FinishSide {
    const float* part;
    int splits;                // partial sums of every row, unless `shares` counts them
    int64_t split, rows, ldp;  // ldp: a multiple of 4
    void* out;
    int64_t ldo;
    int which;                 // exponent in fin of the other operand, or -1
    int terms;                 // G's exponent, or -1: fin[2]
    Shares shares;
};

// Four columns a thread; dx's blocks first.  Bound by reading the partial sums (4,096 + 17,770 rows of 100 floats in two or three
// shares: 10 us).
template <class T>
__global__ __launch_bounds__(256) void k_finish(FinishSide x, FinishSide e, int64_t blocks_x, int cols, float scale, const int32_t* fin) {
    const bool is_x = blockIdx.x < blocks_x;
    const FinishSide& a = is_x ? x : e;
    const int64_t first = is_x ? blockIdx.x : blockIdx.x - blocks_x, stride = is_x ? blocks_x : gridDim.x - blocks_x;
    const int quads = (cols + 3) / 4;
    // G's power of two and the other operand's are taken off one after the other: their product may be below any float
    const float fg = a.terms >= 0 ? ldexpf(1.f, -a.terms) : fin ? ldexpf(1.f, -fin[2]) : 1.f;
    const float f = fin && a.which >= 0 ? ldexpf(scale, -fin[a.which]) : scale;
    for (int64_t i = first * 256 + threadIdx.x; i < a.rows * quads; i += stride * 256) {
        const int64_t r = i / quads;
        const int c = (int)(i - r * quads) * 4;
        const float* from = a.part + r * a.ldp + c;
        f32x4 v = {};
        const int splits = a.shares.len ? a.shares.count(r / 128) : a.splits;
        if (a.shares.len && splits == 1) continue;  // is there
        int s = 0;
        for (; s + 8 <= splits; s += 8) {  // eight reads in flight
            f32x4 q[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) q[k] = *(const f32x4*)(from + (s + k) * a.split);
#pragma unroll
            for (int k = 0; k < 8; ++k) v += q[k];
        }
        for (; s < splits; ++s) v += *(const f32x4*)(from + s * a.split);
        T* o = (T*)a.out + r * a.ldo + c;
        Run<T, 4> t;
#pragma unroll
        for (int j = 0; j < 4; ++j) t.v[j] = (T)(v[j] * fg * f);
        if (c + 4 <= cols) {
            store_run<4>(o, t);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < cols) o[j] = t.v[j];
        }
    }
}

// ---- host --------------------------------------------------------------------------------------
struct Plan {
    int planes = 1;
    bool scaled = false;     // the matrices get powers of two
    bool scale_g = false;    // so does G
    bool grads = false, forward = false;
    bool few = false;        // t <= kFewT: k_few_*
    bool small = false;      // else d <= kSmallD: k_small_*
    int64_t tt, vt, dt;      // blocks of 32
    int ksd;                 // steps of 16 over d
    int64_t kst, ksv;        // over rows, over the whole table
    int64_t vc, tc;          // table entries and rows per piece of the gradients (multiples of 256)
    int64_t tz;              // rows per launch of the logits (a multiple of 256)
    int64_t dp;              // columns of partial sums
    int sx, se;              // splits of the two gradients' contractions
    int sz;                  // shares of the logits' contraction; above 1 all logits are kept, in rows
    int64_t kept = 0;        // table entries whose logits are kept for the gradients, in blocks (0, whole pieces or all)
    Shares lse, dx, de;      // (small)
    int64_t x_tile, xlive_tile, e_tile;  // bundles (small)
    // offsets into the workspace
    bool direct = false;     // t <= kDirectT: the logits by k_direct_logits
    FewShape shape = {};
    int few_parts = 0;       // blocks of the gradients along the table
    int64_t o_z;             // kept logits
    int64_t o_lev, o_item;
    int64_t o_scale, o_xrow, o_erow, o_ek, o_fin, o_xf, o_ef, o_xl, o_o2, o_xn, o_xt, o_et, o_g, o_gt, o_part, o_dx, o_de, bytes;
};

// Of G, and as much again of G^T: pieces of the table, and of the rows where they are many, keep the workspace bounded,
// whatever t and v are; larger ones read and write dx's partial sums less often (8,192 x 131,072 x 4,096: 1.5% less than by
// 128 MiB).
constexpr int64_t kPieceBytes = int64_t(512) << 20;
constexpr int64_t kLeastEntries = 2048;  // of a piece
// The logits' (max, sum) pairs of a launch: at most this, or those of 256 rows.
constexpr int64_t kPairBytes = int64_t(256) << 20;


// A training pass may keep logits between its two halves, in kKeptBytes at most, whatever t and v are.  Written and read
// they cost 8 bytes an entry, computed again a product over the factors: the first is less from some 384 columns on in 32
// bits and 1,024 in 16 (2,000 x 32,003 rows, computed again or kept: 256 floats 529 and 549 us, 512 floats 789 and 729, 1,024
// floats 1,401 and 1,207; 512 halves 390 and 424, 1,024 halves 603 and 577, 4,096 halves 2,020 and 1,679).
constexpr int64_t kKeptBytes = int64_t(1) << 30;
constexpr int keep_from(int planes) { return planes == 2 ? 384 : 1024; }

Plan make_plan(const ccdpp_softmax_t& p, int call) {
    Plan w;
    w.grads = call != CCDPP_SOFTMAX_LOSS;
    w.forward = call != CCDPP_SOFTMAX_GRAD;
    w.planes = p.dtype == CCDPP_F32 ? 2 : 1;
    w.small = p.d <= kSmallD;
    w.scaled = p.dtype == CCDPP_F32 || (p.dtype == CCDPP_BF16 && w.grads && !w.small);
    w.scale_g = w.grads && (w.scaled || p.dtype == CCDPP_F16);
    w.tt = (p.t + 31) / 32, w.vt = (p.v + 31) / 32, w.dt = (p.d + 31) / 32;
    w.kst = w.tt * 2, w.ksv = w.vt * 2;
    int64_t at = 0;
    const auto take = [&](int64_t n) {
        const int64_t o = at;
        at += round_up(std::max<int64_t>(n, 0), 256);
        return o;
    };
    const int es = w.planes == 2 ? 4 : 2;
    w.few = p.t <= kFewT;
    w.direct = w.few || (p.t <= kDirectT && !w.small);
    if (w.direct) {
        w.shape = few_shape(std::max<int64_t>(p.t, 1), p.v, p.d, es);
        w.o_part = take(w.forward ? w.shape.blocks * p.t * 8 : 0);
        w.o_z = take(w.grads ? p.t * w.vt * 32 * 4 : 0);
    }
    if (w.few) {
        const int64_t wide = (int64_t)few_across(p.d, 16 / es) * 16 * (16 / es), beside = (p.d + wide - 1) / wide;
        const int64_t at_once = 256 * (p.t > 16 ? 2 : es == 4 ? 4 : 3);  // blocks, by their registers
        w.few_parts = (int)std::max<int64_t>(1, std::min<int64_t>(at_once / beside, (p.v + 63) / 64));
        w.dp = round_up(p.d, 4);
        w.o_dx = take(w.grads ? w.few_parts * p.t * w.dp * 4 : 0);
        w.bytes = at;
        return w;
    }
    w.o_scale = take(4 * kParts * 4);
    w.o_fin = take(64);
    w.o_xrow = take(w.scaled ? p.t * 4 : 0);
    if (w.small) {
        // As many shares as blocks run at once (a share has four tiles at least).
        const auto shares = [](int64_t kept_tiles, int64_t tiles, int64_t want) {
            const int64_t total = (kept_tiles + 3) / 4 * tiles;
            Shares s = {tiles, std::max<int64_t>((total + want - 1) / want, std::min<int64_t>(tiles, 4)), 0};
            if (s.len >= 8 * tiles) s.len = round_up(s.len, tiles);  // whole blocks: no partial sums, for an eighth more at most
            s.blocks = total ? (total + s.len - 1) / s.len : 0;
            return s;
        };
        w.ksd = small_steps(p.d);
        w.dp = w.dt * 32;
        w.x_tile = (w.planes * w.ksd + 1) * kBlk;
        w.e_tile = w.xlive_tile = w.x_tile + (w.grads ? w.planes * w.dt * 2 * kBlk : 0);
        constexpr int kCus = 256;
        // dx and de run in one launch; a tile of de, whose streamed rows have numbers of their own, takes 5/4 of one of dx
        const int all = kCus * small_grads_per_cu(w.planes, w.ksd), mine = all * 4 / 9;
        w.lse = shares(w.tt, w.vt, kCus * small_lse_per_cu(w.planes, w.ksd));
        w.dx = shares(w.tt, w.vt, mine), w.de = shares(w.vt, w.tt, all - mine);
        w.o_xf = take(w.forward ? w.tt * w.x_tile : 0);
        w.o_ef = take(w.vt * w.e_tile);
        w.o_xl = take(w.grads ? w.tt * w.xlive_tile : 0);
        w.o_part = take(w.forward ? w.lse.most() * p.t * 8 : 0);
        w.o_dx = take(w.grads && !w.dx.whole() ? w.dx.most() * w.tt * 32 * w.dp * 4 : 0);
        w.o_de = take(w.grads && !w.de.whole() ? w.de.most() * w.vt * 32 * w.dp * 4 : 0);
        w.bytes = at;
        return w;
    }
    w.o_erow = take(w.planes == 2 && !w.direct ? p.v * 4 : 0);
    w.o_ek = take(w.planes == 2 ? w.vt * 32 * 4 : 0);
    w.ksd = (int)w.dt * 2;
    w.dp = round_up(p.d, 4);
    w.tc = std::min(round_up(std::max<int64_t>(p.t, 1), 256), kPieceBytes / (kLeastEntries * 2 * w.planes));
    const int64_t pt = std::min(w.tc / 32, std::max<int64_t>(w.tt, 1));  // blocks of 32 rows of a piece
    w.vc = std::max(kLeastEntries, kPieceBytes / (pt * 32 * 2 * w.planes) / 256 * 256);
    w.vc = std::min(w.vc, round_up(p.v, 256));
    w.tz = std::min(round_up(std::max<int64_t>(p.t, 1), 256), std::max<int64_t>(256, kPairBytes / ((w.vt + 7) / 8 * 8) / 256 * 256));
    const auto splits = [](int64_t m, int64_t n, int64_t kb) {
        const int64_t blocks = std::max<int64_t>(1, (m + 7) / 8 * ((n + 7) / 8));
        return (int)std::max<int64_t>(1, std::min<int64_t>({256 / blocks, kb / 8, 64}));
    };
    w.sx = splits(pt, w.dt, w.vc / 32);
    w.se = splits(w.vc / 32, w.dt, pt);
    // With half of the CUs or more without a block of logits the contraction may be cut too.  A step of 32 takes a block
    // half a microsecond (three times that with two planes), in the logits and again in the terms unless they are
    // kept; the kept ones cost a launch, and are written and read at 3 TB/s.  (27 x 2,372 x 3,274 floats, loss and gradients: 396
    // us whole, 98 in 25 shares; 1,796 x 3,893 x 687 in half precision, the loss: 32 whole, 51 in two.)
    const int64_t tiles = (w.vt + 7) / 8 * ((w.tt + 7) / 8);
    w.sz = 1;
    if (tiles <= 128 && !w.direct) {
        const double steps = w.ksd / 2 * (w.planes == 2 ? 1.5 : 0.5), kept = 8e-6 / 3 * (double)p.t * (double)p.v;
        double best = 1.5 * steps;  // (the same for every call, so that their results agree)
        for (int n = 2; n <= 256 / tiles && n <= w.ksd / 4; ++n)
            if (steps / n + 5 + n * kept < best) best = steps / n + 5 + n * kept, w.sz = n;
    }
    if (!w.direct) {
        if (w.sz == 1 && w.forward && w.grads && p.d >= keep_from(w.planes)) {
            const int64_t fit = kKeptBytes / (w.tt * 32 * 4);
            w.kept = fit >= w.vt * 32 ? w.vt * 32 : fit / w.vc * w.vc;
        }
        w.o_z = take(w.sz > 1 ? w.sz * p.t * w.vt * 32 * 4 : w.kept * w.tt * 32 * 4);
        w.o_xf = take(w.planes * w.tt * w.ksd * kBlk);
        w.o_ef = take(w.planes * w.vt * w.ksd * kBlk);
    }
    w.o_o2 = take(w.vt * 32 * 4);
    w.o_xn = take(w.tt * 32 * 4);
    if (!w.direct) w.o_part = take(w.forward ? (w.vt + 7) / 8 * std::min(w.tz, p.t) * 8 : 0);
    if (w.grads) {
        w.o_xt = take(w.planes * w.dt * w.kst * kBlk);
        w.o_et = take(w.planes * w.dt * w.ksv * kBlk);
        w.o_g = take(w.planes * pt * (w.vc / 16) * kBlk);
        w.o_gt = take(w.planes * (w.vc / 32) * pt * 2 * kBlk);
        w.o_lev = take(pt > 2 ? (pt + 1) / 2 * w.vc : 0);
        w.o_item = take(w.vc * 4);
        w.o_dx = take(p.v <= w.vc && w.sx == 1 ? 0 : w.sx * p.t * w.dp * 4);
        w.o_de = take(w.se == 1 && p.t <= w.tc ? 0 : w.se * w.vc * w.dp * 4);
    }
    w.bytes = at;
    return w;
}

#define OPS_LAUNCH(what)                                              \
    do {                                                              \
        const hipError_t e_ = hipGetLastError();                      \
        if (e_ != hipSuccess) return hip_fail(e_, what);              \
    } while (0)

template <class T>
int launch_loss(const ccdpp_softmax_t& p, const float2* part, int64_t pieces, const Shares& shares, float* loss, float* lse, const RowNumbers& num,
                hipStream_t st) {
    constexpr int64_t kMost = 1 << 22;  // blocks (a launch holds 2^32 threads at most)
    if (p.d > 256 || p.t <= 256) k_loss<T, 256><<<(unsigned)std::min(p.t, kMost), 256, 0, st>>>(p, part, pieces, shares, loss, lse, num);
    else k_loss<T, 64><<<(unsigned)std::min((p.t + 3) / 4, kMost), 256, 0, st>>>(p, part, pieces, shares, loss, lse, num);
    OPS_LAUNCH("loss");
    return CCDPP_OK;
}

template <class T>
int finish(const FinishSide& x, const FinishSide& e, int cols, float scale, const int32_t* fin, hipStream_t st) {
    const int64_t quads = (cols + 3) / 4;
    const auto blocks = [&](const FinishSide& a) { return a.out && !a.shares.whole() ? std::min<int64_t>((a.rows * quads + 255) / 256, 1 << 16) : 0; };
    const int64_t bx = blocks(x), be = blocks(e);
    if (bx + be == 0) return CCDPP_OK;
    k_finish<T><<<(unsigned)(bx + be), 256, 0, st>>>(x, e, bx, cols, scale, fin);
    OPS_LAUNCH("gradients");
    return CCDPP_OK;
}

struct Outs {
    float *loss, *lse;
    const float *lse_in, *grad;
    void* dx;
    int64_t lddx;
    void* de;
    int64_t ldde;
};

// The logits of few rows, their loss, and what gradients of very few need.
template <class T>
int run_direct(const ccdpp_softmax_t& p, const Plan& w, const Outs& o, char* ws, hipStream_t st) {
    FewArgs a = {};
    a.t = (int)p.t, a.d = p.d, a.dp = (int)w.dp, a.v = p.v, a.x = p.x, a.table = p.table, a.ldt = p.ldt, a.ldx = p.ldx;
    a.target = p.target, a.target_bits = p.target_bits, a.scale = p.scale, a.offset = p.offset;
    a.part = w.forward ? (float2*)(ws + w.o_part) : nullptr;
    a.z = w.grads ? (float*)(ws + w.o_z) : nullptr, a.z_row = w.vt * 32;
    hipError_t e = launch_few_logits<T>(a, w.shape, st);
    if (e != hipSuccess) return hip_fail(e, "logits");
    if (w.forward)
        if (int rc = launch_loss<T>(p, a.part, w.shape.blocks, Shares{}, o.loss, o.lse, RowNumbers{}, st)) return rc;
    if (!w.few || !w.grads || (!o.dx && !o.de)) return CCDPP_OK;
    a.lse = w.forward ? o.lse : o.lse_in, a.grad = o.grad;
    a.de = o.de, a.ldde = o.ldde, a.dxp = o.dx ? (float*)(ws + w.o_dx) : nullptr, a.parts = w.few_parts;
    e = launch_few_grads<T>(a, (T*)o.dx, o.lddx, st);
    return e == hipSuccess ? CCDPP_OK : hip_fail(e, "gradients");
}

template <int DT>
int run_small(const ccdpp_softmax_t& p, const Plan& w, const Outs& o, const int32_t* fin, char* ws, hipStream_t st) {
    typedef typename Types<DT>::in T;
    typedef typename Types<DT>::op P;
    constexpr int NPL = Types<DT>::planes;
    SmallArgs a = {};
    a.x = ws + w.o_xf, a.xlive = ws + w.o_xl, a.e = ws + w.o_ef;
    a.x_tile = w.x_tile, a.xlive_tile = w.xlive_tile, a.e_tile = w.e_tile;
    a.tt = w.tt, a.vt = w.vt, a.t = p.t, a.v = p.v;
    a.offsets = p.offset != nullptr;
    a.lse = w.lse, a.dx = w.dx, a.de = w.de;
    if (!o.dx) a.dx.blocks = 0;
    if (!o.de) a.de.blocks = 0;
    a.part = (float2*)(ws + w.o_part);
    a.dxp = (float*)(ws + w.o_dx), a.dep = (float*)(ws + w.o_de);
    a.dx_out = {o.dx, o.lddx}, a.de_out = {o.de, o.ldde};
    a.d = p.d, a.scaled = w.scaled, a.fin = fin, a.scale = p.scale;
    RowNumbers num = {};
    if (w.grads) num.first = ws + w.o_xl + NPL * w.ksd * kBlk, num.step = w.xlive_tile, num.grad = o.grad, num.fin = fin;
    if (w.forward) {
        const hipError_t e = launch_small_lse<P, NPL>(w.ksd, a, st);
        if (e != hipSuccess) return hip_fail(e, "logits");
        if (int rc = launch_loss<T>(p, a.part, 0, a.lse, o.loss, o.lse, num, st)) return rc;
    } else {
        k_rows<<<(unsigned)((p.t + 255) / 256), 256, 0, st>>>(p, o.lse_in, num);
        OPS_LAUNCH("rows");
    }
    if (!w.grads) return CCDPP_OK;
    const hipError_t e = launch_small_grads<P, NPL>(w.ksd, a, st);
    if (e != hipSuccess) return hip_fail(e, "gradients");
    const FinishSide x = {a.dxp, 0, w.tt * 32 * w.dp, p.t, w.dp, o.dx, o.lddx, w.scaled ? 0 : -1, kTermExp, w.dx};
    const FinishSide t = {a.dep, 0, w.vt * 32 * w.dp, p.v, w.dp, o.de, o.ldde, w.scaled ? 1 : -1, -1, w.de};
    return finish<T>(x, t, p.d, p.scale, fin, st);
}

// Rows t0 .. of a problem.
ccdpp_softmax_t rows_of(const ccdpp_softmax_t& p, int64_t t0, int64_t n, int64_t value_bytes) {
    ccdpp_softmax_t q = p;
    q.t = n;
    q.x = (const char*)p.x + t0 * p.ldx * value_bytes;
    q.target = (const char*)p.target + t0 * (p.target_bits / 8);
    return q;
}

// The operands of rows t0 .. t0 + n - 1, and what comes of them, in place of all rows'.
void take_rows(GemmArgs& q, const Plan& w, int64_t t0, int64_t n) {
    q.b += t0 / 32 * q.b_tile, q.n_tiles = (n + 31) / 32, q.t = n;
    q.xf += t0;
    q.target = (const char*)q.target + t0 * (q.target_bits / 8);
    if (q.kept) q.kept += t0 / 32 * (w.kept / 32) * 1024;
    if (q.lse) q.lse += t0;
    if (q.grad) q.grad += t0;
}

template <int DT>
int run_wide(const ccdpp_softmax_t& p, const Plan& w, const Outs& out, const int32_t* fin, char* ws, hipStream_t st) {
    typedef typename Types<DT>::in T;
    typedef typename Types<DT>::op P;
    typedef typename Types<DT>::turned PG;
    constexpr int NPL = Types<DT>::planes;
    GemmArgs z = {};
    z.a = ws + w.o_ef, z.b = ws + w.o_xf;
    z.a_plane = w.vt * w.ksd * kBlk, z.b_plane = w.tt * w.ksd * kBlk;
    z.a_tile = z.b_tile = (int64_t)w.ksd * kBlk;
    z.m_tiles = w.vt, z.n_tiles = w.tt, z.kb = w.ksd / 2, z.splits = 1;
    z.t = p.t, z.v = p.v, z.xf = (const float*)(ws + w.o_xn), z.fin = fin, z.o2 = (const float*)(ws + w.o_o2), z.ek = (const int*)(ws + w.o_ek);
    z.scale = p.scale, z.offset = p.offset, z.target = p.target, z.target_bits = p.target_bits;
    z.kept = (float*)(ws + w.o_z), z.kept_tiles = w.kept / 32;
    float2* const part = (float2*)(ws + w.o_part);
    const int64_t pitch = w.vt * 32, chunks = (pitch + 1023) / 1024;
    const auto blocks = [](int64_t m, int64_t n) { return (unsigned)((m + 7) / 8 * ((n + 7) / 8)); };
    if (w.direct) {
        // done
    } else if (w.sz > 1) {
        GemmArgs q = z;
        q.out = z.kept, q.out_split = p.t * pitch, q.ldo = q.cols = pitch, q.rows = p.t, q.splits = w.sz;
        k_gemm<P, PG, NPL, EPI_OUT, T><<<dim3(blocks(w.vt, w.tt), w.sz), kGemmThreads, 0, st>>>(q);
        OPS_LAUNCH("logits");
        const JoinArgs j = {z.kept, w.sz, q.out_split, pitch, p.t, z.xf, z.o2, NPL == 2 ? z.ek : nullptr, w.forward ? part : nullptr};
        k_join<<<dim3((unsigned)chunks, (unsigned)p.t), 256, 0, st>>>(j);
        OPS_LAUNCH("logits");
        if (w.forward)
            if (int rc = launch_loss<T>(p, part, chunks, Shares{}, out.loss, out.lse, RowNumbers{}, st)) return rc;
    } else if (w.forward) {
        for (int64_t t0 = 0; t0 < p.t; t0 += w.tz) {
            const int64_t n = std::min(w.tz, p.t - t0);
            GemmArgs q = z;
            take_rows(q, w, t0, n);
            q.part = part;
            k_gemm<P, PG, NPL, EPI_LSE, T><<<blocks(w.vt, q.n_tiles), kGemmThreads, 0, st>>>(q);
            OPS_LAUNCH("logits");
            if (int rc = launch_loss<T>(rows_of(p, t0, n, sizeof(T)), part, (w.vt + 7) / 8, Shares{}, out.loss + t0, out.lse + t0, RowNumbers{}, st)) return rc;
        }
    }
    if (!w.grads) return CCDPP_OK;
    z.lse = w.forward ? out.lse : out.lse_in, z.grad = out.grad;
    z.g = out.dx ? ws + w.o_g : nullptr, z.gt = out.de ? ws + w.o_gt : nullptr;
    z.item_e = (int*)(ws + w.o_item);
    const bool dx_whole = p.v <= w.vc && w.sx == 1, de_whole = p.t <= w.tc && w.se == 1;
    for (int64_t v0 = 0; v0 < p.v; v0 += w.vc) {
        const int64_t n = std::min(w.vc, p.v - v0), nt = (n + 31) / 32;
        GemmArgs o = {};
        o.m_tiles = w.dt, o.cols = p.d, o.scale = p.scale, o.fin = fin, o.item_e = z.item_e;
        const auto wide = [](const void* at, int64_t ld) { return ((uintptr_t)at | (uintptr_t)(ld * sizeof(T))) % (4 * sizeof(T)) == 0; };
        T* const de = out.de ? (T*)out.de + v0 * out.ldde : nullptr;
        for (int64_t t0 = 0; t0 < p.t; t0 += w.tc) {
            const int64_t tn = std::min(w.tc, p.t - t0);
            GemmArgs q = z;
            take_rows(q, w, t0, tn);
            q.v0 = v0, q.a = z.a + v0 / 32 * z.a_tile, q.o2 = z.o2 + v0, q.ek = z.ek + v0, q.m_tiles = nt;
            q.ksv = nt * 2, q.kst = q.n_tiles * 2;
            q.g_plane = q.n_tiles * q.ksv * kBlk, q.gt_plane = nt * q.kst * kBlk;
            q.lev = q.n_tiles > 2 ? (uint8_t*)(ws + w.o_lev) : nullptr;
            const unsigned tiles = (unsigned)((nt + 3) / 4 * ((q.n_tiles + 1) / 2));
            if (w.sz > 1 || w.direct) k_terms<PG, NPL><<<tiles, 256, 0, st>>>(q, z.kept + v0, pitch);
            else if (v0 < w.kept) k_terms<PG, NPL><<<tiles, 256, 0, st>>>(q, nullptr, 0);
            else k_gemm<P, PG, NPL, EPI_G, T><<<blocks(nt, q.n_tiles), kGemmThreads, 0, st>>>(q);
            OPS_LAUNCH("G");
            if (out.de && q.lev) {
                k_levels<NPL><<<(unsigned)nt, 256, 0, st>>>(q);
                OPS_LAUNCH("G");
            }
            o.grad = q.grad;
            if (out.dx) {
                T* const dx = (T*)out.dx + t0 * out.lddx;
                o.a = ws + w.o_et + v0 / 16 * kBlk, o.a_plane = w.dt * w.ksv * kBlk, o.a_tile = w.ksv * kBlk;
                o.b = q.g, o.b_plane = q.g_plane, o.b_tile = q.ksv * kBlk, o.n_tiles = q.n_tiles, o.rows = tn;
                o.kb = nt, o.splits = w.sx, o.out = (float*)(ws + w.o_dx) + t0 * w.dp, o.out_split = p.t * w.dp, o.add = v0 > 0;
                o.which = w.scaled ? 0 : -1, o.own = kRowsOwn;
                o.last = dx_whole ? dx : nullptr, o.ldo = o.last ? out.lddx : w.dp, o.wide = wide(dx, out.lddx);
                k_gemm<PG, PG, NPL, EPI_OUT, T><<<dim3(blocks(w.dt, q.n_tiles), w.sx), kGemmThreads, 0, st>>>(o);
                OPS_LAUNCH("dx");
            }
            if (out.de) {
                o.a = ws + w.o_xt + t0 / 16 * kBlk, o.a_plane = w.dt * w.kst * kBlk, o.a_tile = w.kst * kBlk;
                o.b = q.gt, o.b_plane = q.gt_plane, o.b_tile = q.kst * kBlk, o.n_tiles = nt, o.rows = n;
                o.kb = q.n_tiles, o.splits = w.se, o.out = (float*)(ws + w.o_de), o.out_split = w.vc * w.dp, o.add = t0 > 0;
                o.which = w.scaled ? 1 : -1, o.own = kItemsOwn;
                o.last = de_whole ? de : nullptr, o.ldo = o.last ? out.ldde : w.dp, o.wide = wide(de, out.ldde);
                k_gemm<PG, PG, NPL, EPI_OUT, T><<<dim3(blocks(w.dt, nt), w.se), kGemmThreads, 0, st>>>(o);
                OPS_LAUNCH("dtable");
            }
        }
        if (out.de && !de_whole) {
            const FinishSide e = {(const float*)(ws + w.o_de), w.se, w.vc * w.dp, n, w.dp, de, out.ldde, w.scaled ? 1 : -1, -1, {}};
            if (int rc = finish<T>(FinishSide{}, e, p.d, p.scale, fin, st)) return rc;
        }
    }
    if (out.dx && !dx_whole)
        return finish<T>(FinishSide{(const float*)(ws + w.o_dx), w.sx, p.t * w.dp, p.t, w.dp, out.dx, out.lddx, w.scaled ? 0 : -1, -1, {}}, FinishSide{}, p.d, p.scale, fin, st);
    return CCDPP_OK;
}

template <int DT>
int run(const ccdpp_softmax_t& p, int call, const Outs& out, char* ws, hipStream_t st) {
    typedef typename Types<DT>::in T;
    constexpr int NPL = Types<DT>::planes;
    const Plan w = make_plan(p, call);
    if (w.direct) {
        const int rc = run_direct<T>(p, w, out, ws, st);
        if (rc != CCDPP_OK || w.few || !w.grads) return rc;
    }
    Scales sc;
    sc.e_part = (float*)(ws + w.o_scale), sc.x_part = sc.e_part + kParts, sc.g_part = sc.x_part + kParts;
    sc.n_part = sc.g_part + kParts;
    sc.fin = (int32_t*)(ws + w.o_fin), sc.x_row = (float*)(ws + w.o_xrow);
    sc.e_row = NPL == 2 && !w.small && !w.direct ? (float*)(ws + w.o_erow) : nullptr;
    const int32_t* fin = w.scaled || w.scale_g ? sc.fin : nullptr;
    if (w.scaled || w.scale_g) {
        k_scales<T><<<kParts, 1024, 0, st>>>(p, out.grad, sc, w.scaled, NPL == 2 && w.small, w.grads);
        OPS_LAUNCH("scales");
    }

    PackArgs pk = {};
    pk.sc = sc, pk.scaled = w.scaled, pk.weights = w.scale_g;
    pk.d = p.d, pk.ksd = w.ksd, pk.target = p.target, pk.target_bits = p.target_bits, pk.v = p.v, pk.scale = p.scale, pk.offset = p.offset, pk.grad = out.grad;
    PackSide &x = pk.x, &e = pk.e;
    x.src = p.x, x.ld = p.ldx, x.rows = p.t, x.tiles = w.tt;
    e.src = p.table, e.ld = p.ldt, e.rows = p.v, e.tiles = w.vt;
    if (w.small) {
        const int64_t rows = NPL * w.ksd * kBlk, turned = rows + kBlk;
        if (w.forward) x.nat = ws + w.o_xf, x.num = x.nat + rows;
        x.nat_row = x.num_row = w.x_tile;
        e.nat = ws + w.o_ef, e.num = e.nat + rows, e.exps = e.num + kNumExp * 128, e.nat_row = e.num_row = w.e_tile;
        x.nat_plane = e.nat_plane = w.ksd * kBlk;
        if (w.grads) {
            x.live = ws + w.o_xl, x.live_num = x.live + rows, x.live_row = x.live_num_row = w.xlive_tile;
            x.turned = x.live + turned, e.turned = e.nat + turned;
            x.turned_row = w.xlive_tile, e.turned_row = w.e_tile;
            x.turned_d = e.turned_d = 2 * kBlk, x.turned_plane = e.turned_plane = w.dt * 2 * kBlk;
        }
    } else {
        if (!w.direct) x.nat = ws + w.o_xf, e.nat = ws + w.o_ef;
        x.nat_plane = w.tt * w.ksd * kBlk;
        e.nat_plane = w.vt * w.ksd * kBlk;
        x.num = ws + w.o_xn, e.num = ws + w.o_o2, e.exps = ws + w.o_ek, x.num_row = e.num_row = 128;
        x.nat_row = e.nat_row = w.ksd * kBlk;
        if (w.grads) {
            x.turned = ws + w.o_xt, x.turned_plane = w.dt * w.kst * kBlk, x.turned_d = w.kst * kBlk;
            e.turned = ws + w.o_et, e.turned_plane = w.dt * w.ksv * kBlk, e.turned_d = w.ksv * kBlk;
            x.turned_row = e.turned_row = 2 * kBlk;
        }
    }
    const dim3 grid((unsigned)(w.tt + w.vt), (p.d + 127) / 128);
    if (w.small) k_pack<DT, true><<<grid, 256, 0, st>>>(pk);
    else k_pack<DT, false><<<grid, 256, 0, st>>>(pk);
    OPS_LAUNCH("pack");
    return w.small ? run_small<DT>(p, w, out, fin, ws, st) : run_wide<DT>(p, w, out, fin, ws, st);
}

uintptr_t value_bytes(const ccdpp_softmax_t& p) { return p.dtype == CCDPP_F32 ? 4 : 2; }

int check(const ccdpp_softmax_t* p, bool pointers) {
    if (!p) return fail(CCDPP_EINVAL, "the problem is NULL");
    if (p->t < 0 || p->t >= int64_t(1) << 26) return fail(CCDPP_EINVAL, "t must be in [0, 2^26)");
    if (p->v < 1 || p->v >= int64_t(1) << 28) return fail(CCDPP_EINVAL, "v must be in [1, 2^28)");
    if (p->d < 1 || p->d > 65536) return fail(CCDPP_EINVAL, "d must be in [1, 65536]");
    if (p->dtype < CCDPP_F32 || p->dtype > CCDPP_F16) return fail(CCDPP_EINVAL, "dtype must be CCDPP_F32, CCDPP_BF16 or CCDPP_F16");
    if (p->ldx < p->d || p->ldt < p->d) return fail(CCDPP_EINVAL, "ldx and ldt must be at least d");
    if ((double)p->t * (double)p->v >= 549755813888.0) return fail(CCDPP_EINVAL, "t * v must be below 2^39: take fewer rows at a time");
    if (p->target_bits != 32 && p->target_bits != 64) return fail(CCDPP_EINVAL, "target_bits must be 32 or 64");
    if (!std::isfinite(p->scale)) return fail(CCDPP_EINVAL, "scale must be finite");
    if (!pointers) return CCDPP_OK;
    if (!p->table || (p->t > 0 && (!p->x || !p->target))) return fail(CCDPP_EINVAL, "x, table and target must be non-NULL");
    const uintptr_t value = value_bytes(*p);
    if ((uintptr_t)p->table % value || (uintptr_t)p->x % value || (uintptr_t)p->target % (p->target_bits / 8) || (uintptr_t)p->offset % 4)
        return fail(CCDPP_EINVAL, "x, table, target and offset must be aligned to their types");
    return CCDPP_OK;
}

int call(const ccdpp_softmax_t* p, int what, float* loss, float* lse, const float* lse_in, const float* grad, void* dx, int64_t lddx,
         void* de, int64_t ldde, void* ws, int64_t ws_bytes, void* stream) {
    if (int rc = check(p, true)) return rc;
    if (what != CCDPP_SOFTMAX_GRAD && p->t > 0 && (!loss || !lse)) return fail(CCDPP_EINVAL, "loss and lse must be non-NULL");
    if (what == CCDPP_SOFTMAX_GRAD && p->t > 0 && !lse_in) return fail(CCDPP_EINVAL, "lse must be non-NULL");
    if (what != CCDPP_SOFTMAX_LOSS && ((dx && lddx < p->d) || (de && ldde < p->d))) return fail(CCDPP_EINVAL, "lddx and lddt must be at least d");
    if ((((uintptr_t)loss | (uintptr_t)lse | (uintptr_t)lse_in | (uintptr_t)grad) % 4) || (((uintptr_t)dx | (uintptr_t)de) % value_bytes(*p)))
        return fail(CCDPP_EINVAL, "loss, lse, grad, dx and dtable must be aligned to their types");
    const Plan w = make_plan(*p, what);
    if (ws_bytes < w.bytes || (!ws && w.bytes > 0)) return fail(CCDPP_EINVAL, "the workspace is too small");
    if ((uintptr_t)ws % 256) return fail(CCDPP_EINVAL, "the workspace must be aligned to 256 bytes");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    const Outs out = {loss, lse, lse_in, grad, dx, lddx, de, ldde};
    if (p->t == 0) {  // no rows: the table's gradient is zero
        const FinishSide none = {nullptr, 0, 0, p->v, 0, what == CCDPP_SOFTMAX_LOSS ? nullptr : de, ldde, -1, -1, {}};
        return p->dtype == CCDPP_F32 ? finish<float>(FinishSide{}, none, p->d, 0.f, nullptr, st)
                                     : finish<_Float16>(FinishSide{}, none, p->d, 0.f, nullptr, st);  // all bits 0, as in bfloat16
    }
    switch (p->dtype) {
        case CCDPP_F32: return run<CCDPP_F32>(*p, what, out, (char*)ws, st);
        case CCDPP_BF16: return run<CCDPP_BF16>(*p, what, out, (char*)ws, st);
        default: return run<CCDPP_F16>(*p, what, out, (char*)ws, st);
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
