// Softmax loss of few rows (t <= 128) and gradients of very few (t <= 32): a request, a handful of tokens, a small
// evaluation (gfx950).
//
// Bound by reading the table, once for the logits and, for gradients, once more, and by writing its gradient: nothing is
// packed or turned.  The logits of so few rows are kept for the gradients.
//
// k_direct_logits: a wave takes 16 table rows (or twice that) against all rows of x.  Each lane reads 16 bytes of its table
// row at a time, 64 bytes a row and step, straight into the operand of 16 x 16 products: of 16-bit values 32 columns a
// step, of 32-bit ones 16 columns in four v_mfma_f32_16x16x4_f32, with exact products.  Any order of the columns will do
// as long as x, which comes from LDS, has the same.  Where table rows are few, waves share their columns.  (5 x 131,072 x
// 4,096 in bfloat16: 212 us, 5.1 TB/s, what a copy of that size reaches.)
//
// k_few_grads: 16 table rows and 16 rows of x at a time (v_mfma_f32_16x16x4_f32, or 16x16x16 for 16-bit types): the
// table's values are the operand of dx as they are read, x's are kept in registers for dtable, and the terms G stay in 32
// bits, or two 16-bit planes.  A row's values go to and from 16 lanes by 16 bytes.  Blocks share the table's rows evenly,
// as many blocks as run at once.  (16 x 618,991: 192 floats 188 us, 5.1 TB/s of table and gradient; 384 in bfloat16 272 us,
// 3.5 TB/s: rows whose length is no multiple of 16 bytes, and the 16-bit kernel's registers, cost the rest.)
#include <algorithm>

#include "softmax_device.hpp"

namespace ccdops {
namespace {

constexpr int kWaves = 8;

template <class T> struct Few;
template <> struct Few<float> {
    static __device__ __forceinline__ f32x4 step(u32x4 a, u32x4 b, f32x4 c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[k], y[k], c, 0, 0, 0);
        return c;
    }
};
template <> struct Few<__bf16> {
    static __device__ __forceinline__ f32x4 step(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Few<_Float16> {
    static __device__ __forceinline__ f32x4 step(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

// 16 bytes of a row from column c on; columns past d are 0.
template <class T>
__device__ __forceinline__ u32x4 piece(const T* row, int c, int d, int64_t room) {
    return __builtin_bit_cast(u32x4, load_tail<16 / sizeof(T)>(row, c, d, room));
}

constexpr int kBatch = 128;  // table rows whose terms are in LDS at a time

// TG: 16 rows of x each; R: 16 table rows each that a wave takes at a time.
template <class T, int TG, int R>
__global__ __launch_bounds__(kWaves * 64) void k_direct_logits(FewArgs a) {
    constexpr int N = 16 / sizeof(T), U = R * TG > 8 ? 2 : R * TG > 1 ? 4 : 8;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, q = lane >> 4;
    const int steps = (a.d + 4 * N - 1) / (4 * N), pitch = a.chunk * 64 + 16;
    const int part = wave & (a.share - 1), mine = wave / a.share, per = kWaves / a.share;  // `share` waves share their columns
    const char* x[TG];
#pragma unroll
    for (int g = 0; g < TG; ++g) x[g] = lds + min(g * 16 + m, a.t - 1) * pitch + q * 16;
    const float f = a.scale * kLog2e;
    float top[TG], sum[TG];
#pragma unroll
    for (int g = 0; g < TG; ++g) top[g] = -INFINITY, sum[g] = 0.f;
    const int64_t groups = (a.v + 31) / 32 * 2, blocks = (groups + per * R - 1) / (per * R);
    bool staged = false;
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        const int64_t g0 = (b * per + mine) * R;
        const T* row[R];
        int64_t room[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t v = min((g0 + r) * 16 + m, a.v - 1);
            row[r] = (const T*)a.table + v * a.ldt, room[r] = (a.v - 1 - v) * a.ldt + a.d;
        }
        f32x4 z[R][TG] = {};
        for (int c0 = 0; c0 < steps; c0 += a.chunk) {
            const int n = min(a.chunk, steps - c0);
            if (!staged || a.chunk < steps) {
                __syncthreads();
                const int all = a.t * n * 4;
                for (int i = threadIdx.x; i < all; i += kWaves * 64 * 4) {  // four reads in flight
                    u32x4 p[4];
                    int to[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int k = min(i + u * kWaves * 64, all - 1), t = k / (n * 4), c = k - t * n * 4;
                        to[u] = t * pitch + c * 16;
                        p[u] = piece((const T*)a.x + t * a.ldx, (c0 * 4 + c) * N, a.d, (a.t - 1 - t) * a.ldx + a.d);
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) *(u32x4*)(lds + to[u]) = p[u];
                }
                __syncthreads();
                staged = true;
            }
            const int first = n * part / a.share, last = n * (part + 1) / a.share;
            const int whole = min(last, a.d / (4 * N) - c0);
            int s = first;
            for (; s + U <= whole; s += U) {
                u32x4 e[U][R];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int r = 0; r < R; ++r) e[u][r] = __builtin_bit_cast(u32x4, load_run<N>(row[r] + ((c0 + s + u) * 4 + q) * N));
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int g = 0; g < TG; ++g) {
                        const u32x4 k = *(const u32x4*)(x[g] + (s + u) * 64);
#pragma unroll
                        for (int r = 0; r < R; ++r) z[r][g] = Few<T>::step(e[u][r], k, z[r][g]);
                    }
            }
            for (; s < last; ++s)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const u32x4 e = piece(row[r], ((c0 + s) * 4 + q) * N, a.d, room[r]);
#pragma unroll
                    for (int g = 0; g < TG; ++g) z[r][g] = Few<T>::step(e, *(const u32x4*)(x[g] + s * 64), z[r][g]);
                }
        }
        if (a.share > 1) {  // the sharing waves' sums, in order, behind the rows of x
            f32x4* const shared = (f32x4*)(lds + a.t * pitch);
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int g = 0; g < TG; ++g) shared[(wave * R * TG + r * TG + g) * 64 + lane] = z[r][g];
            __syncthreads();
            if (part == 0)
                for (int w = 1; w < a.share; ++w)
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int g = 0; g < TG; ++g) z[r][g] += shared[((wave + w) * R * TG + r * TG + g) * 64 + lane];
        }
        if (part != 0) continue;
        // lane (m, q): row m of x, table rows 4 q + i
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t v0 = (g0 + r) * 16 + 4 * q;
            if (g0 + r >= groups) continue;
            float o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] = v0 + i >= a.v ? -INFINITY : a.offset ? a.offset[v0 + i] : 0.f;
                if (o[i] < kExcluded) o[i] = -INFINITY;
            }
#pragma unroll
            for (int g = 0; g < TG; ++g) {
                float ref = top[g];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[r][g][i] = o[i] == -INFINITY ? -INFINITY : fmaf(z[r][g][i], f, o[i] * kLog2e);
                    ref = fmaxf(ref, z[r][g][i]);
                }
                if (a.z && g * 16 + m < a.t) *(f32x4*)(a.z + (g * 16 + m) * a.z_row + v0) = z[r][g];
                const float base = ref == -INFINITY ? 0.f : ref;
                sum[g] *= exp2_fast(top[g] - base);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[g] += exp2_fast(z[r][g][i] - base);
                top[g] = ref;
            }
        }
    }
    if (!a.part) return;
    __syncthreads();
    float2* const share = (float2*)lds;
#pragma unroll
    for (int g = 0; g < TG; ++g) {
#pragma unroll
        for (int k = 16; k < 64; k <<= 1) {
            const float top2 = __shfl_xor(top[g], k), sum2 = __shfl_xor(sum[g], k);
            const float ref = fmaxf(top[g], top2), r = ref == -INFINITY ? 0.f : ref;
            sum[g] = sum[g] * exp2_fast(top[g] - r) + sum2 * exp2_fast(top2 - r);
            top[g] = ref;
        }
        if (q == 0) share[wave * TG * 16 + g * 16 + m] = make_float2(top[g], sum[g]);
    }
    __syncthreads();
    for (int t = threadIdx.x; t < a.t; t += kWaves * 64) {
        float2 p = share[t];
        for (int w = 1; w < kWaves; ++w) {
            const float2 o = share[w * TG * 16 + t];
            const float ref = fmaxf(p.x, o.x), r = ref == -INFINITY ? 0.f : ref;
            p = make_float2(ref, p.y * exp2_fast(p.x - r) + o.y * exp2_fast(o.x - r));
        }
        a.part[blockIdx.x * (int64_t)a.t + t] = p;
    }
}

// What the terms of the rows take, in LDS.
struct FewRows {
    float w[kFewT], l2[kFewT];  // weight (times scale), lse in base 2
    int y[kFewT];               // target; -1: past the table; kOut: the row does not count
    int e[kFewT];               // OWN: the weight is taken times this power of two, which brings it to 2^12 .. 2^13
};

constexpr int kOut = -2;

// Power of two that brings a term to 2^12 .. 2^13.
__device__ __forceinline__ int term_exp(float top) {
    const float a = fabsf(top);
    return a > 0.f && finite(a) ? min(126, 12 + 127 - (int)(__float_as_uint(a) >> 23)) : 0;
}

// By the whole block; returns the largest finite |weight|.
template <bool OWN>
__device__ __forceinline__ float few_rows(const FewArgs& a, FewRows& rows) {
    const int t = threadIdx.x & (kFewT - 1);
    float w = 0.f, l2 = 0.f;
    int y = kOut;
    if (t < a.t) {
        const int64_t yt = load_target(a.target, a.target_bits, t);
        if (row_counts(yt, a.v, a.offset)) {
            w = yt < a.v ? (a.grad ? a.grad[t] : 1.f) * a.scale : NAN;
            l2 = a.lse[t] * kLog2e;
            y = yt < a.v ? (int)yt : -1;
        }
    }
    if (threadIdx.x < kFewT) {
        const int e = OWN ? term_exp(w) : 0;
        rows.w[t] = OWN ? ldexpf(w, e) : w, rows.l2[t] = l2, rows.y[t] = y, rows.e[t] = e;
    }
    return wave_max(finite(w) ? fabsf(w) : 0.f);
}

// The terms of table rows b .. b + n - 1 (128 at most) by 256 threads: a thread has one table row and every other row of x,
// its logits' reads all in flight.  G: 16 rows of x each.  put(table row, row of x, its number among this thread's, term); keep(table row, whether the item counts).
template <int G, class F, class K>
__device__ __forceinline__ void few_terms(const FewArgs& a, const FewRows& rows, int64_t b, int n, float up, float up2, F&& put, K&& keep) {
    const int r = threadIdx.x & (kBatch - 1), t0 = threadIdx.x / kBatch;
    const int64_t v = b + min(r, n - 1);
    float z[8 * G];
#pragma unroll
    for (int k = 0; k < 8 * G; ++k) z[k] = a.z[min(t0 + 2 * k, a.t - 1) * a.z_row + v];
    if (t0 == 0) keep(r, r < n && !(a.offset && a.offset[v] < kExcluded));
#pragma unroll
    for (int k = 0; k < 8 * G; ++k) {
        const int t = t0 + 2 * k;
        const float w = rows.w[t] * up * up2;
        float g = w * (exp2_fast(z[k] - rows.l2[t]) - (rows.y[t] == v ? 1.f : 0.f));
        if (r >= n || rows.y[t] == kOut) g = 0.f;
        put(r, t, k, g);
    }
}

// Waves that took different rows are added in order; a block leaves one partial sum of dx.
template <int C>
__device__ __forceinline__ void add_waves(const FewArgs& a, const float (*red)[16 * 16 * C], int first) {  // rows of x from `first` on
    const int across = a.across, down = 4 / across;
    __syncthreads();
    for (int i = threadIdx.x; i < min(16, a.t - first) * across * 16 * C; i += 256) {
        const int t = i / (across * 16 * C), k = i - t * across * 16 * C, w = k / (16 * C), col = blockIdx.x * across * 16 * C + k;
        if (col >= a.dp) continue;
        float s = 0.f;
        for (int y = 0; y < down; ++y) s += red[y * across + w][t * 16 * C + (k - w * 16 * C)];
        a.dxp[((int64_t)blockIdx.y * a.t + first + t) * a.dp + col] = s;
    }
}

// G: 16 rows of x each.
template <class T, int G>
__global__ __launch_bounds__(256, G == 1 ? 3 : 2) void k_few_grads(FewArgs a) {
    constexpr int C = 16 / sizeof(T);  // columns of a lane: 16 C of them are beside each other
    typedef Run<T, C> Piece;
    __shared__ FewRows info;
    __shared__ float terms[kBatch][16 * G + 1];
    __shared__ float keep[kBatch];
    __shared__ __align__(16) float red[4][16 * 16 * C];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, q = lane >> 4;
    const int across = a.across, wx = wave & (across - 1), wy = wave / across, down = 4 / across;
    const int c = (blockIdx.x * across + wx) * 16 * C + n * C;
    const bool idle = c - n * C >= a.d;  // the wave's columns are past the row
    const int64_t r0 = a.v * blockIdx.y / gridDim.y, r1 = a.v * (blockIdx.y + 1) / gridDim.y;
    // x as the operand of dtable: rows 4 j + q, zero where they do not count
    float x[4 * G][C];
#pragma unroll
    for (int j = 0; j < 4 * G; ++j) {
        const int t = 4 * j + q;
        Piece row = {};
        if (a.de && t < a.t && row_counts(load_target(a.target, a.target_bits, t), a.v, a.offset))
            row = load_tail<C>((const T*)a.x + t * a.ldx, c, a.d, (a.t - 1 - t) * a.ldx + a.d);
#pragma unroll
        for (int i = 0; i < C; ++i) x[j][i] = (float)row.v[i];
    }
    few_rows<false>(a, info);
    f32x4 dx[G][C] = {};
    const auto read = [&](int64_t row, Piece& e) { e = load_tail<C>((const T*)a.table + row * a.ldt, c, a.d, (a.v - 1 - row) * a.ldt + a.d); };
    for (int64_t b = r0; b < r1; b += kBatch) {
        const int rows = (int)min((int64_t)kBatch, r1 - b);
        __syncthreads();
        few_terms<G>(a, info, b, rows, 1.f, 1.f, [&](int r, int t, int, float g) { terms[r][t] = g; },
                  [&](int r, bool counts) { keep[r] = counts ? 1.f : 0.f; });
        __syncthreads();
        const int tiles = idle ? 0 : (rows + 15) / 16;
        Piece next[4];
        if (wy < tiles)
#pragma unroll
            for (int j = 0; j < 4; ++j) read(b + min(wy * 16 + 4 * j + q, rows - 1), next[j]);
        for (int i = wy; i < tiles; i += down) {
            Piece e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = next[j];
            if (i + down < tiles)
#pragma unroll
                for (int j = 0; j < 4; ++j) read(b + min((i + down) * 16 + 4 * j + q, rows - 1), next[j]);
            f32x4 de[C] = {};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = i * 16 + 4 * j + q;
                const bool k = keep[row] != 0.f;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const float gx = terms[row][16 * g + n], ge = terms[i * 16 + n][16 * g + 4 * j + q];
#pragma unroll
                    for (int l = 0; l < C; ++l) {
                        dx[g][l] = __builtin_amdgcn_mfma_f32_16x16x4f32(gx, k ? (float)e[j].v[l] : 0.f, dx[g][l], 0, 0, 0);
                        de[l] = __builtin_amdgcn_mfma_f32_16x16x4f32(ge, x[4 * g + j][l], de[l], 0, 0, 0);
                    }
                }
            }
            if (!a.de) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = i * 16 + 4 * q + r;
                if (row >= rows) continue;
                Piece o;
#pragma unroll
                for (int l = 0; l < C; ++l) o.v[l] = (T)de[l][r];
                store_tail<C>((T*)a.de + (b + row) * a.ldde, c, a.d, o);
            }
        }
    }
    if (!a.dxp) return;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        if (g) __syncthreads();
#pragma unroll
        for (int l = 0; l < C; ++l)
#pragma unroll
            for (int r = 0; r < 4; ++r) red[wave][(4 * q + r) * 16 * C + n * C + l] = dx[g][l][r];
        add_waves<C>(a, red, 16 * g);
    }
}

// 16-bit types: the same with v_mfma_f32_16x16x16 on the values as they are; the terms are the sum of two 16-bit planes.  In
// bfloat16 all have a power of two of the largest weight; half precision, whose range ends at 2^-24, has one for each row
// of x (for dx) and, for dtable, one for each table row, so that light rows and unlikely items keep their digits.
template <class T> struct Half;
template <> struct Half<_Float16> {
    typedef _Float16 vec __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x4 mfma(vec a, vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0); }
};
template <> struct Half<__bf16> {
    typedef __bf16 vec __attribute__((ext_vector_type(4)));
    typedef short bits __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x4 mfma(vec a, vec b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(bits, a), __builtin_bit_cast(bits, b), c, 0, 0, 0);
    }
};

template <class T, int G>
__global__ __launch_bounds__(256, G == 1 ? 3 : 2) void k_few_grads16(FewArgs a) {
    constexpr int C = 8;
    typedef Run<T, C> Piece;
    typedef typename Half<T>::vec V;
    __shared__ __align__(16) T by_row[2][kBatch][16 * G + 4];  // [plane][table row][row of x], pitch against bank conflicts
    __shared__ __align__(16) T by_x[2][16 * G][kBatch + 8];    // [plane][row of x][table row]
    __shared__ FewRows info;
    __shared__ uint16_t keep[kBatch];
    __shared__ __align__(16) float red[4][16 * 16 * C];
    constexpr bool OWN = std::is_same<T, _Float16>::value;
    // in `red`, which is not used before the end: a third block on a CU has no room for more
    float(*const tops)[kBatch] = (float(*)[kBatch])red[0];
    int* const item_e = (int*)red[1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, q = lane >> 4;
    const int across = a.across, wx = wave & (across - 1), wy = wave / across, down = 4 / across;
    const int c = (blockIdx.x * across + wx) * 16 * C + n * C;
    const bool idle = c - n * C >= a.d;  // the wave's columns are past the row
    const int64_t r0 = a.v * blockIdx.y / gridDim.y, r1 = a.v * (blockIdx.y + 1) / gridDim.y;
    const float most = few_rows<OWN>(a, info);
    const int e2 = OWN ? 0 : scale_exp(most) - 2;
    const float up = ldexpf(1.f, e2 / 2), up2 = ldexpf(1.f, e2 - e2 / 2), back = ldexpf(1.f, -(e2 / 2)), back2 = ldexpf(1.f, -(e2 - e2 / 2));
    V x[G][C];  // the operand of dtable: rows 4 q + i of each 16, zero where they do not count
#pragma unroll
    for (int k = 0; k < 4 * G; ++k) {
        const int g = k / 4, i = k % 4, t = 16 * g + 4 * q + i;
        Piece row = {};
        if (a.de && t < a.t && row_counts(load_target(a.target, a.target_bits, t), a.v, a.offset))
            row = load_tail<C>((const T*)a.x + t * a.ldx, c, a.d, (a.t - 1 - t) * a.ldx + a.d);
#pragma unroll
        for (int l = 0; l < C; ++l) x[g][l][i] = row.v[l];
    }
    f32x4 dx[G][C] = {};
    const auto read = [&](int64_t row, Piece& e) { e = load_tail<C>((const T*)a.table + row * a.ldt, c, a.d, (a.v - 1 - row) * a.ldt + a.d); };
    for (int64_t b = r0; b < r1; b += kBatch) {
        const int rows = (int)min((int64_t)kBatch, r1 - b);
        const int tiles = idle ? 0 : (rows + 15) / 16;
        Piece next[4];
        if (wy < tiles)
#pragma unroll
            for (int j = 0; j < 4; ++j) read(b + min(wy * 16 + 4 * q + j, rows - 1), next[j]);
        __syncthreads();
        float own[8 * G], top = 0.f;  // OWN: the terms as they are
        few_terms<G>(a, info, b, rows, up, up2,
                  [&](int r, int t, int k, float g) {
                      const T hi = (T)g, lo = finite((float)hi) ? (T)(g - (float)hi) : (T)0.f;
                      by_x[0][t][r] = hi, by_x[1][t][r] = lo;
                      if constexpr (OWN) own[k] = __builtin_amdgcn_ldexpf(g, -info.e[t]), top = fmaxf(top, fabsf(own[k]));
                      else by_row[0][r][t] = hi, by_row[1][r][t] = lo;
                  },
                  [&](int r, bool counts) { keep[r] = counts ? 0xffff : 0; });
        if constexpr (OWN) {
            const int r = threadIdx.x & (kBatch - 1), t0 = threadIdx.x / kBatch;
            tops[t0][r] = top;
            __syncthreads();
            const int e = term_exp(fmaxf(tops[0][r], tops[1][r]));
            if (t0 == 0) item_e[r] = e;
#pragma unroll
            for (int k = 0; k < 8 * G; ++k) {
                const float g = __builtin_amdgcn_ldexpf(own[k], e);
                const T hi = (T)g, lo = finite((float)hi) ? (T)(g - (float)hi) : (T)0.f;
                by_row[0][r][t0 + 2 * k] = hi, by_row[1][r][t0 + 2 * k] = lo;
            }
        }
        __syncthreads();
        for (int i = wy; i < tiles; i += down) {
            Piece e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = next[j];
            if (i + down < tiles)
#pragma unroll
                for (int j = 0; j < 4; ++j) read(b + min((i + down) * 16 + 4 * q + j, rows - 1), next[j]);
            uint16_t k[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = keep[i * 16 + 4 * q + j];
            V gx[G][2], ge[G][2];
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    gx[g][p] = *(const V*)&by_x[p][16 * g + n][i * 16 + 4 * q];
                    ge[g][p] = *(const V*)&by_row[p][i * 16 + n][16 * g + 4 * q];
                }
            f32x4 de[C] = {};
#pragma unroll
            for (int l = 0; l < C; ++l) {
                V v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(T, (uint16_t)(__builtin_bit_cast(uint16_t, e[j].v[l]) & k[j]));
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        dx[g][l] = Half<T>::mfma(gx[g][p], v, dx[g][l]);
                        de[l] = Half<T>::mfma(ge[g][p], x[g][l], de[l]);
                    }
            }
            if (!a.de) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = i * 16 + 4 * q + r;
                if (row >= rows) continue;
                Piece o;
#pragma unroll
                for (int l = 0; l < C; ++l) o.v[l] = (T)(OWN ? __builtin_amdgcn_ldexpf(de[l][r], -item_e[row]) : de[l][r] * back * back2);
                store_tail<C>((T*)a.de + (b + row) * a.ldde, c, a.d, o);
            }
        }
    }
    if (!a.dxp) return;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        if (g || OWN) __syncthreads();
#pragma unroll
        for (int l = 0; l < C; ++l)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                red[wave][(4 * q + r) * 16 * C + n * C + l] = OWN ? __builtin_amdgcn_ldexpf(dx[g][l][r], -info.e[16 * g + 4 * q + r]) : dx[g][l][r] * back * back2;
        add_waves<C>(a, red, 16 * g);
    }
}

// dx from the blocks' partial sums: 16 quads of columns x 16 shares of the partial sums a block, joined in order.  (A few us:
// there are at most 1,024 partial sums of each value.)
template <class T>
__global__ __launch_bounds__(256) void k_few_finish(FewArgs a, int parts, T* dx, int64_t lddx) {
    __shared__ f32x4 red[16][16];
    const int quads = a.dp / 4, per_row = (quads + 15) / 16;
    const int t = blockIdx.x / per_row, quad = (blockIdx.x - t * per_row) * 16 + (threadIdx.x & 15), k0 = threadIdx.x >> 4;
    f32x4 s = {};
    if (quad < quads)
#pragma unroll 4
        for (int k = k0; k < parts; k += 16) s += *(const f32x4*)(a.dxp + ((int64_t)k * a.t + t) * a.dp + quad * 4);
    red[k0][threadIdx.x & 15] = s;
    __syncthreads();
    if (k0 != 0 || quad >= quads) return;
    for (int k = 1; k < 16; ++k) s += red[k][threadIdx.x];
    for (int j = 0; j < 4; ++j)
        if (quad * 4 + j < a.d) dx[t * lddx + quad * 4 + j] = (T)s[j];
}

template <class T, int TG, int R>
hipError_t logits(const FewArgs& a, int blocks, size_t lds, hipStream_t st) {
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)k_direct_logits<T, TG, R>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return e;
    }
    k_direct_logits<T, TG, R><<<blocks, kWaves * 64, lds, st>>>(a);
    return hipGetLastError();
}

}  // namespace

// Groups of 16 rows of x that the kernels are built for.
static int few_groups(int64_t t) {
    const int n = (int)((t + 15) / 16);
    return n == 7 ? 8 : n;
}

FewShape few_shape(int64_t t, int64_t v, int d, int bytes) {
    FewShape s;
    const int64_t groups = (v + 31) / 32 * 2, steps = ((int64_t)d * bytes + 63) / 64;
    // Waves for all CUs, eight each: where groups of 16 table rows are fewer, up to eight waves share one, four steps each,
    // as long as a block still has as many table rows as rows of x, which it brings to LDS.
    s.share = 1;
    while (s.share < kWaves && groups * s.share < 2048 && steps >= 8 * s.share && kWaves / (2 * s.share) * 16 >= t) s.share *= 2;
    s.rows = t > 16 && s.share == 1 && groups >= 8192 ? 2 : 1;
    // x in LDS, all of it or by columns, so that two blocks fit a CU
    const int64_t room = 78 * 1024 - (s.share > 1 ? kWaves * ((t + 15) / 16) * 1024 : 0);
    s.chunk = (int)std::max<int64_t>(1, std::min<int64_t>(steps, (room / t - 16) / 64));
    const int64_t per = (int64_t)(kWaves / s.share) * s.rows;
    s.blocks = (int)std::min<int64_t>(512, (groups + per - 1) / per);
    const int tg = few_groups(t);
    s.lds = std::max<int64_t>(t * (s.chunk * 64 + 16) + (s.share > 1 ? kWaves * s.rows * tg * 1024 : 0), kWaves * tg * 16 * 8);
    return s;
}

template <class T>
hipError_t launch_few_logits(const FewArgs& a, const FewShape& s, hipStream_t st) {
    FewArgs b = a;
    b.share = s.share, b.chunk = s.chunk;
    const bool two = s.rows == 2;
    switch (few_groups(a.t)) {
        case 1: return logits<T, 1, 1>(b, s.blocks, s.lds, st);
        case 2: return two ? logits<T, 2, 2>(b, s.blocks, s.lds, st) : logits<T, 2, 1>(b, s.blocks, s.lds, st);
        case 3: return two ? logits<T, 3, 2>(b, s.blocks, s.lds, st) : logits<T, 3, 1>(b, s.blocks, s.lds, st);
        case 4: return two ? logits<T, 4, 2>(b, s.blocks, s.lds, st) : logits<T, 4, 1>(b, s.blocks, s.lds, st);
        case 5: return two ? logits<T, 5, 2>(b, s.blocks, s.lds, st) : logits<T, 5, 1>(b, s.blocks, s.lds, st);
        case 6: return two ? logits<T, 6, 2>(b, s.blocks, s.lds, st) : logits<T, 6, 1>(b, s.blocks, s.lds, st);
        default: return two ? logits<T, 8, 2>(b, s.blocks, s.lds, st) : logits<T, 8, 1>(b, s.blocks, s.lds, st);
    }
}

template <class T>
hipError_t launch_few_grads(const FewArgs& a, T* dx, int64_t lddx, hipStream_t st) {
    constexpr int C = 16 / sizeof(T);
    FewArgs b = a;
    b.across = few_across(a.d, C);
    const dim3 grid((a.d + b.across * 16 * C - 1) / (b.across * 16 * C), a.parts);
    if constexpr (sizeof(T) == 4) {
        if (a.t <= 16) k_few_grads<T, 1><<<grid, 256, 0, st>>>(b);
        else k_few_grads<T, 2><<<grid, 256, 0, st>>>(b);
    } else {
        if (a.t <= 16) k_few_grads16<T, 1><<<grid, 256, 0, st>>>(b);
        else k_few_grads16<T, 2><<<grid, 256, 0, st>>>(b);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !dx) return e;
    k_few_finish<T><<<a.t * ((a.dp / 4 + 15) / 16), 256, 0, st>>>(a, a.parts, dx, lddx);
    return hipGetLastError();
}

int few_across(int d, int columns) {
    int n = 1;
    while (n < 4 && n * 16 * columns < d) n *= 2;
    return n;
}

template hipError_t launch_few_logits<float>(const FewArgs&, const FewShape&, hipStream_t);
template hipError_t launch_few_logits<__bf16>(const FewArgs&, const FewShape&, hipStream_t);
template hipError_t launch_few_logits<_Float16>(const FewArgs&, const FewShape&, hipStream_t);
template hipError_t launch_few_grads<float>(const FewArgs&, float*, int64_t, hipStream_t);
template hipError_t launch_few_grads<__bf16>(const FewArgs&, __bf16*, int64_t, hipStream_t);
template hipError_t launch_few_grads<_Float16>(const FewArgs&, _Float16*, int64_t, hipStream_t);

}  // namespace ccdops
