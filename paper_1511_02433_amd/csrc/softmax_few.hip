// Softmax loss and gradients of few rows (t <= 16): a request, a handful of tokens (gfx950).
//
// Bound by reading the table, once for the logits and, for gradients, once more, and by writing its gradient: nothing is
// packed or turned.  The logits of so few rows are smaller than the table, so gradients keep them in the workspace.
//
// k_few_logits: a wave takes 16 table rows against 16 rows of x (those that exist, from LDS).  Each lane reads 16 bytes of
// its table row at a time, 64 bytes a row and step, straight into the operand of a 16 x 16 product: of 16-bit values
// 32 columns a step, of 32-bit ones 16 columns in four v_mfma_f32_16x16x4_f32, with exact products.  Any order of the
// columns will do as long as x has the same.
//
// k_few_grads: a thread owns a few columns; it reads them row by row of the table, adds to its columns of dx and writes
// those of dtable, 2 t operations for each value read and written.
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
__device__ __forceinline__ u32x4 piece(const T* row, int c, int d) {
    constexpr int N = 16 / sizeof(T);
    if (c + N <= d) return __builtin_bit_cast(u32x4, *(const Run<T, N>*)(row + c));
    struct alignas(16) { T v[N]; } q;
#pragma unroll
    for (int j = 0; j < N; ++j) q.v[j] = c + j < d ? row[c + j] : (T)0.f;
    return __builtin_bit_cast(u32x4, q);
}

template <class T>
__global__ __launch_bounds__(kWaves * 64) void k_few_logits(FewArgs a) {
    constexpr int N = 16 / sizeof(T);
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, q = lane >> 4;
    const int steps = (a.d + 4 * N - 1) / (4 * N), whole = a.d / (4 * N), pitch = steps * 64 + 16;
    for (int i = threadIdx.x; i < a.t * steps * 4; i += kWaves * 64) {
        const int t = i / (steps * 4), c = i - t * steps * 4;
        *(u32x4*)(lds + t * pitch + c * 16) = piece((const T*)a.x + t * a.ldx, c * N, a.d);
    }
    __syncthreads();
    const char* const mine = lds + min(m, a.t - 1) * pitch + q * 16;
    const float f = a.scale * kLog2e;
    float top = -INFINITY, sum = 0.f;
    const int64_t groups = (a.v + 15) / 16;
    for (int64_t g = (int64_t)blockIdx.x * kWaves + wave; g < groups; g += (int64_t)gridDim.x * kWaves) {
        const T* const row = (const T*)a.table + min(g * 16 + m, a.v - 1) * a.ldt;
        f32x4 z = {};
        int s = 0;
        for (; s + 8 <= whole; s += 8) {  // eight reads in flight
            u32x4 e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) e[k] = __builtin_bit_cast(u32x4, *(const Run<T, N>*)(row + ((s + k) * 4 + q) * N));
#pragma unroll
            for (int k = 0; k < 8; ++k) z = Few<T>::step(e[k], *(const u32x4*)(mine + (s + k) * 64), z);
        }
        for (; s < steps; ++s) z = Few<T>::step(piece(row, (s * 4 + q) * N, a.d), *(const u32x4*)(mine + s * 64), z);
        // lane (m, q): row m of x, table rows 4 q + i
        const int64_t v0 = g * 16 + 4 * q;
        float ref = top;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float o = v0 + i >= a.v ? -INFINITY : a.offset ? a.offset[v0 + i] : 0.f;
            z[i] = o < kExcluded ? -INFINITY : fmaf(z[i], f, o * kLog2e);
            ref = fmaxf(ref, z[i]);
        }
        if (a.z && m < a.t) *(f32x4*)(a.z + m * a.z_row + v0) = z;
        const float r = ref == -INFINITY ? 0.f : ref;
        sum *= exp2_fast(top - r);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += exp2_fast(z[i] - r);
        top = ref;
    }
    if (!a.part) return;
#pragma unroll
    for (int k = 16; k < 64; k <<= 1) {
        const float top2 = __shfl_xor(top, k), sum2 = __shfl_xor(sum, k);
        const float ref = fmaxf(top, top2), r = ref == -INFINITY ? 0.f : ref;
        sum = sum * exp2_fast(top - r) + sum2 * exp2_fast(top2 - r);
        top = ref;
    }
    __syncthreads();
    float2* const share = (float2*)lds;
    if (q == 0) share[wave * 16 + m] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x < a.t) {
        for (int w = 0; w < kWaves; ++w) {
            const float2 p = share[w * 16 + threadIdx.x];
            if (w == 0) {
                top = p.x, sum = p.y;
                continue;
            }
            const float ref = fmaxf(top, p.x), r = ref == -INFINITY ? 0.f : ref;
            sum = sum * exp2_fast(top - r) + p.y * exp2_fast(p.x - r);
            top = ref;
        }
        a.part[blockIdx.x * a.part_row + threadIdx.x] = make_float2(top, sum);
    }
}

// TT: rows that registers are kept for; C: columns of a thread.
constexpr int kBatch = 128;  // table rows whose terms are in LDS at a time

template <class T, int TT, int C>
__global__ __launch_bounds__(256) void k_few_grads(FewArgs a) {
    __shared__ float terms[kBatch][TT];
    __shared__ float keep[kBatch];
    __shared__ __align__(16) float red[256 * C];
    const int across = a.across, tx = threadIdx.x & (across - 1), ty = threadIdx.x / across, down = 256 / across;
    const int c = (blockIdx.x * across + tx) * C;
    const int64_t r0 = a.v * blockIdx.y / gridDim.y, r1 = a.v * (blockIdx.y + 1) / gridDim.y;
    float x[TT][C], dx[TT][C];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const bool counts = t < a.t && row_counts(load_target(a.target, a.target_bits, t), a.v, a.offset);
#pragma unroll
        for (int j = 0; j < C; ++j) {
            dx[t][j] = 0.f;
            x[t][j] = counts && a.de && c + j < a.d ? (float)((const T*)a.x)[t * a.ldx + c + j] : 0.f;
        }
    }
    typedef Run<T, C> Piece;
    const bool whole = c + C <= a.d;
    for (int64_t b = r0; b < r1; b += kBatch) {
        const int n = (int)min((int64_t)kBatch, r1 - b);
        __syncthreads();
        for (int i = threadIdx.x; i < TT * kBatch; i += 256) {
            const int t = i / kBatch, r = i % kBatch;
            float g = 0.f;
            if (t < a.t && r < n) {
                const int64_t y = load_target(a.target, a.target_bits, t);
                if (row_counts(y, a.v, a.offset)) {
                    const float w = y < a.v ? (a.grad ? a.grad[t] : 1.f) * a.scale : NAN;
                    const float p = exp2_fast(a.z[t * a.z_row + b + r] - a.lse[t] * kLog2e);
                    g = w * (p - (y == b + r ? 1.f : 0.f));
                }
            }
            terms[r][t] = g;
            if (t == 0) keep[r] = r < n && a.offset && a.offset[b + r] < kExcluded ? 0.f : 1.f;
        }
        __syncthreads();
        constexpr int U = 4;  // rows in flight
        for (int r = ty; r < n; r += down * U) {
            Piece e[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t v = b + min(r + u * down, n - 1);
                const T* const row = (const T*)a.table + v * a.ldt + c;
                if (whole) {
                    e[u] = *(const Piece*)row;
                } else {
#pragma unroll
                    for (int j = 0; j < C; ++j) e[u].v[j] = c + j < a.d ? row[j] : (T)0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = r + u * down;
                if (at >= n) break;
                const bool k = keep[at] != 0.f;
                float de[C];
#pragma unroll
                for (int j = 0; j < C; ++j) de[j] = 0.f;
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    const float g = terms[at][t];
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        dx[t][j] = fmaf(g, k ? (float)e[u].v[j] : 0.f, dx[t][j]);
                        de[j] = fmaf(g, x[t][j], de[j]);
                    }
                }
                if (!a.de) continue;
                T* const to = (T*)a.de + (b + at) * a.ldde + c;
                Piece o;
#pragma unroll
                for (int j = 0; j < C; ++j) o.v[j] = (T)de[j];
                if (whole) {
                    *(Piece*)to = o;
                } else {
#pragma unroll
                    for (int j = 0; j < C; ++j)
                        if (c + j < a.d) to[j] = o.v[j];
                }
            }
        }
    }
    if (!a.dxp) return;
    // Rows that went down different threads are added in order; a block leaves one partial sum.
    for (int t = 0; t < TT; ++t) {
        if (t >= a.t) break;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < TT; ++k)
                if (k == t) v = dx[k][j];
            red[(ty * across + tx) * C + j] = v;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < across * C; i += 256) {
            const int col = blockIdx.x * across * C + i;
            if (col >= a.dp) continue;
            float s = 0.f;
            for (int k = 0; k < down; ++k) s += red[k * across * C + i];
            a.dxp[((int64_t)blockIdx.y * a.t + t) * a.dp + col] = s;
        }
    }
}

// dx from the blocks' partial sums: 16 quads of columns x 16 shares of the partial sums a block, joined in order.
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

template <class T, int TT>
void grads(const FewArgs& a, hipStream_t st) {
    // 16 bytes a thread, four columns where registers are short
    constexpr int C = TT > 8 ? 4 : 16 / sizeof(T);
    FewArgs b = a;
    b.across = few_across(a.d, C);
    const dim3 grid((a.d + b.across * C - 1) / (b.across * C), a.parts);
    k_few_grads<T, TT, C><<<grid, 256, 0, st>>>(b);
}

}  // namespace

int few_across(int d, int columns) {
    int n = 8;
    while (n < 256 && n * columns < d) n *= 2;
    return n;
}

template <class T>
hipError_t launch_few_logits(const FewArgs& a, int blocks, hipStream_t st) {
    constexpr int N = 16 / sizeof(T);
    const int steps = (a.d + 4 * N - 1) / (4 * N);
    const size_t lds = std::max<size_t>((size_t)a.t * (steps * 64 + 16), kWaves * 16 * sizeof(float2));
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)k_few_logits<T>, hipFuncAttributeMaxDynamicSharedMemorySize, kFewLds);
        if (e != hipSuccess) return e;
    }
    k_few_logits<T><<<blocks, kWaves * 64, lds, st>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t launch_few_grads(const FewArgs& a, T* dx, int64_t lddx, hipStream_t st) {
    if (a.t <= 1) grads<T, 1>(a, st);
    else if (a.t <= 2) grads<T, 2>(a, st);
    else if (a.t <= 4) grads<T, 4>(a, st);
    else if (a.t <= 8) grads<T, 8>(a, st);
    else grads<T, 16>(a, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !dx) return e;
    k_few_finish<T><<<a.t * ((a.dp / 4 + 15) / 16), 256, 0, st>>>(a, a.parts, dx, lddx);
    return hipGetLastError();
}

template hipError_t launch_few_logits<float>(const FewArgs&, int, hipStream_t);
template hipError_t launch_few_logits<__bf16>(const FewArgs&, int, hipStream_t);
template hipError_t launch_few_logits<_Float16>(const FewArgs&, int, hipStream_t);
template hipError_t launch_few_grads<float>(const FewArgs&, float*, int64_t, hipStream_t);
template hipError_t launch_few_grads<__bf16>(const FewArgs&, __bf16*, int64_t, hipStream_t);
template hipError_t launch_few_grads<_Float16>(const FewArgs&, _Float16*, int64_t, hipStream_t);

}  // namespace ccdops
