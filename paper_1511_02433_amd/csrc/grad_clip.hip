// Global norm of many gradient tensors, and their clipping (gfx950).
//
//   norm = sqrt(sum_i sum_j g_ij^2),   out_i = c g_i,   c = min(1, max_norm / (norm + eps))
//
// Bound by memory: the gradients are read once for the norm, and once more and written for the clipping.  The tensors
// of a launch come as a table in the kernel's arguments, cut into chunks of kChunk values that the blocks take in
// turn; squares are summed in 64 bits, so no gradient that its type can hold overflows them.  Every block leaves one
// partial sum, and later launches (more than kTable tensors) add to it, in stream order: the result does not depend on timing.
// (10^9 bfloat16 in 60 tensors: 477 us for the norm, 4.2 TB/s, and 715 for the clipping, 5.6 TB/s, of a copy's 5.15; 2 10^7 floats in
// 7: 15.5 and 27.4 us.)
#include <algorithm>
#include <cmath>

#include "ops_internal.hpp"

namespace ccdops {
namespace {

constexpr int kTable = 64;      // tensors per launch
constexpr int kBlocks = 1024;   // partial sums
constexpr int64_t kChunk = 8192;
// What one block takes in one launch: kMine chunks of kLittleChunk bytes for each of its waves.  (49,000 floats by one
// block 10.4 us a call, the host's share included, 52,000 by two launches 13.5; more chunks would not stay in registers.)
constexpr int kMine = 6;
constexpr int64_t kLittleChunk = 2048;

struct Table {
    const void* in[kTable];
    void* out[kTable];
    int64_t size[kTable];
    int64_t first[kTable];   // first chunk of each tensor
    int32_t dtype[kTable];
    int n;
    int64_t chunks;
};

template <class T>
__device__ __forceinline__ double chunk_squares(const void* base, int64_t lo, int64_t n, int lane, int lanes) {
    const T* g = (const T*)base + lo;
    constexpr int W = 16 / sizeof(T);
    double s = 0.0;
    for (int64_t k = lane; k < n / W; k += lanes) {
        const Run<T, W> q = load_run<W>(g + k * W);
        for (int j = 0; j < W; ++j) s += (double)(float)q.v[j] * (double)(float)q.v[j];
    }
    for (int64_t i = n / W * W + lane; i < n; i += lanes) s += (double)(float)g[i] * (double)(float)g[i];
    return s;
}

template <class T>
__device__ __forceinline__ void chunk_scale(const void* base, void* out, int64_t lo, int64_t n, float c, int lane, int lanes) {
    const T* g = (const T*)base + lo;
    T* o = (T*)out + lo;
    constexpr int W = 16 / sizeof(T);
    for (int64_t k = lane; k < n / W; k += lanes) {
        Run<T, W> q = load_run<W>(g + k * W);
        for (int j = 0; j < W; ++j) q.v[j] = (T)((float)q.v[j] * c);
        store_run<W>(o + k * W, q);
    }
    for (int64_t i = n / W * W + lane; i < n; i += lanes) o[i] = (T)((float)g[i] * c);
}

// The tensor that a chunk belongs to.
__device__ __forceinline__ int find(const Table& t, int64_t chunk) {
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double s, double* red) {
    for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    double all = 0.0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) all += red[w];
    return all;
}

template <class F>
__device__ __forceinline__ void typed(int dtype, F&& body) {
    if (dtype == CCDPP_F32) body(float());
    else if (dtype == CCDPP_BF16) body((__bf16)0.f);
    else body((_Float16)0.f);
}

__global__ __launch_bounds__(256) void k_squares(Table t, double* parts, int add) {
    __shared__ double red[4];
    double s = 0.0;
    for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int i = find(t, c);
        const int64_t lo = (c - t.first[i]) * kChunk, n = min(kChunk, t.size[i] - lo);
        typed(t.dtype[i], [&](auto z) { s += chunk_squares<decltype(z)>(t.in[i], lo, n, threadIdx.x, 256); });
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) parts[blockIdx.x] = add ? parts[blockIdx.x] + s : s;
}

// The norm from kBlocks partial sums in a fixed order, by 256 threads.
__device__ __forceinline__ float norm_of(const double* parts, double* red) {
    double s = 0.0;
    for (int i = threadIdx.x; i < kBlocks; i += 256) s += parts[i];
    return (float)sqrt(block_sum(s, red));
}

__global__ __launch_bounds__(256) void k_norm(const double* parts, float* norm) {
    __shared__ double red[4];
    const float n = norm_of(parts, red);
    if (threadIdx.x == 0) *norm = n;
}

// min(1, max_norm / (norm + eps)); NaN for a norm that is NaN, 1 without a limit.
__device__ __forceinline__ float clip_factor(float norm, float max_norm, float eps) {
    if (norm != norm) return norm;
    return isinf(max_norm) || norm + eps <= max_norm ? 1.f : max_norm / (norm + eps);
}

// Every block adds up the partial sums itself (8 KB from L2), which saves a launch; block 0 leaves the norm.  The
// chunks that were read last come first: the memory-side cache may still hold them.
__global__ __launch_bounds__(256) void k_scale(Table t, const double* parts, float* norm, float max_norm, float eps) {
    __shared__ double red[4];
    const float nv = norm_of(parts, red);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = nv;
    const float c = clip_factor(nv, max_norm, eps);
    for (int64_t k = t.chunks - 1 - blockIdx.x; k >= 0; k -= gridDim.x) {
        const int i = find(t, k);
        if (c == 1.f && t.out[i] == t.in[i]) continue;
        const int64_t lo = (k - t.first[i]) * kChunk, n = min(kChunk, t.size[i] - lo);
        typed(t.dtype[i], [&](auto z) { chunk_scale<decltype(z)>(t.in[i], t.out[i], lo, n, c, threadIdx.x, 256); });
    }
}

// Little in all: one block, one launch.  Its time is that of the round trips to memory, so there is one: a wave reads
// all its chunks at once, two runs of 16 bytes a lane, and a thread one of the values that tensors have over (eight
// threads a tensor); all are kept for the clipping.  A choice between accesses would wait for them, so that of the types
// comes after them.
__global__ __launch_bounds__(1024) void k_little(Table t, int clip, float* norm, float max_norm, float eps) {
    typedef Loose<2>::four loose;
    __shared__ double red[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int first = lane < t.n ? (int)t.first[lane] : INT32_MAX;
    const int mine = min((int)threadIdx.x >> 3, kTable - 1);
    int type = t.dtype[mine];
    int64_t size = t.size[mine], from = (int64_t)t.in[mine];
    asm volatile("" : "+v"(first), "+v"(type), "+v"(size), "+v"(from));  // are there before the reads below, which are not to be waited for
    words4 run[kMine][2] = {};
    // body(tensor, first byte, bytes of the chunk, its runs)
    const auto each = [&](auto&& body) {
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int chunk = wave + 16 * k;
            if (chunk < t.chunks) {
                const int i = __popcll(__ballot(first <= chunk)) - 1;
                const int64_t lo = (chunk - t.first[i]) * kLittleChunk, all = t.size[i] << (t.dtype[i] == CCDPP_F32 ? 2 : 1);
                body(i, lo, (int)min(kLittleChunk, all - lo), run[k]);
            }
        }
    };
    each([&](int i, int64_t lo, int n, words4* q) {
        const char* const g = (const char*)t.in[i] + lo;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (j * 1024 + lane * 16 + 16 <= n) q[j] = *(const loose*)(g + j * 1024 + lane * 16);
    });
    const int per = type == CCDPP_F32 ? 4 : 8;
    const int64_t at = size / per * per + (threadIdx.x & 7);
    const bool has = (int)threadIdx.x >> 3 < t.n && at < size;
    float over = 0.f;
    if (has) typed(type, [&](auto z) { over = (float)((const decltype(z)*)from)[at]; });
    double s = (double)over * (double)over;
    each([&](int i, int64_t, int, words4* q) {
        typed(t.dtype[i], [&](auto z) {
            typedef decltype(z) T;
            constexpr int W = 16 / sizeof(T);
#pragma unroll
            for (int j = 0; j < 2 * W; ++j) {
                const float v = (float)__builtin_bit_cast(Run<T, W>, q[j / W]).v[j % W];
                s += (double)v * (double)v;
            }
        });
    });
    const float nv = (float)sqrt(block_sum(s, red));
    if (threadIdx.x == 0) *norm = nv;
    if (!clip) return;
    const float c = clip_factor(nv, max_norm, eps);
    const auto as_it_is = [&](int i) { return c == 1.f && t.out[i] == t.in[i]; };
    each([&](int i, int64_t lo, int n, words4* q) {
        if (as_it_is(i)) return;
        char* const o = (char*)t.out[i] + lo;
        typed(t.dtype[i], [&](auto z) {
            typedef decltype(z) T;
            constexpr int W = 16 / sizeof(T);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                Run<T, W> r = __builtin_bit_cast(Run<T, W>, q[j]);
#pragma unroll
                for (int w = 0; w < W; ++w) r.v[w] = (T)((float)r.v[w] * c);
                if (j * 1024 + lane * 16 + 16 <= n) store_run<W>((T*)(o + j * 1024 + lane * 16), r);
            }
        });
    });
    if (has && !as_it_is(mine)) typed(type, [&](auto z) { ((decltype(z)*)t.out[mine])[at] = (decltype(z))(over * c); });
}

int64_t size_of(int32_t dtype) { return dtype == CCDPP_F32 ? 4 : 2; }

// Chunks of whole runs of 16 bytes.
int64_t little_chunks(int64_t size, int32_t dtype) { return (size * size_of(dtype) / 16 * 16 + kLittleChunk - 1) / kLittleChunk; }

int run(bool clip, int32_t n, const void* const* in, void* const* out, const int64_t* sizes, const int32_t* dtypes, float max_norm, float eps,
        float* norm, void* ws, int64_t ws_bytes, void* stream) {
    if (n < 0) return fail(CCDPP_EINVAL, "n must be >= 0");
    if (n > 0 && (!in || !sizes || !dtypes || (clip && !out))) return fail(CCDPP_EINVAL, "the tables of tensors must be non-NULL");
    if (!norm) return fail(CCDPP_EINVAL, "norm must be non-NULL");
    if (clip && (!(max_norm >= 0.f) || !(eps >= 0.f) || std::isinf(eps))) return fail(CCDPP_EINVAL, "max_norm must be >= 0 and eps finite and >= 0");
    for (int32_t i = 0; i < n; ++i) {
        if (sizes[i] < 0) return fail(CCDPP_EINVAL, "a tensor's size is negative");
        if (dtypes[i] < CCDPP_F32 || dtypes[i] > CCDPP_F16) return fail(CCDPP_EINVAL, "dtypes must be CCDPP_F32, CCDPP_BF16 or CCDPP_F16");
        if (sizes[i] > 0 && (!in[i] || (clip && !out[i]))) return fail(CCDPP_EINVAL, "a tensor is NULL");
        const uintptr_t es = size_of(dtypes[i]);
        if (sizes[i] > 0 && ((uintptr_t)in[i] % es || (clip && (uintptr_t)out[i] % es))) return fail(CCDPP_EINVAL, "a tensor is not aligned to its type");
    }
    if (!ws || (uintptr_t)ws % 256 || ws_bytes < kBlocks * 8) return fail(CCDPP_EINVAL, "the workspace is too small or not aligned to 256 bytes");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    double* parts = (double*)ws;
    Table t;
    t.n = 0, t.chunks = 0;
    bool little = false;
    const auto add = [&](int32_t i) {
        t.in[t.n] = in[i], t.out[t.n] = clip ? out[i] : nullptr;
        t.size[t.n] = sizes[i], t.first[t.n] = t.chunks, t.dtype[t.n] = dtypes[i];
        t.chunks += little ? little_chunks(sizes[i], dtypes[i]) : (sizes[i] + kChunk - 1) / kChunk;
        ++t.n;
    };
    int64_t filled = 0, pieces = 0;
    for (int32_t i = 0; i < n; ++i)
        if (sizes[i]) ++filled, pieces += little_chunks(sizes[i], dtypes[i]);
    if (filled <= kTable && pieces <= 16 * kMine) {
        little = true;
        for (int32_t i = 0; i < n; ++i)
            if (sizes[i]) add(i);
        k_little<<<1, 1024, 0, st>>>(t, clip, norm, max_norm, eps);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? CCDPP_OK : hip_fail(e, "gradient norm");
    }
    for (int pass = 0; pass < (clip ? 2 : 1); ++pass) {
        bool first = true;
        for (int32_t i = 0; i < n; ++i) {
            if (sizes[i]) add(i);
            if (!t.n || (t.n < kTable && i + 1 < n)) continue;
            if (pass == 0) k_squares<<<first ? kBlocks : (int)std::min<int64_t>(kBlocks, t.chunks), 256, 0, st>>>(t, parts, !first);
            else k_scale<<<(unsigned)std::min<int64_t>(4 * kBlocks, t.chunks), 256, 0, st>>>(t, parts, norm, max_norm, eps);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return hip_fail(e, "gradient norm");
            first = false;
            t.n = 0, t.chunks = 0;
        }
    }
    if (!clip) {
        k_norm<<<1, 256, 0, st>>>(parts, norm);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gradient norm");
    }
    return CCDPP_OK;
}

}  // namespace
}  // namespace ccdops

extern "C" {

int ccdpp_grad_norm_workspace(int64_t* bytes) {
    if (!bytes) return ccdops::fail(CCDPP_EINVAL, "bytes is NULL");
    *bytes = ccdops::kBlocks * 8;
    return CCDPP_OK;
}

int ccdpp_grad_norm(int32_t n, const void* const* tensors, const int64_t* sizes, const int32_t* dtypes, float* norm, void* workspace,
                    int64_t workspace_bytes, void* stream) {
    return ccdops::run(false, n, tensors, nullptr, sizes, dtypes, 0.f, 0.f, norm, workspace, workspace_bytes, stream);
}

int ccdpp_clip_grads(int32_t n, const void* const* tensors, void* const* out, const int64_t* sizes, const int32_t* dtypes, float max_norm,
                     float eps, float* norm, void* workspace, int64_t workspace_bytes, void* stream) {
    return ccdops::run(true, n, tensors, out, sizes, dtypes, max_norm, eps, norm, workspace, workspace_bytes, stream);
}

}  // extern "C"
