// Global norm of many gradient tensors, and their clipping (gfx950).
//
//   norm = sqrt(sum_i sum_j g_ij^2),   out_i = c g_i,   c = min(1, max_norm / (norm + eps))
//
// Bound by memory: the gradients are read once for the norm, and once more and written for the clipping.  The tensors
// of a launch come as a table in the kernel's arguments, cut into chunks of kChunk values that the blocks take in
// turn; squares are summed in 64 bits, so no gradient that its type can hold overflows them.  Every block leaves one
// partial sum, and later launches (more than kTable tensors) add to it, in stream order: the result does not depend on timing.
#include <algorithm>
#include <cmath>

#include "ops_internal.hpp"

namespace ccdops {
namespace {

constexpr int kTable = 64;      // tensors per launch
constexpr int kBlocks = 1024;   // partial sums
constexpr int64_t kChunk = 8192;
constexpr int64_t kLittle = 32768;  // values that one block takes in one launch
constexpr int64_t kLittleChunk = 512;

struct Table {
    const void* in[kTable];
    void* out[kTable];
    int64_t size[kTable];
    int64_t first[kTable];   // first chunk of each tensor
    uint8_t dtype[kTable];
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

// Little in all (kLittle values): one block, one launch; a wave takes a chunk of kLittleChunk values.
__global__ __launch_bounds__(1024) void k_little(Table t, int clip, float* norm, float max_norm, float eps) {
    __shared__ double red[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const auto each = [&](auto&& body) {
        for (int k = wave; k < (int)t.chunks; k += 16) {
            const int i = find(t, k);
            const int64_t lo = (k - t.first[i]) * kLittleChunk, n = min(kLittleChunk, t.size[i] - lo);
            typed(t.dtype[i], [&](auto z) { body(z, i, lo, n); });
        }
    };
    double s = 0.0;
    each([&](auto z, int i, int64_t lo, int64_t n) { s += chunk_squares<decltype(z)>(t.in[i], lo, n, lane, 64); });
    const float nv = (float)sqrt(block_sum(s, red));
    if (threadIdx.x == 0) *norm = nv;
    if (!clip) return;
    const float c = clip_factor(nv, max_norm, eps);
    each([&](auto z, int i, int64_t lo, int64_t n) {
        if (c != 1.f || t.out[i] != t.in[i]) chunk_scale<decltype(z)>(t.in[i], t.out[i], lo, n, c, lane, 64);
    });
}

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
        const uintptr_t es = dtypes[i] == CCDPP_F32 ? 4 : 2;
        if (sizes[i] > 0 && ((uintptr_t)in[i] % es || (clip && (uintptr_t)out[i] % es))) return fail(CCDPP_EINVAL, "a tensor is not aligned to its type");
    }
    if (!ws || (uintptr_t)ws % 256 || ws_bytes < kBlocks * 8) return fail(CCDPP_EINVAL, "the workspace is too small or not aligned to 256 bytes");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    double* parts = (double*)ws;
    Table t;
    int64_t values = 0;
    t.n = 0, t.chunks = 0;
    int64_t chunk = kChunk;
    const auto add = [&](int32_t i) {
        t.in[t.n] = in[i], t.out[t.n] = clip ? out[i] : nullptr;
        t.size[t.n] = sizes[i], t.first[t.n] = t.chunks, t.dtype[t.n] = (uint8_t)dtypes[i];
        t.chunks += (sizes[i] + chunk - 1) / chunk;
        ++t.n;
    };
    int32_t filled = 0;
    for (int32_t i = 0; i < n; ++i)
        if (sizes[i]) ++filled, values += sizes[i];
    if (filled <= kTable && values <= kLittle) {
        chunk = kLittleChunk;
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
