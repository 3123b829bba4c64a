// The best continuations of beams, and the beams' states in their order (gfx950).
//
// Beam b continued by item i has the score  s_b + z_bi - L_b,  L_b = log sum_j exp z_bj.  Within a beam the order is that of z, which is
// exact in 32 bits: a row leaves its k greatest keys (z, then the lowest item).  Between beams scores are compared in 64 bits.
#include <cmath>

#include "ccdpp_seq.h"
#include "ops_internal.hpp"

namespace ccdops {
namespace {

constexpr int kMost = 64;  // beams of a group, and continuations

// Descending order as a whole number: NaN first, -0 as 0.  The key of -inf is kNone.
constexpr uint32_t kNone = 0x007FFFFFu;
__device__ __forceinline__ uint32_t order_of(float z) {
    if (z != z) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(z + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    if (o == 0xFFFFFFFFu) return NAN;
    return __uint_as_float(o >> 31 ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ uint64_t order_of(double z) {
    if (z != z) return ~0ull;
    const uint64_t u = (uint64_t)__double_as_longlong(z + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}

struct Beam {
    int64_t groups, v, ld, end;
    int beams, k;
    const void* logits;
    const float *score, *offset;
    const uint8_t* done;
    float* out_score;
    int64_t *parent, *item;
    uint8_t* out_done;
    double* sums;     // L of each row
    uint64_t* keys;   // k of each row, descending; 0: none
};

template <class T>
__device__ __forceinline__ float logit(const Beam& a, int64_t row, int64_t i) {
    const float z = (float)((const T*)a.logits)[row * a.ld + i];
    if (!a.offset) return z;
    const float o = a.offset[i];
    return o < -1e38f ? -INFINITY : z + o;
}

template <class V, class F>
__device__ __forceinline__ V block_join(V v, V* red, F&& f) {
    for (int k = 32; k > 0; k >>= 1) v = f(v, __shfl_xor(v, k));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) v = f(v, red[w]);
    return v;
}

// One block a row, which it reads k + 2 times.
template <class T>
__global__ __launch_bounds__(256) void k_beam_rows(Beam a) {
    __shared__ uint64_t red[4];
    const int64_t row = blockIdx.x;
    const float s = a.score[row];
    if (s == -INFINITY || (a.done && a.done[row])) return;
    uint32_t top = 0;
    for (int64_t i = threadIdx.x; i < a.v; i += 256) top = max(top, order_of(logit<T>(a, row, i)));
    top = (uint32_t)block_join((uint64_t)top, red, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
    const float m = value_of(top);
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < a.v; i += 256) {
        const float z = logit<T>(a, row, i);
        sum += z == -INFINITY ? 0.0 : exp((double)z - m);
    }
    sum = block_join(sum, (double*)red, [](double p, double q) { return p + q; });
    if (threadIdx.x == 0) a.sums[row] = top == kNone ? -INFINITY : m + log(sum);
    uint64_t last = ~0ull;
    for (int j = 0; j < a.k; ++j) {
        uint64_t best = 0;
        for (int64_t i = threadIdx.x; i < a.v; i += 256) {
            const uint32_t o = order_of(logit<T>(a, row, i));
            const uint64_t key = (uint64_t)o << 32 | (uint32_t)~(uint32_t)i;
            if (o != kNone && key < last && key > best) best = key;
        }
        last = block_join(best, red, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
        if (threadIdx.x == 0) a.keys[row * a.k + j] = last;
    }
}

// One wave a group: lane b goes down the list of beam b.
__global__ __launch_bounds__(64) void k_beam_join(Beam a) {
    const int64_t g = blockIdx.x;
    const int b = threadIdx.x;
    const int64_t row = g * a.beams + b;
    float s = -INFINITY;
    bool done = false;
    if (b < a.beams) s = a.score[row], done = a.done && a.done[row];
    const bool live = s != -INFINITY;
    const double sum = live && !done ? a.sums[row] : 0.0;
    int at = 0;
    for (int j = 0; j < a.k; ++j) {
        double value = -INFINITY;
        int64_t item = -1;
        if (live && done && at == 0) value = s, item = a.end;
        if (live && !done && at < a.k) {
            const uint64_t key = a.keys[row * a.k + at];
            if (key) value = s + ((double)value_of((uint32_t)(key >> 32)) - sum), item = (uint32_t)~(uint32_t)key;
        }
        const uint64_t mine = order_of(value);
        uint64_t best = mine;
        for (int k = 32; k > 0; k >>= 1) {
            const uint64_t o = __shfl_xor(best, k);
            best = o > best ? o : best;
        }
        const bool none = best == order_of((double)-INFINITY);
        const uint64_t who = __ballot(mine == best);
        const int winner = __ffsll((unsigned long long)who) - 1;
        if (b == winner) {
            const int64_t out = g * a.k + j;
            a.out_score[out] = none ? -INFINITY : (float)value;
            a.parent[out] = none ? -1 : b;
            a.item[out] = none ? -1 : item;
            if (a.out_done) a.out_done[out] = none || item == a.end;
            ++at;
        }
    }
}

constexpr int kTable = 16;  // tensors a launch

struct Moves {
    const char* in[kTable];
    char* out[kTable];
    int64_t stride[kTable], bytes[kTable];
    const int64_t* parent;
    int beams, k, n;
};

__global__ __launch_bounds__(256) void k_reorder(Moves m) {
    const int64_t at = blockIdx.x, g = at / m.k, parent = m.parent[at];
    const bool there = parent >= 0 && parent < m.beams;
    for (int t = 0; t < m.n; ++t) {
        const char* from = m.in[t] + (g * m.beams + (there ? parent : 0)) * m.stride[t];
        char* to = m.out[t] + at * m.bytes[t];
        for (int64_t i = threadIdx.x; i < m.bytes[t]; i += 256) to[i] = there ? from[i] : (char)0;
    }
}

int check(const ccdpp_beam_t* p) {
    if (!p) return fail(CCDPP_EINVAL, "the problem is NULL");
    if (p->groups < 0 || p->groups >= 1 << 24) return fail(CCDPP_EINVAL, "groups must be in [0, 2^24)");
    if (p->beams < 1 || p->beams > kMost || p->k < 1 || p->k > kMost) return fail(CCDPP_EINVAL, "beams and k must be in [1, 64]");
    if (p->v < 1 || p->v >= 1 << 28) return fail(CCDPP_EINVAL, "v must be in [1, 2^28)");
    if (p->dtype < CCDPP_F32 || p->dtype > CCDPP_F16) return fail(CCDPP_EINVAL, "dtype must be CCDPP_F32, CCDPP_BF16 or CCDPP_F16");
    if (p->ld < p->v) return fail(CCDPP_EINVAL, "ld must be at least v");
    if (p->end < -1 || p->end >= p->v) return fail(CCDPP_EINVAL, "end must be an item, or -1");
    if (p->done && p->end < 0) return fail(CCDPP_EINVAL, "done needs the item that ends a beam");
    if (p->reserved) return fail(CCDPP_EINVAL, "reserved must be 0");
    return CCDPP_OK;
}

int64_t workspace(const ccdpp_beam_t* p) { return round_up(p->groups * p->beams * 8 * (1 + (int64_t)p->k), 256) + 256; }

}  // namespace
}  // namespace ccdops

extern "C" {

int ccdpp_beam_workspace(const ccdpp_beam_t* p, int64_t* bytes) {
    using namespace ccdops;
    if (!bytes) return fail(CCDPP_EINVAL, "bytes is NULL");
    if (int rc = check(p)) return rc;
    *bytes = workspace(p);
    return CCDPP_OK;
}

int ccdpp_beam_select(const ccdpp_beam_t* p, float* out_score, int64_t* parent, int64_t* item, uint8_t* out_done, void* ws, int64_t ws_bytes,
                      void* stream) {
    using namespace ccdops;
    if (int rc = check(p)) return rc;
    const int64_t rows = p->groups * p->beams;
    if (rows > 0 && (!p->logits || !p->score || !out_score || !parent || !item)) return fail(CCDPP_EINVAL, "logits, score and outputs must be non-NULL");
    if ((uintptr_t)p->logits % (p->dtype == CCDPP_F32 ? 4 : 2) || (uintptr_t)p->score % 4 || (uintptr_t)p->offset % 4 || (uintptr_t)out_score % 4 ||
        (uintptr_t)parent % 8 || (uintptr_t)item % 8)
        return fail(CCDPP_EINVAL, "pointers must be aligned to their types");
    if (!ws || (uintptr_t)ws % 256 || ws_bytes < workspace(p)) return fail(CCDPP_EINVAL, "the workspace is too small or not aligned to 256 bytes");
    if (int rc = check_device()) return rc;
    if (rows == 0) return CCDPP_OK;
    Beam a = {p->groups, p->v, p->ld, p->end, p->beams, p->k, p->logits, p->score, p->offset, p->done, out_score, parent, item, out_done,
              (double*)ws, (uint64_t*)ws + rows};
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == CCDPP_F32) k_beam_rows<float><<<(unsigned)rows, 256, 0, st>>>(a);
    else if (p->dtype == CCDPP_BF16) k_beam_rows<__bf16><<<(unsigned)rows, 256, 0, st>>>(a);
    else k_beam_rows<_Float16><<<(unsigned)rows, 256, 0, st>>>(a);
    k_beam_join<<<(unsigned)p->groups, 64, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CCDPP_OK : hip_fail(e, "beam selection");
}

int ccdpp_beam_reorder(int64_t groups, int32_t beams, int32_t k, const int64_t* parent, int32_t n, const void* const* in, const int64_t* in_stride,
                       void* const* out, const int64_t* row_bytes, void* stream) {
    using namespace ccdops;
    if (groups < 0 || groups >= 1 << 24) return fail(CCDPP_EINVAL, "groups must be in [0, 2^24)");
    if (beams < 1 || beams > kMost || k < 1 || k > kMost) return fail(CCDPP_EINVAL, "beams and k must be in [1, 64]");
    if (n < 0 || (n > 0 && (!in || !in_stride || !out || !row_bytes))) return fail(CCDPP_EINVAL, "n must be >= 0 and the tables of tensors non-NULL");
    if (groups > 0 && (!parent || (uintptr_t)parent % 8)) return fail(CCDPP_EINVAL, "parent must be non-NULL and aligned to its type");
    for (int32_t i = 0; i < n; ++i) {
        if (row_bytes[i] < 0 || in_stride[i] < row_bytes[i]) return fail(CCDPP_EINVAL, "row_bytes must be >= 0, and rows no less apart");
        if (groups > 0 && row_bytes[i] > 0 && (!in[i] || !out[i])) return fail(CCDPP_EINVAL, "a tensor is NULL");
    }
    if (int rc = check_device()) return rc;
    if (groups == 0) return CCDPP_OK;
    Moves m;
    m.parent = parent, m.beams = beams, m.k = k, m.n = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (row_bytes[i]) m.in[m.n] = (const char*)in[i], m.out[m.n] = (char*)out[i], m.stride[m.n] = in_stride[i], m.bytes[m.n] = row_bytes[i], ++m.n;
        if (!m.n || (m.n < kTable && i + 1 < n)) continue;
        k_reorder<<<(unsigned)(groups * k), 256, 0, (hipStream_t)stream>>>(m);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "beam reordering");
        m.n = 0;
    }
    return CCDPP_OK;
}

}  // extern "C"
