// Gated linear recurrences over packed sequences, their gradients, and one more row of each (gfx950).
//
//   h_t = a_t h_(t-1) + u_t;   GIVEN: a = gate, u = x;   SIGMOID: a = 1 / (1 + e^-gate), u = (1 - a) x
//   l_t = dy_t + a_(t+1) l_(t+1);   dx_t = l_t (times 1 - a_t),  dgate_t = l_t h_(t-1)  (or l_t (h_(t-1) - x_t) a_t (1 - a_t))
#include "ccdpp_seq.h"
#include "ops_internal.hpp"

namespace ccdops {
namespace {

constexpr int kKeep = 16;  // rows for each state that is kept

// Both a and 1 - a to some 2^-22 of themselves, for gates of either sign: e = exp(-|gate|), with what the product by log2 e
// rounds off put back.
struct Gate { float a, rest; };
__device__ __forceinline__ Gate sigmoid_of(float gate) {
    const float z = -fabsf(gate), p = z * 1.44269504f;
    const float off = fmaf(z, 1.44269504f, -p) + z * 1.92596299e-8f;  // z log2 e - p
    float e = __builtin_amdgcn_exp2f(p);
    e = p > -200.f ? fmaf(e, off * 0.693147181f, e) : e;
    const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
    return gate >= 0.f ? Gate{big, small} : gate < 0.f ? Gate{small, big} : Gate{gate, gate};
}

struct Terms { float a, u, rest; };
template <bool SIGMOID>
__device__ __forceinline__ Terms terms_of(float x, float gate) {
    if constexpr (!SIGMOID) return {gate, x, 1.f};
    const Gate g = sigmoid_of(gate);
    return {g.a, g.rest * x, g.rest};
}

struct Scan {
    int64_t n, s, ldx, ldg, ldy, lddx, lddg;
    int d, bits;
    const void *x, *gate, *starts;
    const float *initial, *dlast, *kept;
    void *y, *dx, *dgate;  // y: the states, or dy
    float *last, *keep, *dinitial;
};

__device__ __forceinline__ int64_t start_of(const Scan& a, int64_t q) {
    const int64_t v = a.bits == 64 ? ((const int64_t*)a.starts)[q] : ((const int32_t*)a.starts)[q];
    return min(max(v, (int64_t)0), a.n);
}

// Rows that belong to no sequence get zeros; a block takes rows in turn.
template <class T>
__global__ __launch_bounds__(256) void k_outside(Scan a, void* y, int64_t ldy) {
    const int64_t lo = a.s ? start_of(a, 0) : a.n, hi = a.s ? start_of(a, a.s) : a.n;
    for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
        if (r >= lo && r < hi) continue;
        for (int c = threadIdx.x; c < a.d; c += 256) ((T*)y)[r * ldy + c] = (T)0.f;
    }
}

// A thread for each sequence and column.
template <class T, bool SIGMOID>
__global__ __launch_bounds__(64) void k_scan(Scan a) {
    const int64_t q = blockIdx.x;
    const int64_t lo = start_of(a, q), hi = start_of(a, q + 1);
    for (int c = threadIdx.x; c < a.d; c += 64) {
        float h = a.initial ? a.initial[q * a.d + c] : 0.f;
        for (int64_t t = lo; t < hi; ++t) {
            if (a.keep && t % kKeep == 0) a.keep[t / kKeep * a.d + c] = h;
            const Terms m = terms_of<SIGMOID>((float)((const T*)a.x)[t * a.ldx + c], (float)((const T*)a.gate)[t * a.ldg + c]);
            h = fmaf(m.a, h, m.u);
            ((T*)a.y)[t * a.ldy + c] = (T)h;
        }
        if (a.last) a.last[q * a.d + c] = h;
    }
}

template <class T, bool SIGMOID>
__global__ __launch_bounds__(64) void k_scan_grad(Scan a) {
    const int64_t q = blockIdx.x;
    const int64_t lo = start_of(a, q), hi = start_of(a, q + 1);
    for (int c = threadIdx.x; c < a.d; c += 64) {
        float m = a.dlast ? a.dlast[q * a.d + c] : 0.f;
        for (int64_t t = hi - 1; t >= lo; --t) {
            // The state before row t, from what was kept last.
            const int64_t from = max(t / kKeep * kKeep, lo);
            float h = from == lo ? (a.initial ? a.initial[q * a.d + c] : 0.f) : a.kept[t / kKeep * a.d + c];
            for (int64_t i = from; i < t; ++i) {
                const Terms w = terms_of<SIGMOID>((float)((const T*)a.x)[i * a.ldx + c], (float)((const T*)a.gate)[i * a.ldg + c]);
                h = fmaf(w.a, h, w.u);
            }
            const float x = (float)((const T*)a.x)[t * a.ldx + c];
            const Terms w = terms_of<SIGMOID>(x, (float)((const T*)a.gate)[t * a.ldg + c]);
            const float l = (float)((const T*)a.y)[t * a.ldy + c] + m;
            ((T*)a.dx)[t * a.lddx + c] = (T)(SIGMOID ? w.rest * l : l);
            ((T*)a.dgate)[t * a.lddg + c] = (T)(SIGMOID ? l * (h - x) * (w.a * w.rest) : l * h);
            m = w.a * l;
        }
        if (a.dinitial) a.dinitial[q * a.d + c] = m;
    }
}

template <class T, bool SIGMOID>
__global__ __launch_bounds__(256) void k_step(int64_t n, int d, const T* x, int64_t ldx, const T* gate, int64_t ldg, float* state, int64_t lds, T* y,
                                              int64_t ldy) {
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n * d; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / d, c = i - r * d;
        const Terms w = terms_of<SIGMOID>((float)x[r * ldx + c], (float)gate[r * ldg + c]);
        const float h = fmaf(w.a, state[r * lds + c], w.u);
        state[r * lds + c] = h;
        y[r * ldy + c] = (T)h;
    }
}

// body(a value of the type, whether the gate goes through a sigmoid)
template <class F>
void typed(int dtype, int mode, F&& body) {
    const auto of = [&](auto z) {
        if (mode == CCDPP_SCAN_SIGMOID) body(z, std::true_type());
        else body(z, std::false_type());
    };
    if (dtype == CCDPP_F32) of(float());
    else if (dtype == CCDPP_BF16) of((__bf16)0.f);
    else of((_Float16)0.f);
}

int check(const ccdpp_scan_t* p) {
    if (!p) return fail(CCDPP_EINVAL, "the problem is NULL");
    if (p->n < 0 || p->n >= (int64_t)1 << 31 || p->s < 0 || p->s >= (int64_t)1 << 31) return fail(CCDPP_EINVAL, "n and s must be in [0, 2^31)");
    if (p->d < 1 || p->d > 65536) return fail(CCDPP_EINVAL, "d must be in [1, 65536]");
    if (p->dtype < CCDPP_F32 || p->dtype > CCDPP_F16) return fail(CCDPP_EINVAL, "dtype must be CCDPP_F32, CCDPP_BF16 or CCDPP_F16");
    if (p->mode != CCDPP_SCAN_GIVEN && p->mode != CCDPP_SCAN_SIGMOID) return fail(CCDPP_EINVAL, "mode must be CCDPP_SCAN_GIVEN or CCDPP_SCAN_SIGMOID");
    if (p->starts_bits != 32 && p->starts_bits != 64) return fail(CCDPP_EINVAL, "starts_bits must be 32 or 64");
    if (p->ldx < p->d || p->ldg < p->d) return fail(CCDPP_EINVAL, "ldx and ldg must be at least d");
    return CCDPP_OK;
}

bool misaligned(const void* p, uintptr_t bytes) { return (uintptr_t)p % bytes != 0; }

int check_pointers(const ccdpp_scan_t* p, const void* kept, const void* ws, int64_t ws_bytes, int64_t need) {
    const uintptr_t es = p->dtype == CCDPP_F32 ? 4 : 2;
    if ((p->n > 0 && (!p->x || !p->gate)) || !p->starts) return fail(CCDPP_EINVAL, "x, gate and starts must be non-NULL");
    if (misaligned(p->x, es) || misaligned(p->gate, es) || misaligned(p->starts, p->starts_bits / 8) || misaligned(p->initial, 4) || misaligned(kept, 16))
        return fail(CCDPP_EINVAL, "pointers must be aligned to their types, and kept to 16 bytes");
    if (!ws || misaligned(ws, 256) || ws_bytes < need) return fail(CCDPP_EINVAL, "the workspace is too small or not aligned to 256 bytes");
    return CCDPP_OK;
}

int64_t workspace(const ccdpp_scan_t*, int32_t) { return 256; }

}  // namespace
}  // namespace ccdops

extern "C" {

int ccdpp_scan_workspace(const ccdpp_scan_t* p, int32_t call, int64_t* bytes) {
    using namespace ccdops;
    if (!bytes) return fail(CCDPP_EINVAL, "bytes is NULL");
    if (call != CCDPP_SCAN_FORWARD && call != CCDPP_SCAN_GRAD) return fail(CCDPP_EINVAL, "call must be CCDPP_SCAN_FORWARD or CCDPP_SCAN_GRAD");
    if (int rc = check(p)) return rc;
    *bytes = workspace(p, call);
    return CCDPP_OK;
}

int ccdpp_scan_kept(const ccdpp_scan_t* p, int64_t* bytes) {
    using namespace ccdops;
    if (!bytes) return fail(CCDPP_EINVAL, "bytes is NULL");
    if (int rc = check(p)) return rc;
    *bytes = (p->n + kKeep - 1) / kKeep * p->d * 4;
    return CCDPP_OK;
}

int ccdpp_gated_scan(const ccdpp_scan_t* p, void* y, int64_t ldy, float* last, void* kept, void* ws, int64_t ws_bytes, void* stream) {
    using namespace ccdops;
    if (int rc = check(p)) return rc;
    if (int rc = check_pointers(p, kept, ws, ws_bytes, workspace(p, CCDPP_SCAN_FORWARD))) return rc;
    if (p->n > 0 && !y) return fail(CCDPP_EINVAL, "y must be non-NULL");
    if (ldy < p->d) return fail(CCDPP_EINVAL, "ldy must be at least d");
    if (misaligned(y, p->dtype == CCDPP_F32 ? 4 : 2) || misaligned(last, 4)) return fail(CCDPP_EINVAL, "pointers must be aligned to their types");
    if (int rc = check_device()) return rc;
    Scan a = {};
    a.n = p->n, a.s = p->s, a.ldx = p->ldx, a.ldg = p->ldg, a.ldy = ldy, a.d = p->d, a.bits = p->starts_bits;
    a.x = p->x, a.gate = p->gate, a.starts = p->starts, a.initial = p->initial, a.y = y, a.last = last, a.keep = (float*)kept;
    hipStream_t st = (hipStream_t)stream;
    typed(p->dtype, p->mode, [&](auto z, auto sigmoid) {
        typedef decltype(z) T;
        if (a.n) k_outside<T><<<1024, 256, 0, st>>>(a, y, ldy);
        if (a.s) k_scan<T, decltype(sigmoid)::value><<<(unsigned)a.s, 64, 0, st>>>(a);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CCDPP_OK : hip_fail(e, "gated scan");
}

int ccdpp_gated_scan_grad(const ccdpp_scan_t* p, const void* dy, int64_t lddy, const float* dlast, const void* kept, void* dx, int64_t lddx, void* dgate,
                          int64_t lddg, float* dinitial, void* ws, int64_t ws_bytes, void* stream) {
    using namespace ccdops;
    if (int rc = check(p)) return rc;
    if (int rc = check_pointers(p, kept, ws, ws_bytes, workspace(p, CCDPP_SCAN_GRAD))) return rc;
    if (p->n > 0 && (!dy || !kept || !dx || !dgate)) return fail(CCDPP_EINVAL, "dy, kept, dx and dgate must be non-NULL");
    if (lddy < p->d || lddx < p->d || lddg < p->d) return fail(CCDPP_EINVAL, "lddy, lddx and lddg must be at least d");
    const uintptr_t es = p->dtype == CCDPP_F32 ? 4 : 2;
    if (misaligned(dy, es) || misaligned(dx, es) || misaligned(dgate, es) || misaligned(dlast, 4) || misaligned(dinitial, 4))
        return fail(CCDPP_EINVAL, "pointers must be aligned to their types");
    if (int rc = check_device()) return rc;
    Scan a = {};
    a.n = p->n, a.s = p->s, a.ldx = p->ldx, a.ldg = p->ldg, a.ldy = lddy, a.lddx = lddx, a.lddg = lddg, a.d = p->d, a.bits = p->starts_bits;
    a.x = p->x, a.gate = p->gate, a.starts = p->starts, a.initial = p->initial, a.dlast = dlast, a.kept = (const float*)kept;
    a.y = const_cast<void*>(dy), a.dx = dx, a.dgate = dgate, a.dinitial = dinitial;
    hipStream_t st = (hipStream_t)stream;
    typed(p->dtype, p->mode, [&](auto z, auto sigmoid) {
        typedef decltype(z) T;
        if (a.n) k_outside<T><<<1024, 256, 0, st>>>(a, dx, lddx);
        if (a.n) k_outside<T><<<1024, 256, 0, st>>>(a, dgate, lddg);
        if (a.s) k_scan_grad<T, decltype(sigmoid)::value><<<(unsigned)a.s, 64, 0, st>>>(a);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CCDPP_OK : hip_fail(e, "gated scan gradients");
}

int ccdpp_gated_scan_step(int64_t n, int32_t d, int32_t dtype, int32_t mode, const void* x, int64_t ldx, const void* gate, int64_t ldg, float* state,
                          int64_t lds, void* y, int64_t ldy, void* stream) {
    using namespace ccdops;
    ccdpp_scan_t p = {n, 0, d, dtype, mode, 64, x, ldx, gate, ldg, nullptr, nullptr};
    if (int rc = check(&p)) return rc;
    if (lds < d || ldy < d) return fail(CCDPP_EINVAL, "lds and ldy must be at least d");
    if (n > 0 && (!x || !gate || !state || !y)) return fail(CCDPP_EINVAL, "x, gate, state and y must be non-NULL");
    const uintptr_t es = dtype == CCDPP_F32 ? 4 : 2;
    if (misaligned(x, es) || misaligned(gate, es) || misaligned(y, es) || misaligned(state, 4)) return fail(CCDPP_EINVAL, "pointers must be aligned to their types");
    if (int rc = check_device()) return rc;
    if (n == 0) return CCDPP_OK;
    const int64_t blocks = (n * d + 255) / 256;
    typed(dtype, mode, [&](auto z, auto sigmoid) {
        typedef decltype(z) T;
        k_step<T, decltype(sigmoid)::value><<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, (hipStream_t)stream>>>(n, d, (const T*)x, ldx, (const T*)gate, ldg,
                                                                                                                       state, lds, (T*)y, ldy);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CCDPP_OK : hip_fail(e, "gated scan step");
}

}  // extern "C"
