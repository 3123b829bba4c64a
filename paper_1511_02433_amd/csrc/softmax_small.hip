// Softmax loss and gradients where rows have few factors (d <= 128): the products pass G from registers to registers.
//
// A block keeps 128 rows of one side (four waves of 32), their fragments in registers, and streams the other side
// through LDS, 32 rows at a time.  The logits of a 32 x 32 tile come as an accumulator whose lanes hold one kept row and 16
// streamed ones: sums over the streamed side are sums within a lane, and the terms G of the gradients are, as they
// stand, the other operand of the product with the turned streamed rows.  Nothing of the size of the logits is
// written.  The streamed side is cut into shares so that there are blocks for all CUs; shares leave partial sums that
// k_loss and k_finish add in order; a kept block whose streamed side is in one share is written as a result.
//
// Per tile and wave the matrix cores need 32 cycles a product, 3 (d / 16) + 6 (d / 32) of them for 32-bit values, the
// vector units 16 values of some 5 instructions and an exponential (and the split into two halves): at d = 100 the
// products bound it, at d = 40 the logits' exponentials do.  Measured, in 32 bits: the logits of 1,500 x 624,961 x 40 302 us
// (3.1 10^12 exponentials a second, 0.9 PFLOP/s of products), of 4,096 x 17,770 x 100 56 us; both gradients of the latter 225 us (1.2
// PFLOP/s of products executed, in 2 blocks a CU), of 1,024 x 10,681 x 40 25 us.  Within a wave a tile's exponentials follow its
// products; the matrix cores are busy 58% of the time, and the CU's other waves fill the rest in part.
#include "softmax_device.hpp"

namespace ccdops {

int small_steps(int d) {
    return (d + 15) / 16;
}

namespace {

template <class P, int NPL, int KS, bool TURNED>
struct Stream {
    static constexpr int DT = (KS + 1) / 2;
    static constexpr int kRows = NPL * KS;              // block of the rows' numbers
    static constexpr int kTurned = kRows + 1;           // first block of turned rows
    static constexpr int kCount = TURNED ? kTurned + NPL * DT * 2 : kTurned;
    static constexpr int kPer = (kCount + 3) / 4;       // fetches per wave and tile
    static constexpr int kStages = 3 * kCount <= 80 ? 3 : 2;
};

// out: [kStages][kCount] KB of LDS.  body(tile, slot) is called for each tile first .. last - 1 with the tile's data in slot.
template <class S, class F>
__device__ __forceinline__ void stream(const char* from, int64_t tile_bytes, int64_t first, int64_t last, char* lds, F&& body) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (first >= last) return;
    // Past the end the last tile is fetched again, and past the last block the last block: counts stay the same.
    const auto next = [&](int64_t i, int slot) {
        const char* src = from + min(i, last - 1) * tile_bytes + lane * 16;
        char* dst = lds + slot * (S::kCount * kBlk);
#pragma unroll
        for (int k = 0; k < S::kPer; ++k) {
            const int c = min(wave + 4 * k, S::kCount - 1);
            fetch(src + c * kBlk, dst + c * kBlk);
        }
    };
    for (int k = 0; k < S::kStages - 1; ++k) next(first + k, k);
    int slot = 0;
    for (int64_t i = first; i < last; ++i) {
        if constexpr (S::kStages == 3) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(S::kPer) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int free_slot = slot == 0 ? S::kStages - 1 : slot - 1;
        next(i + S::kStages - 1, free_slot);
        body(i, lds + slot * (S::kCount * kBlk));
        slot = slot + 1 == S::kStages ? 0 : slot + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // the next stream may take the slots
    asm volatile("" ::: "memory");
}

// Calls body(kept block, first tile, last tile, place among the kept block's shares) for the parts of a share.
template <class F>
__device__ __forceinline__ void each_part(const Shares& s, int64_t share, int64_t kept_blocks, F&& body) {
    const int64_t end = min((share + 1) * s.len, kept_blocks * s.tiles);
    for (int64_t u = share * s.len; u < end;) {
        const int64_t kb = u / s.tiles, first = u - kb * s.tiles, n = min(s.tiles - first, end - u);
        body(kb, first, first + n, share - s.first(kb));
        u += n;
    }
}

template <class P, int NPL, int KS>
struct Kept {
    typename P::vec f[NPL][KS];
    __device__ __forceinline__ void load(const char* bundle, int lane) {
#pragma unroll
        for (int p = 0; p < NPL; ++p)
#pragma unroll
            for (int k = 0; k < KS; ++k) f[p][k] = *(const typename P::vec*)(bundle + (p * KS + k) * kBlk + lane * 16);
    }
};

// Order of a run of N x (READS reads from LDS, PRODUCTS products): the reads AHEAD of the products they are for, the first
// HAD of them made before.
template <int N, int READS, int PRODUCTS, int AHEAD, int HAD>
__device__ __forceinline__ void interleave() {
    constexpr int A = AHEAD < N ? AHEAD : N;
    if constexpr (A > HAD) __builtin_amdgcn_sched_group_barrier(0x100, READS * (A - HAD), 0);
#pragma unroll
    for (int i = 0; i < N - A; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS * A, 0);
}

// 32 x 32 products of streamed rows (LDS) and kept rows, on top of acc: lane (n, h) gets kept row n, streamed rows
// 8 q + 4 h + r.
template <class P, int NPL, int KS>
__device__ __forceinline__ f32x16 tile_product(const char* slot, const Kept<P, NPL, KS>& kept, int lane, f32x16 acc) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        const typename P::vec a = *(const typename P::vec*)(slot + k * kBlk + lane * 16);
        acc = P::mfma(a, kept.f[0][k], acc);
        if constexpr (NPL == 2) {
            const typename P::vec b = *(const typename P::vec*)(slot + (KS + k) * kBlk + lane * 16);
            acc = P::mfma(a, kept.f[1][k], acc);
            acc = P::mfma(b, kept.f[0][k], acc);
        }
    }
    interleave<KS, NPL, NPL == 2 ? 3 : 1, NPL == 2 ? 2 : 4, 0>();
    __builtin_amdgcn_sched_barrier(0);
    return acc;
}

// The numbers `which` of this lane's 16 streamed rows.
__device__ __forceinline__ f32x16 row_numbers(const char* rows, int which, int h) {
    f32x16 o;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x4 v = *(const f32x4*)(rows + which * 128 + (8 * q + 4 * h) * 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[4 * q + r] = v[r];
    }
    return o;
}

// Sums of exponentials stay relative to `ref`, which the first tile with a finite logit sets; it is only moved when a tile's
// sum leaves what 32 bits hold well (above 2^40), so that an entry costs its exponential and its addition alone: the
// logits' accumulator starts at -ref.  Where the reference has to move, the tile's products are made again from 0: the
// first reference may be a finite mask's (-1e9), and what was added to that has lost its last digits.
constexpr float kSumLimit = 1099511627776.f;

// Logits from accumulated products of kept and streamed rows: `f` is x's number, `k` the table's exponent (kOwn).
__device__ __forceinline__ float own_logit(float acc, float f, int k, float add) { return __builtin_amdgcn_ldexpf(acc, __float_as_int(f) + k) + add; }

// WAY: the accumulated products are the logits (kUnit), have a factor for each row of x (kFactor), or exponents (kOwn).
template <class P, int NPL, int KS, int WAY>
__device__ __forceinline__ void small_lse(const SmallArgs& a, int64_t first, int64_t last, const Kept<P, NPL, KS>& kept, float f, char* lds,
                                          float& ref_out, float& sum_out) {
    typedef Stream<P, NPL, KS, false> S;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    float ref = 0.f, sum = 0.f;
    bool set = false;
    stream<S>(a.e, a.e_tile, first, last, lds, [&](int64_t i, const char* slot) {
        const bool offsets = a.offsets || i == a.vt - 1;  // the last tile's missing entries are -inf
        const auto logits = [&](float from) {
            f32x16 z;
#pragma unroll
            for (int r = 0; r < 16; ++r) z[r] = WAY == kUnit ? from : 0.f;
            if (WAY == kUnit && offsets) z += row_numbers(slot + S::kRows * kBlk, kNumOffset, h);
            z = tile_product<P, NPL, KS>(slot, kept, lane, z);
            if constexpr (WAY != kUnit) {
                const f32x16 k = WAY == kOwn ? row_numbers(slot + S::kRows * kBlk, kNumExp, h) : f32x16{};
#pragma unroll
                for (int r = 0; r < 16; ++r) z[r] = WAY == kOwn ? own_logit(z[r], f, __float_as_int(k[r]), from) : fmaf(z[r], f, from);
                if (offsets) z += row_numbers(slot + S::kRows * kBlk, kNumOffset, h);
            }
            return z;
        };
        f32x16 z = logits(-ref);
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) s += exp2_fast(z[r]);
        const bool moves = !set || s > kSumLimit;
        if (__any(moves)) {
            if (__any(set && moves)) z = logits(0.f);  // (relative to 0 as they are in lanes that have no reference yet)
            float m = set ? ref : -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) m = fmaxf(m, z[r]);
            if (moves && m != -INFINITY) {
                s = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) s += exp2_fast(z[r] - m);
                if (set) sum *= exp2_fast(ref - m);  // (0 before: the factor would be infinite for low logits)
                ref = m;
                set = true;
            }
        }
        sum += s;
    });
    ref_out = set ? ref : -INFINITY;
    sum_out = sum;
}

template <class P, int NPL, int KS>
__global__ __launch_bounds__(256, small_lse_per_cu(NPL, KS)) void k_small_lse(SmallArgs a) {
    typedef Stream<P, NPL, KS, false> S;
    __shared__ __align__(16) char lds[S::kStages * S::kCount * kBlk];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 31, h = lane >> 5;
    each_part(a.lse, blockIdx.x, (a.tt + 3) / 4, [&](int64_t kb, int64_t first, int64_t last, int64_t place) {
        const int64_t tile = min(kb * 4 + wave, a.tt - 1);
        const char* const mine = a.x + tile * a.x_tile;
        Kept<P, NPL, KS> kept;
        kept.load(mine, lane);
        const float f = *(const float*)(mine + S::kRows * kBlk + kNumFactor * 128 + n * 4);
        float top, sum;
        const int way = NPL == 2 ? a.fin[3] : kFactor;
        if (NPL == 2 && way == kUnit) small_lse<P, NPL, KS, kUnit>(a, first, last, kept, f, lds, top, sum);
        else if (NPL == 2 && way == kOwn) small_lse<P, NPL, KS, kOwn>(a, first, last, kept, f, lds, top, sum);
        else small_lse<P, NPL, KS, kFactor>(a, first, last, kept, f, lds, top, sum);
        const float top2 = __shfl_xor(top, 32), sum2 = __shfl_xor(sum, 32);
        const float m = fmaxf(top, top2), ref = m == -INFINITY ? 0.f : m;
        sum = sum * exp2_fast(top - ref) + sum2 * exp2_fast(top2 - ref);
        const int64_t t = (kb * 4 + wave) * 32 + n;
        if (h == 0 && t < a.t) a.part[place * a.t + t] = make_float2(m, sum);
    });
}

// Half-precision terms of an item whose largest one so far, in their common scale (at most 2^13), is below kTermLow or
// above kTermHigh get a power of two of their own that brings it to 2^kTermStart: an item that is unlikely for every row,
// or whose rows weigh little, keeps its digits (relative to its own largest term, two planes hold 2^-24 or better).
constexpr float kTermLow = 0.5f, kTermHigh = 32768.f, kTermLeast = 7.9e-31f;  // (2^-100)
constexpr int kTermStart = 7;

// One side's gradients for 128 kept rows: out += turned streamed rows x G.  ITEMS: the kept rows are the table's; returns the
// power of two that this lane's sums are yet to be multiplied with.
// The accumulator of the logits starts at what is added to them, so that a term costs its exponential alone.
template <class P, int NPL, int KS, bool ITEMS>
__device__ __forceinline__ int small_terms(const SmallArgs& a, int64_t tile, int64_t first, int64_t last, const Kept<P, NPL, KS>& kept, const float* own, char* lds,
                                            f32x16* out) {
    typedef Stream<P, NPL, KS, true> S;
    constexpr int DT = S::DT;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const float factor = own[kNumFactor * 32];                                     // x
    float base = ITEMS ? own[kNumOffset * 32] : own[kNumLse * 32] + kTermExp;  // what this row adds to its logits
    const int own_y = ITEMS ? 0 : __float_as_int(own[kNumTarget * 32]);
    constexpr bool MOVES = ITEMS && std::is_same<P, HF>::value;
    int ref = 0;       // MOVES: terms are taken times 2^-ref
    float most = 0.f;  // and the largest one so far
    const int way = NPL == 2 ? a.fin[3] : kFactor;
    const bool unit = way == kUnit;
    stream<S>(ITEMS ? a.xlive : a.e, ITEMS ? a.xlive_tile : a.e_tile, first, last, lds, [&](int64_t i, const char* slot) {
        const char* const rows = slot + S::kRows * kBlk;
        const int y = ITEMS ? ((const int*)rows)[kNumTarget * 32 + n] - (int)(tile * 32) : own_y - (int)(i * 32);
        const auto added = [&]() {
            f32x16 add;
            if constexpr (ITEMS) {
                add = row_numbers(rows, kNumTerm, h);
                if (__any(base != 0.f)) add += base;
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) add[r] = base;
                if (a.offsets || i == a.vt - 1) add += row_numbers(rows, kNumOffset, h);
            }
            return add;
        };
        f32x16 z = added();
        if (!unit) z = f32x16{};
        z = tile_product<P, NPL, KS>(slot, kept, lane, z);
        if (!unit) {
            const f32x16 add = added();
            if (NPL == 2 && way == kOwn) {
                const f32x16 k = row_numbers(rows, ITEMS ? kNumFactor : kNumExp, h);
                const float mine = ITEMS ? own[kNumExp * 32] : factor;
#pragma unroll
                for (int r = 0; r < 16; ++r) z[r] = own_logit(z[r], mine, __float_as_int(k[r]), add[r]);
            } else {
                const f32x16 f = ITEMS ? row_numbers(rows, kNumFactor, h) : f32x16{};
#pragma unroll
                for (int r = 0; r < 16; ++r) z[r] = fmaf(z[r], ITEMS ? f[r] : factor, add[r]);
            }
        }
        // The first turned fragments arrive while the terms are computed.
        constexpr int kAhead = NPL == 2 ? 2 : 4;
        typename P::vec tf[NPL][DT * 2];
        const auto turned = [&](int i) {
#pragma unroll
            for (int p = 0; p < NPL; ++p) tf[p][i] = *(const typename P::vec*)(slot + (S::kTurned + p * DT * 2 + i) * kBlk + lane * 16);
        };
#pragma unroll
        for (int i = 0; i < (kAhead < DT * 2 ? kAhead : DT * 2); ++i) turned(i);
        asm volatile("" ::: "memory");
        float g[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) g[r] = exp2_fast(z[r]);
        if constexpr (ITEMS) {
            if (__any(y >= 0 && y < 32)) {  // popular items: nearly every tile
                const f32x16 ys = row_numbers(rows, kNumTarget, h), ws = row_numbers(rows, kNumWeight, h);
                const float up = MOVES ? pow2i(-ref) : 1.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) g[r] = fmaf(__float_as_int(ys[r]) == (int)(tile * 32) + n ? ws[r] : 0.f, -up, g[r]);
            }
        } else {
            if (__any(y >= 0 && y < 32)) {
#pragma unroll
                for (int r = 0; r < 16; ++r) g[r] -= y == 8 * (r >> 2) + 4 * h + (r & 3) ? (float)(1 << kTermExp) : 0.f;
            }
        }
        if constexpr (MOVES) {
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(g[r]));
            // (none, and terms below 2^-113 of the largest weight, stay as they are)
            const auto moves = [&]() { return most > kTermHigh || (most < kTermLow && most > kTermLeast); };
            if (__any(moves())) {
                most = halves_max(most);
                const bool mine = moves() && finite(most);
                const int up = mine ? kTermStart - ((int)(__float_as_uint(most) >> 23) - 127) : 0;
                if (__any(mine)) {
                    const float f = pow2i(up);
                    ref -= up, base += (float)up, most *= f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) g[r] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d) out[d] *= f;
                }
            }
        }
        // Two planes of G for 16-bit types too: the products are not what bounds these, and one plane's rounding would
        // cost as much as that of the result.
        typename P::vec pl[2][2];
        split_terms<P, 2>(g, pl);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = kAhead; i < DT * 2; ++i) turned(i);
#pragma unroll
        for (int i = 0; i < DT * 2; ++i) {
            f32x16& o = out[i >> 1];
            o = P::mfma(tf[0][i], pl[0][i & 1], o);
            o = P::mfma(tf[0][i], pl[1][i & 1], o);
            if constexpr (NPL == 2) o = P::mfma(tf[1][i], pl[0][i & 1], o);
        }
        interleave<DT * 2, NPL, NPL + 1, kAhead, (kAhead < DT * 2 ? kAhead : DT * 2)>();
        __builtin_amdgcn_sched_barrier(0);
    });
    return ref;
}

// What the sums are multiplied with, one after the other: G's power of two is taken off, and the other operand's.
__device__ __forceinline__ float small_terms_factor(const SmallArgs& a, bool items) { return items ? (a.fin ? ldexpf(1.f, -a.fin[2]) : 1.f) : ldexpf(1.f, -kTermExp); }
__device__ __forceinline__ float small_factor(const SmallArgs& a, bool items) { return a.scaled ? ldexpf(a.scale, -a.fin[items ? 1 : 0]) : a.scale; }

template <class P, int NPL, int KS, bool ITEMS>
__device__ __forceinline__ void small_grad(const SmallArgs& a, int64_t share, char* lds) {
    typedef Stream<P, NPL, KS, true> S;
    constexpr int DT = S::DT;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 31, h = lane >> 5;
    const int64_t tiles = ITEMS ? a.vt : a.tt;
    each_part(ITEMS ? a.de : a.dx, share, (tiles + 3) / 4, [&](int64_t kb, int64_t first, int64_t last, int64_t place) {
        const int64_t at = kb * 4 + wave, tile = min(at, tiles - 1);
        const char* const mine = ITEMS ? a.e + tile * a.e_tile : a.xlive + tile * a.xlive_tile;
        Kept<P, NPL, KS> kept;
        kept.load(mine, lane);
        const float* const own = (const float*)(mine + S::kRows * kBlk) + n;
        f32x16 out[DT] = {};
        const int ref = small_terms<P, NPL, KS, ITEMS>(a, tile, first, last, kept, own, lds, out);
        if (at >= tiles) return;
        const float w = ITEMS ? pow2i(ref) : own[kNumRaw * 32];
        const SmallOut& o = ITEMS ? a.de_out : a.dx_out;
        if (first == 0 && last == (ITEMS ? a.de : a.dx).tiles) {  // nothing to add: the result itself
            typedef typename std::conditional<NPL == 2, float, typename P::elem>::type T;
            const int64_t row = tile * 32 + n;
            if (row >= (ITEMS ? a.v : a.t)) return;
            const float fg = small_terms_factor(a, ITEMS), f = small_factor(a, ITEMS);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    Run<T, 4> v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v.v[r] = (T)(out[d][q * 4 + r] * w * fg * f);
                    T* const at = (T*)o.to + row * o.ld + 4 * h;
                    if (d < DT - 1) store_run<4>(at + d * 32 + q * 8, v);  // columns that there are
                    else store_tail<4>(at, d * 32 + q * 8, a.d - 4 * h, v);
                }
            return;
        }
        float* const to = (ITEMS ? a.dep : a.dxp) + ((place * tiles + tile) * 32 + n) * (DT * 32) + 4 * h;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = out[d][q * 4 + r] * w;
                *(f32x4*)(to + d * 32 + q * 8) = v;
            }
    });
}

// Blocks for dx first, then blocks for de.
template <class P, int NPL, int KS>
__global__ __launch_bounds__(256, small_grads_per_cu(NPL, KS)) void k_small_grads(SmallArgs a) {
    typedef Stream<P, NPL, KS, true> S;
    __shared__ __align__(16) char lds[S::kStages * S::kCount * kBlk];
    if (blockIdx.x < a.dx.blocks) small_grad<P, NPL, KS, false>(a, blockIdx.x, lds);
    else small_grad<P, NPL, KS, true>(a, blockIdx.x - a.dx.blocks, lds);
}

}  // namespace

template <class P, int NPL>
hipError_t launch_small_lse(int ksd, const SmallArgs& a, hipStream_t st) {
    const unsigned blocks = (unsigned)a.lse.blocks;
    switch (ksd) {
        case 1: k_small_lse<P, NPL, 1><<<blocks, 256, 0, st>>>(a); break;
        case 2: k_small_lse<P, NPL, 2><<<blocks, 256, 0, st>>>(a); break;
        case 3: k_small_lse<P, NPL, 3><<<blocks, 256, 0, st>>>(a); break;
        case 4: k_small_lse<P, NPL, 4><<<blocks, 256, 0, st>>>(a); break;
        case 5: k_small_lse<P, NPL, 5><<<blocks, 256, 0, st>>>(a); break;
        case 6: k_small_lse<P, NPL, 6><<<blocks, 256, 0, st>>>(a); break;
        case 7: k_small_lse<P, NPL, 7><<<blocks, 256, 0, st>>>(a); break;
        default: k_small_lse<P, NPL, 8><<<blocks, 256, 0, st>>>(a); break;
    }
    return hipGetLastError();
}

template <class P, int NPL>
hipError_t launch_small_grads(int ksd, const SmallArgs& a, hipStream_t st) {
    const unsigned blocks = (unsigned)(a.dx.blocks + a.de.blocks);
    if (!blocks) return hipSuccess;
    switch (ksd) {
        case 1: k_small_grads<P, NPL, 1><<<blocks, 256, 0, st>>>(a); break;
        case 2: k_small_grads<P, NPL, 2><<<blocks, 256, 0, st>>>(a); break;
        case 3: k_small_grads<P, NPL, 3><<<blocks, 256, 0, st>>>(a); break;
        case 4: k_small_grads<P, NPL, 4><<<blocks, 256, 0, st>>>(a); break;
        case 5: k_small_grads<P, NPL, 5><<<blocks, 256, 0, st>>>(a); break;
        case 6: k_small_grads<P, NPL, 6><<<blocks, 256, 0, st>>>(a); break;
        case 7: k_small_grads<P, NPL, 7><<<blocks, 256, 0, st>>>(a); break;
        default: k_small_grads<P, NPL, 8><<<blocks, 256, 0, st>>>(a); break;
    }
    return hipGetLastError();
}

template hipError_t launch_small_lse<BF, 1>(int, const SmallArgs&, hipStream_t);
template hipError_t launch_small_lse<HF, 1>(int, const SmallArgs&, hipStream_t);
template hipError_t launch_small_lse<HF, 2>(int, const SmallArgs&, hipStream_t);
template hipError_t launch_small_grads<BF, 1>(int, const SmallArgs&, hipStream_t);
template hipError_t launch_small_grads<HF, 1>(int, const SmallArgs&, hipStream_t);
template hipError_t launch_small_grads<HF, 2>(int, const SmallArgs&, hipStream_t);

}  // namespace ccdops
