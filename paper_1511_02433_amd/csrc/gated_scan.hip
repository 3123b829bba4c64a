// Gated linear recurrences over packed sequences, their gradients, and one more row of each (gfx950).
//
//   h_t = a_t h_(t-1) + u_t;   GIVEN: a = gate, u = x;   SIGMOID: a = 1 / (1 + e^-gate), u = (1 - a) x
//   l_t = dy_t + a_(t+1) l_(t+1);   dx_t = l_t (times 1 - a_t),  dgate_t = l_t h_(t-1)  (or l_t (h_(t-1) - x_t) a_t (1 - a_t))
//
// Bound by memory where there is much: rows are read once and written once.  A row's state is A h + H of the state h before a chain of
// rows, whatever those rows are, so chains are joined: a thread takes W columns of a chunk of kRows rows into registers, the groups of a
// block, a chunk each, pass their (A, H) on through LDS, and a block goes on by `groups` chunks at a time down a share of the rows (up,
// for the gradients), with the next chunks' loads in flight.  Shares of a strip of columns are as many as blocks fill the device.  A
// sequence that goes on from one share to the next has its rows there read a second time, by a launch before, for their (A, H); so
// shares begin where a sequence does if one does nearby.  Lengths are known to the device alone: every rule here holds for any of them.
//
// 32,768 x 4,096 bfloat16 in 16 sequences: 457 us both ways one after the other; the forward call alone, again and again, 193 (872 MB with the
// kept states, 4.5 TB/s), that of the gradients 289 (1,409 MB, 4.9), of a copy's 5.13; vector instructions are issued in 75% and 60% of the
// cycles (a value takes some 30 forward, 40 back).  1,000,209 x 40 floats in 6,041 sequences 108 + 22 us (22: the launch before); one sequence of
// 65,537 x 100 bfloat16 18.5 + 7.5, which is what the rounds to memory of a block take one after another.
// Times at the choices below are of calls, again and again, in one run that had both sides in turn (histories: the 1,000,209 x 40 floats).
#include <algorithm>
#include <type_traits>

#include "ccdpp_seq.h"
#include "seq_device.hpp"

namespace ccdops {
namespace {

// kRows: of a chunk, of which one state is kept for the gradients (half a byte a value).  With 16 the gradients' registers leave fewer waves:
// 312 us in place of 289 for 32,768 x 4,096 bfloat16; the histories take 143 in place of 134, 10,007 x 777 half precision, both ways, 110 in
// place of 78.
// kThreads: with 256 a block has half the chunks side by side and twice the steps: 10,007 x 777 half precision 86 us in place of 78, the histories
// 138 in place of 134, 32,768 x 4,096 both ways 547 in place of 454; one long sequence takes the same.
constexpr int kRows = 8;
constexpr int kThreads = 512;  // of a block
constexpr int kLanes = 64;     // of a group, at most

// Both a and 1 - a to some 2^-21 of themselves, for gates of either sign: e = exp(-|gate|), with what the product by log2 e rounded off put
// back.  (e is 0 to 32 bits where -104 takes the place of less, and a product of infinities would be NaN; a gate that is NaN stays it.)
struct Gate { float a, rest; };
__device__ __forceinline__ Gate sigmoid_of(float gate) {
    const float z = __builtin_elementwise_maximum(-fabsf(gate), -104.f), p = z * 1.44269504f;
    const float off = fmaf(-p, -1.90465430e-9f, fmaf(-p, 0.693147182f, z));  // z - p ln 2
    float e = __builtin_amdgcn_exp2f(p);
    e = fmaf(e, off, e);
    const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
    const bool up = gate >= 0.f;
    return {up ? big : small, up ? small : big};
}

struct Terms { float a, u, rest; };
template <bool SIGMOID>
__device__ __forceinline__ Terms terms_of(float x, float gate) {
    if constexpr (!SIGMOID) return {gate, x, 1.f};
    const Gate g = sigmoid_of(gate);
    return {g.a, g.rest * x, g.rest};
}

// W values of a row as they lie in memory, in one access that is aligned to their type alone.  Two of 16 bits stay one word until
// they are used: of an array of them the compiler makes a register each.
template <class T, int W>
struct Few {
    static_assert(W == 1 || sizeof(T) == 4, "");
    Run<T, W> r;
    __device__ __forceinline__ void load(const T* at) {
        if constexpr (W == 1) r.v[0] = *at;
        else r = load_run<W>(at);
    }
    __device__ __forceinline__ void store(T* at) const {
        if constexpr (W == 1) *at = r.v[0];
        else store_run<W>(at, r);
    }
    __device__ __forceinline__ float get(int w) const { return (float)r.v[w]; }
    // The same, but unknown to the compiler: what it computes of it here is not computed before a branch for both its sides.
    __device__ __forceinline__ Few again() const {
        Few f = *this;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int w = 0; w < W; ++w) asm("" : "+v"(f.r.v[w]));
        } else {
            uint32_t word = __builtin_bit_cast(uint16_t, f.r.v[0]);
            asm("" : "+v"(word));
            f.r.v[0] = __builtin_bit_cast(T, (uint16_t)word);
        }
        return f;
    }
    __device__ __forceinline__ void set(const float (&v)[W]) {
#pragma unroll
        for (int w = 0; w < W; ++w) r.v[w] = (T)v[w];
    }
};
template <class T>
struct Pair {
    typedef T two __attribute__((ext_vector_type(2)));
    typedef uint32_t loose __attribute__((aligned(2), may_alias));
    uint32_t word;
    __device__ __forceinline__ void load(const T* at) { word = *(const loose*)at; }
    __device__ __forceinline__ void store(T* at) const { *(loose*)at = word; }
    __device__ __forceinline__ float get(int w) const {
        if constexpr (std::is_same<T, __bf16>::value) return __uint_as_float(w ? word & 0xFFFF0000u : word << 16);
        else return (float)__builtin_bit_cast(two, word)[w];
    }
    __device__ __forceinline__ Pair again() const {
        Pair f = *this;
        asm("" : "+v"(f.word));
        return f;
    }
    __device__ __forceinline__ void set(const float (&v)[2]) { word = __builtin_bit_cast(uint32_t, (two){(T)v[0], (T)v[1]}); }
};
template <> struct Few<__bf16, 2> : Pair<__bf16> {};
template <> struct Few<_Float16, 2> : Pair<_Float16> {};

// Where a share of rows begins.  q >= 0: within sequence q, which has rows prev to next - 1; else where a sequence begins, or in no
// sequence at all.  The rows of all sequences lie in [start0, start_s), which the table of shares has beside each, so that a block has them with
// its share's begin.
struct Share {
    int64_t begin, prev, next;
    int64_t q;
    int64_t start0, start_s;
};
// kRows rows of a chunk: the sequence of the first one (-1 or s: none), and a bit for each row that begins a sequence (or the rows
// behind all), bit kRows for the row after the chunk.  kSkips: sequences without rows begin in it, too; of_row says which begin there.
constexpr uint32_t kSkips = 1u << 31;
struct Chunk {
    int32_t q;
    uint32_t begins;
};

struct Scan {
    int64_t n, s, ldx, ldg, ldy, lddx, lddg;
    int d, bits;
    const void *x, *gate, *starts;
    const float *initial, *dlast, *kept;
    void *y, *dx, *dgate;  // y: the states, or dy
    float *last, *keep, *dinitial;
    // How the work is shared out.
    int strips, lanes, groups, shares;  // a block has `groups` groups of `lanes` lanes
    int64_t rows, near;                 // of a share, before it is moved to where a sequence begins, and how far it is moved at most
    int64_t chunks;
    Share* share;      // shares + 1
    Chunk* chunk;      // chunks
    int32_t* of_row;   // the sequence that begins at a row, for such rows alone
    float* carry;      // A and H of each share and column
    int sums, tables, marks;  // blocks of each kind in the first launch
};

__device__ __forceinline__ int64_t start_of(const Scan& a, int64_t q) {
    const int64_t v = a.bits == 64 ? ((const int64_t*)a.starts)[q] : ((const int32_t*)a.starts)[q];
    return min(max(v, (int64_t)0), a.n);
}

// The first of the s + 1 starts that is at least `row`, by a wave: 64 probes at a time.
__device__ int64_t find_start(const Scan& a, int64_t row) {
    int64_t lo = 0, hi = a.s + 1;
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, at = lo + (threadIdx.x & 63) * step;
        const int below = __popcll(__ballot(at < hi && start_of(a, min(at, a.s)) < row));
        const int64_t from = lo;
        if (below) lo = from + (below - 1) * step + 1;
        if (below < 64) hi = min(hi, from + below * step);
    }
    return lo;
}

// Share p begins at row p * rows, or where a sequence does if that is near: within 3 / 16 of a share.  (Blocks wait for the longest share, so
// shares of unlike lengths cost more than rows read twice: with 3 / 8, 65,000 x 1,000 bfloat16 in 64 sequences by a power law 173 us in
// place of 155, 32,768 x 4,096 in 16 such sequences both ways 640 in place of 613.  With 1 / 8 157 and 613, and the histories 130 in place of 134.)
__device__ Share share_of(const Scan& a, int64_t p) {
    if (p <= 0) return {0, 0, 0, -1};
    if (p >= a.shares) return {a.n, 0, 0, -1};
    const int64_t row = p * a.rows, j = find_start(a, row);
    const int64_t next = j <= a.s ? start_of(a, j) : a.n, prev = j > 0 ? start_of(a, j - 1) : 0;
    if (next >= row && next - row <= a.near) return {next, 0, 0, -1};
    if (j > 0 && prev <= row && row - prev <= a.near) return {prev, 0, 0, -1};
    if (j == 0 || j > a.s || prev > row || next < row) return {row, 0, 0, -1};
    return {row, prev, next, j - 1};
}

// What a chain of rows does to the state before it: A state + H; where a sequence begins in it the state behind it is H, whatever
// was before (A is kReset then, a bit pattern that no product has: products have no signalling NaN).
constexpr uint32_t kReset = 0x7F800001u;

// A thread's place: `lanes` lanes side by side take the columns of a strip, W each, and `groups` of them a chunk each, one after
// another.  The last lanes of a row take its last W columns, if need be with another lane, which gets the same.
template <int W>
struct Place {
    int lane, group, col;
    bool works;
    __device__ Place(const Scan& a, int strip) {
        group = threadIdx.x / a.lanes, lane = threadIdx.x - group * a.lanes;
        works = group < a.groups;
        col = min((strip * a.lanes + lane) * W, a.d - W);
    }
};

template <int W>
struct Exchange {
    struct alignas(8 * W) Link {
        float A[W], H[W];
    };
    Link of[2][kThreads];
    float behind[2][kLanes][W];  // the state behind the last group's rows
};

// The state before this group's rows, from the chains of the groups before it and the state before all: `first` at the first step,
// then what the last group left (leave).  One barrier a step; steps alternate between two buffers.
template <int W>
__device__ __forceinline__ void join(Exchange<W>& e, const Scan& a, const Place<W>& at, int step, const float (&A)[W], const float (&H)[W], bool reset,
                                     const float (&first)[W], float (&c)[W]) {
    typename Exchange<W>::Link* const of = e.of[step & 1];
    typename Exchange<W>::Link own;
#pragma unroll
    for (int w = 0; w < W; ++w) own.A[w] = reset ? __uint_as_float(kReset) : A[w], own.H[w] = H[w];
    of[threadIdx.x] = own;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) c[w] = step ? e.behind[step & 1][at.lane][w] : first[w];
    const int before = at.works ? at.group : 0;
#pragma unroll 4
    for (int g = 0; g < before; ++g) {
        const typename Exchange<W>::Link one = of[g * a.lanes + at.lane];
        const bool begins = __float_as_uint(one.A[0]) == kReset;
#pragma unroll
        for (int w = 0; w < W; ++w) c[w] = begins ? one.H[w] : fmaf(one.A[w], c[w], one.H[w]);
    }
}
template <int W>
__device__ __forceinline__ void leave(Exchange<W>& e, const Scan& a, const Place<W>& at, int step, const float (&h)[W]) {
    if (at.group == a.groups - 1)
#pragma unroll
        for (int w = 0; w < W; ++w) e.behind[(step + 1) & 1][at.lane][w] = h[w];
}

// The same over all groups: c goes in as the state before them and out as that behind; `all` takes the product of their A.
template <int W>
__device__ __forceinline__ void join_all(const Scan& a, Exchange<W>& e, const Place<W>& at, int step, const float (&A)[W], const float (&H)[W], bool reset,
                                         float (&c)[W], float (&all)[W]) {
    typename Exchange<W>::Link* const of = e.of[step & 1];
    typename Exchange<W>::Link own;
#pragma unroll
    for (int w = 0; w < W; ++w) own.A[w] = reset ? __uint_as_float(kReset) : A[w], own.H[w] = H[w];
    of[threadIdx.x] = own;
    __syncthreads();
#pragma unroll 4
    for (int g = 0; g < a.groups; ++g) {
        const typename Exchange<W>::Link one = of[g * a.lanes + at.lane];
        const bool begins = __float_as_uint(one.A[0]) == kReset;
#pragma unroll
        for (int w = 0; w < W; ++w) c[w] = begins ? one.H[w] : fmaf(one.A[w], c[w], one.H[w]), all[w] *= one.A[w];
    }
}

// The address of the next row from that of this one: eight multiples of every stride at once would not stay in registers.
template <class T>
__device__ __forceinline__ void next(T*& at, int64_t ld) {
    at += ld;
    asm("" : "+v"(at));
}

template <class T, int W>
struct Rows {
    Few<T, W> v[kRows];
    // Those of a chunk that lie in [lo, hi): no other row is read.
    __device__ __forceinline__ void load(const void* base, int64_t ld, int64_t row, int64_t lo, int64_t hi, int col) {
        const T* at = (const T*)base + row * ld + col;
        if (row >= lo && row + kRows <= hi) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) v[i].load(at), next(at, ld);
        } else {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                if (row + i >= lo && row + i < hi) v[i].load(at);
                next(at, ld);
            }
        }
    }
};

// The sequence of row i of a chunk.
__device__ __forceinline__ int64_t sequence_of(const Scan& a, Chunk k, int64_t row, int i) {
    const uint32_t up_to = k.begins & ((2u << i) - 1) & ~1u;
    if (!(k.begins & kSkips) || !up_to) return k.q + __popc(up_to);
    return a.of_row[row + 31 - __builtin_clz(up_to)];
}

// A row of the s x d states of sequences; NULL for what is no sequence.
template <class P>
__device__ __forceinline__ P* states_of(const Scan& a, P* base, int64_t q, int col) {
    return base && (uint64_t)q < (uint64_t)a.s ? base + q * a.d + col : nullptr;
}

// The rows of a chunk within [lo, hi), as bits.
__device__ __forceinline__ uint32_t rows_within(int64_t row, int64_t lo, int64_t hi) {
    const int from = (int)min(max(lo - row, (int64_t)0), (int64_t)kRows), to = (int)min(max(hi - row, (int64_t)0), (int64_t)kRows);
    return to > from ? ((1u << to) - 1) & ~((1u << from) - 1) : 0u;
}

constexpr uint32_t kAll = (1u << kRows) - 1;

// The first launch: what the rows of a sequence that goes on behind a share do to the state before them (for the gradients: of one that
// began before it), for every share and strip; the shares; the chunks; and the states of sequences without rows.
template <class T, int W, bool SIGMOID, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_scan_first(Scan a) {
    __shared__ Exchange<W> e;
    __shared__ Share two[2];
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    int block = blockIdx.x;
    if (block < a.sums) {
        const int strip = block % a.strips, p = block / a.strips + (GRAD ? 1 : 0);
        if (wave < 2) {
            const Share s = share_of(a, p + wave);
            if ((threadIdx.x & 63) == 0) two[wave] = s;
        }
        __syncthreads();
        const Share at_begin = two[0], at_end = two[1];
        const Share& edge = GRAD ? at_begin : at_end;
        if (edge.q < 0) return;
        const int64_t lo = GRAD ? at_begin.begin : max(at_begin.begin, edge.prev), hi = GRAD ? min(at_end.begin, edge.next) : at_end.begin;
        const Place<W> at(a, strip);
        // A group takes `per` chunks one after another, so that the groups join once.
        const int64_t c0 = lo / kRows, c1 = (hi + kRows - 1) / kRows, per = (c1 - c0 + a.groups - 1) / a.groups;
        const int64_t from = at.group * per, to = at.works ? min(from + per, c1 - c0) : 0;
        Rows<T, W> x, gate;  // x: dy for the gradients
        const auto chunk_of = [&](int64_t i) { return GRAD ? c1 - 1 - i : c0 + i; };
        const auto load = [&](int64_t i) {
            if (i >= to) return;
            gate.load(a.gate, a.ldg, chunk_of(i) * kRows, lo, hi, at.col);
            if (GRAD) x.load(a.y, a.ldy, chunk_of(i) * kRows, lo, hi, at.col);
            else x.load(a.x, a.ldx, chunk_of(i) * kRows, lo, hi, at.col);
        };
        load(from);
        float first[W], A[W], H[W], C[W], all[W];  // first: the state before a sequence's first row, or behind its last one
        const bool ends = GRAD ? edge.next <= at_end.begin : edge.prev >= at_begin.begin;
        const float* states = GRAD ? a.dlast : a.initial;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            first[w] = ends && states ? states[edge.q * a.d + at.col + w] : 0.f;
            A[w] = all[w] = 1.f, H[w] = C[w] = 0.f;
        }
        for (int64_t i = from; i < to; ++i) {
            const int64_t row = chunk_of(i) * kRows;
            const uint32_t in = rows_within(row, lo, hi);
            float d[kRows][W], u[kRows][W];
#pragma unroll
            for (int k = 0; k < kRows; ++k)
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const Terms m = terms_of<SIGMOID && !GRAD>(x.v[k].get(w), gate.v[k].get(w));
                    d[k][w] = GRAD && SIGMOID ? sigmoid_of(gate.v[k].get(w)).a : m.a, u[k][w] = m.u;
                }
            load(i + 1);
            if (in != kAll) {
#pragma unroll
                for (int k = 0; k < kRows; ++k)
#pragma unroll
                    for (int w = 0; w < W; ++w)
                        if (!(in >> k & 1)) d[k][w] = 1.f, u[k][w] = 0.f;
            }
            // (The state that comes in at lo, or at hi - 1, is put in before the chunk: the chunk's rows before it are none.)
            if (GRAD ? hi - 1 - row < kRows && hi > row : lo >= row)
#pragma unroll
                for (int w = 0; w < W; ++w) H[w] = first[w];
#pragma unroll
            for (int k = 0; k < kRows; ++k)
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const int r = GRAD ? kRows - 1 - k : k;
                    A[w] *= d[r][w];
                    H[w] = GRAD ? d[r][w] * (u[r][w] + H[w]) : fmaf(d[r][w], H[w], u[r][w]);
                }
        }
        join_all<W>(a, e, at, 0, A, H, false, C, all);
        if (at.group == 0) {
            float* out = a.carry + ((int64_t)p * a.d + at.col) * 2;
#pragma unroll
            for (int w = 0; w < W; ++w) out[2 * w] = all[w], out[2 * w + 1] = C[w];
        }
        return;
    }
    block -= a.sums;
    if (block < a.tables) {
        // The first start from `row` on, in [lo, hi].
        const auto find = [&](int64_t row, int64_t lo, int64_t hi) {
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (start_of(a, mid) < row) lo = mid + 1;
                else hi = mid;
            }
            return lo;
        };
        // A wave looks for its first chunk's row together, and each lane for its own among the next 64 starts, where they go that far.
        const int64_t c = block * (int64_t)blockDim.x + threadIdx.x, row = c * kRows, row0 = (c - (threadIdx.x & 63)) * kRows;
        const int64_t j0 = find_start(a, row0), near = min(j0 + 64, a.s + 1);
        if (c >= a.chunks) return;
        int64_t j = find(row, j0, near > a.s || start_of(a, near) >= row0 + 64 * kRows ? near : a.s + 1), r = -1;
        Chunk k = {(int32_t)(j - 1), 0u};
        int64_t q = j - 1;  // the last sequence so far
        while (j <= a.s) {
            const int64_t begin = start_of(a, j);
            if (begin < row || begin > row + kRows || begin <= r) break;
            r = begin;
            const bool more = j < a.s && start_of(a, j + 1) == r;  // sequences without rows begin there, too
            j = more ? find(r + 1, j + 1, a.s + 1) : j + 1;
            k.begins |= 1u << (r - row);
            if (r == row) k.q = (int32_t)(j - 1), q = j - 1;
            else if (j - 1 != ++q) k.begins |= kSkips, q = j - 1;
            if (r < row + kRows && r < a.n) a.of_row[r] = (int32_t)(j - 1);
        }
        a.chunk[c] = k;
        return;
    }
    block -= a.tables;
    if (block < a.marks) {
        const int p = block * waves + wave;
        if (p > a.shares) return;
        Share s = share_of(a, p);
        s.start0 = a.s ? start_of(a, 0) : a.n, s.start_s = start_of(a, a.s);
        if ((threadIdx.x & 63) == 0) a.share[p] = s;
        return;
    }
    block -= a.marks;
    float* const out = GRAD ? a.dinitial : a.last;
    const float* const from = GRAD ? a.dlast : a.initial;
    const int64_t q0 = ((int64_t)block * waves + wave) * 64, mine = q0 + (threadIdx.x & 63);
    uint64_t none = __ballot(mine < a.s && start_of(a, min(mine, a.s)) >= start_of(a, min(mine + 1, a.s)));
    while (none) {
        const int64_t q = q0 + __ffsll((unsigned long long)none) - 1;
        none &= none - 1;
        for (int c = threadIdx.x & 63; c < a.d; c += 64) out[q * a.d + c] = from ? from[q * a.d + c] : 0.f;
    }
}

// The state that comes into a share from those before it (for the gradients: after it): the groups take a part of the shares each, and
// join what they have.
template <int W, bool GRAD>
__device__ void carry_in(const Scan& a, Exchange<W>& e, const Place<W>& at, int p, const Share& edge, float (&c)[W]) {
#pragma unroll
    for (int w = 0; w < W; ++w) c[w] = 0.f;
    if (edge.q < 0) return;
    // The share in which the sequence begins (ends); there, nothing comes in.
    // (Share i begins at i * rows or where the sequence does if that is near, as share_of has it.)
    const int64_t i = (GRAD ? edge.next - 1 : edge.prev) / a.rows;
    int far;
    if (GRAD) far = (int)min(max(edge.next - i * a.rows <= a.near ? i - 1 : i, (int64_t)p + 1), (int64_t)a.shares - 1);
    else far = (int)min(max((i + 1) * a.rows - edge.prev <= a.near ? i + 1 : i, (int64_t)0), (int64_t)p - 1);
    const int count = GRAD ? far - p : p - far, per = (count + a.groups - 1) / a.groups;
    const int from = min(at.group * per, count), to = min(from + per, count);
    float A[W], H[W];
#pragma unroll
    for (int w = 0; w < W; ++w) A[w] = 1.f, H[w] = 0.f;
    if (at.works) {
        constexpr int kAtOnce = 16;  // that are read together
        for (int i0 = from; i0 < to; i0 += kAtOnce) {
            float f[kAtOnce][W], g[kAtOnce][W];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int i = min(i0 + u, to - 1);
                const float* k = a.carry + ((int64_t)(GRAD ? far - i : far + i) * a.d + at.col) * 2;
#pragma unroll
                for (int w = 0; w < W; ++w) f[u][w] = k[2 * w], g[u][w] = k[2 * w + 1];
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if (i0 + u >= to) continue;
                    if (i0 + u == 0) H[w] = g[u][w];
                    else H[w] = fmaf(f[u][w], H[w], g[u][w]), A[w] *= f[u][w];
                }
        }
    }
    float all[W] = {};
    join_all<W>(a, e, at, 0, A, H, at.works && from == 0 && to > 0, c, all);
    __syncthreads();
}

// A chunk whose rows are all of one sequence, and neither its first nor its last, can take the plain way; the other does each row by what it
// is.  A wave takes one of them for all its chunks: both would take the time of both.
__device__ __forceinline__ bool all_plain(bool here, uint32_t in, uint32_t ends) { return !__ballot(here && (in != kAll || ends)); }

// The chunks of a share, and those of them that have rows of sequences ([lo, hi)): only these are read and stepped through.
// (65,536 x 4,096 bfloat16 of which 8 rows are in sequences: 163 us forward and 207 for the gradients, mostly zeros; stepped through like others they
// take 504 and 723, more than rows of sequences do, which take 322 and 568.)
struct Range {
    int64_t c0, c1, all0, all1;
    __device__ Range(int64_t begin, int64_t end, int64_t lo, int64_t hi) {
        all0 = begin / kRows, all1 = (end + kRows - 1) / kRows;
        c0 = lo < hi ? lo / kRows : all1, c1 = lo < hi ? (hi + kRows - 1) / kRows : all1;
    }
    // body(chunk) for the others, a group each.
    template <int W, class F>
    __device__ __forceinline__ void others(const Scan& a, const Place<W>& at, F&& body) const {
        if (!at.works) return;
        for (int64_t c = all0 + at.group; c < c0; c += a.groups) body(c);
        for (int64_t c = c1 + at.group; c < all1; c += a.groups) body(c);
    }
};
template <class T, int W>
__device__ __forceinline__ void clear_rows(void* base, int64_t ld, int64_t row, uint32_t which, int col) {
    const float zero[W] = {};
    Few<T, W> r;
    r.set(zero);
    T* at = (T*)base + row * ld + col;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (which >> i & 1) r.store(at);
        next(at, ld);
    }
}

template <class T, int W, bool SIGMOID>
__global__ __launch_bounds__(kThreads) void k_scan(Scan a) {
    __shared__ Exchange<W> e;
    const int strip = blockIdx.x % a.strips, p = blockIdx.x / a.strips;
    const Place<W> at(a, strip);
    const Share share = a.share[p];
    const int64_t begin = share.begin, end = a.share[p + 1].begin;
    const int64_t lo = max(share.start0, begin), hi = min(share.start_s, end);  // rows of sequences
    const Range range(begin, end, lo, hi);
    const int64_t c0 = range.c0, c1 = range.c1, steps = (c1 - c0 + a.groups - 1) / a.groups;
    Rows<T, W> x, gate;
    Chunk k;
    const auto load = [&](int64_t step) {
        const int64_t c = c0 + step * a.groups + at.group;
        if (!at.works || c >= c1) return;
        k = a.chunk[c];
        x.load(a.x, a.ldx, c * kRows, share.start0, share.start_s, at.col);
        gate.load(a.gate, a.ldg, c * kRows, share.start0, share.start_s, at.col);
    };
    load(0);
    float carry[W];
    carry_in<W, false>(a, e, at, p, share, carry);
    for (int64_t step = 0; step < steps; ++step) {
        const int64_t c = c0 + step * a.groups + at.group, row = c * kRows;
        const bool here = at.works && c < c1;
        const uint32_t mine = here ? rows_within(row, begin, end) : 0u, in = here ? rows_within(row, lo, hi) : 0u;
        const uint32_t firsts = here ? k.begins & mine : 0u, lasts = here ? k.begins >> 1 & in : 0u;
        const bool plain = here && all_plain(here, in, firsts | lasts), other = here && !plain;
        const Chunk now = k;
        float d[kRows][W], u[kRows][W];
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const Terms m = terms_of<SIGMOID>(x.v[i].get(w), gate.v[i].get(w));
                d[i][w] = m.a, u[i][w] = m.u;
            }
        load(step + 1);
        float A[W], H[W], h[W];
#pragma unroll
        for (int w = 0; w < W; ++w) A[w] = 1.f, H[w] = 0.f;
        if (plain) {
#pragma unroll
            for (int i = 0; i < kRows; ++i)
#pragma unroll
                for (int w = 0; w < W; ++w) A[w] *= d[i][w], H[w] = fmaf(d[i][w], H[w], u[i][w]);
        } else if (other) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const bool inside = in >> i & 1, first = firsts >> i & 1;
                const float* from = nullptr;
                if (first && inside && a.initial) from = states_of(a, a.initial, sequence_of(a, now, row, i), at.col);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if (!inside) d[i][w] = 1.f, u[i][w] = 0.f;
                    if (from) u[i][w] = fmaf(d[i][w], from[w], u[i][w]);
                    A[w] *= d[i][w], H[w] = first ? u[i][w] : fmaf(d[i][w], H[w], u[i][w]);
                }
            }
        }
        join<W>(e, a, at, (int)step, A, H, firsts != 0, carry, h);
        if (a.keep && (mine & 1)) {
            Few<float, W> r;
            r.set(h);
            r.store(a.keep + c * a.d + at.col);
        }
        T* y = (T*)a.y + row * a.ldy + at.col;
        if (plain) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
#pragma unroll
                for (int w = 0; w < W; ++w) h[w] = fmaf(d[i][w], h[w], u[i][w]);
                Few<T, W> r;
                r.set(h);
                r.store(y);
                next(y, a.ldy);
            }
        } else if (other) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const bool inside = in >> i & 1, first = firsts >> i & 1;
                float out[W];
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    h[w] = first ? u[i][w] : fmaf(d[i][w], h[w], u[i][w]);
                    out[w] = inside ? h[w] : 0.f;
                }
                Few<T, W> r;
                r.set(out);
                if (mine >> i & 1) r.store(y);
                next(y, a.ldy);
                if (float* const to = (lasts >> i & 1) && a.last ? states_of(a, a.last, sequence_of(a, now, row, i), at.col) : nullptr)
#pragma unroll
                    for (int w = 0; w < W; ++w) to[w] = h[w];
            }
        }
        leave<W>(e, a, at, (int)step, h);
    }
    range.others<W>(a, at, [&](int64_t c) {
        const uint32_t mine = rows_within(c * kRows, begin, end);
        clear_rows<T, W>(a.y, a.ldy, c * kRows, mine, at.col);
        if (a.keep && (mine & 1)) clear_rows<float, W>(a.keep, a.d, c, 1, at.col);
    });
}

// Up the rows.  Each chunk's states are computed once more from the one that was kept, which gives what l is multiplied by for dgate; then
// l goes through it as the state does forward, from the last row to the first.
template <class T, int W, bool SIGMOID>
__global__ __launch_bounds__(kThreads) void k_scan_grad(Scan a) {
    __shared__ Exchange<W> e;
    const int strip = blockIdx.x % a.strips, p = blockIdx.x / a.strips;
    const Place<W> at(a, strip);
    const Share share = a.share[p + 1];
    const int64_t begin = a.share[p].begin, end = share.begin;
    const int64_t lo = max(share.start0, begin), hi = min(share.start_s, end);
    const Range range(begin, end, lo, hi);
    const int64_t c0 = range.c0, c1 = range.c1, steps = (c1 - c0 + a.groups - 1) / a.groups;
    Rows<T, W> x, gate, dy;
    Few<float, W> h0;
    Chunk k;
    const auto load = [&](int64_t step) {
        const int64_t c = c1 - 1 - step * a.groups - at.group;
        if (!at.works || c < c0) return;
        k = a.chunk[c];
        h0.load(a.kept + c * a.d + at.col);
        x.load(a.x, a.ldx, c * kRows, share.start0, share.start_s, at.col);
        gate.load(a.gate, a.ldg, c * kRows, share.start0, share.start_s, at.col);
        dy.load(a.y, a.ldy, c * kRows, share.start0, share.start_s, at.col);
    };
    load(0);
    float carry[W];
    carry_in<W, true>(a, e, at, p, share, carry);
    for (int64_t step = 0; step < steps; ++step) {
        const int64_t c = c1 - 1 - step * a.groups - at.group, row = c * kRows;
        const bool here = at.works && c >= c0;
        const uint32_t mine = here ? rows_within(row, begin, end) : 0u, in = here ? rows_within(row, lo, hi) : 0u;
        const uint32_t firsts = here ? k.begins & in : 0u, lasts = here ? k.begins >> 1 & in : 0u;
        const bool plain = here && all_plain(here, in, firsts | lasts), other = here && !plain;
        const Chunk now = k;
        // Kept in registers from the pass down the rows for the two up: a, 1 - a, what l is multiplied by for dgate, and dy as it is.
        float d[kRows][W], rest[kRows][W], f[kRows][W];
        const Rows<T, W> g = dy;
        // One row down: its f, and the state behind it.
        const auto down = [&](int i, int w, const auto& x, const auto& gate, float& h) {
            const float v = x.get(w), z = gate.get(w);
            const Terms m = terms_of<SIGMOID>(v, z);
            d[i][w] = m.a, rest[i][w] = m.rest;
            f[i][w] = SIGMOID ? (h - v) * (m.a * m.rest) : h;
            h = fmaf(m.a, h, m.u);
        };
        float h[W], A[W], H[W], m[W];
#pragma unroll
        for (int w = 0; w < W; ++w) h[w] = h0.get(w), A[w] = 1.f, H[w] = 0.f;
        if (plain) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
#pragma unroll
                for (int w = 0; w < W; ++w) down(i, w, x.v[i], gate.v[i], h[w]);
            }
        } else if (other) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                if (firsts >> i & 1) {
                    const float* from = a.initial ? states_of(a, a.initial, sequence_of(a, now, row, i), at.col) : nullptr;
#pragma unroll
                    for (int w = 0; w < W; ++w) h[w] = from ? from[w] : 0.f;
                }
                const auto xi = x.v[i].again(), zi = gate.v[i].again();
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    float to = h[w];
                    down(i, w, xi, zi, to);
                    h[w] = in >> i & 1 ? to : h[w];
                }
            }
        }
        load(step + 1);
        if (plain) {
#pragma unroll
            for (int i = kRows - 1; i >= 0; --i)
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    A[w] *= d[i][w], H[w] = d[i][w] * (g.v[i].get(w) + H[w]);
                }
        } else if (other) {
#pragma unroll
            for (int i = kRows - 1; i >= 0; --i) {
                if (lasts >> i & 1) {
                    const float* from = states_of(a, a.dlast, a.dlast ? sequence_of(a, now, row, i) : 0, at.col);
#pragma unroll
                    for (int w = 0; w < W; ++w) H[w] = from ? from[w] : 0.f;
                }
                const auto gi = g.v[i].again();
#pragma unroll
                for (int w = 0; w < W; ++w)
                    if (in >> i & 1) A[w] *= d[i][w], H[w] = d[i][w] * (gi.get(w) + H[w]);
            }
        }
        join<W>(e, a, at, (int)step, A, H, lasts != 0, carry, m);
        T* dx = (T*)a.dx + (row + kRows - 1) * a.lddx + at.col;
        T* dg = (T*)a.dgate + (row + kRows - 1) * a.lddg + at.col;
        // One row up: its gradients, and what goes on to the row before it.
        const auto up = [&](int i, int w, const auto& g, float& m, float& to_x, float& to_gate) {
            const float l = g.get(w) + m;
            to_x = SIGMOID ? rest[i][w] * l : l, to_gate = l * f[i][w];
            m = d[i][w] * l;
        };
        if (plain) {
#pragma unroll
            for (int i = kRows - 1; i >= 0; --i) {
                float to_x[W], to_gate[W];
#pragma unroll
                for (int w = 0; w < W; ++w) up(i, w, g.v[i], m[w], to_x[w], to_gate[w]);
                Few<T, W> r, t;
                r.set(to_x), t.set(to_gate);
                r.store(dx), t.store(dg);
                next(dx, -a.lddx), next(dg, -a.lddg);
            }
        } else if (other) {
#pragma unroll
            for (int i = kRows - 1; i >= 0; --i) {
                if (lasts >> i & 1) {
                    const float* from = states_of(a, a.dlast, a.dlast ? sequence_of(a, now, row, i) : 0, at.col);
#pragma unroll
                    for (int w = 0; w < W; ++w) m[w] = from ? from[w] : 0.f;
                }
                float to_x[W], to_gate[W];
                const auto gi = g.v[i].again();
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    float to = m[w];
                    up(i, w, gi, to, to_x[w], to_gate[w]);
                    if (in >> i & 1) m[w] = to;
                    else to_x[w] = to_gate[w] = 0.f;
                }
                Few<T, W> r, t;
                r.set(to_x), t.set(to_gate);
                if (mine >> i & 1) r.store(dx), t.store(dg);
                next(dx, -a.lddx), next(dg, -a.lddg);
                if (float* const to = (firsts >> i & 1) && a.dinitial ? states_of(a, a.dinitial, sequence_of(a, now, row, i), at.col) : nullptr)
#pragma unroll
                    for (int w = 0; w < W; ++w) to[w] = m[w];
            }
        }
        leave<W>(e, a, at, (int)step, m);
    }
    range.others<W>(a, at, [&](int64_t c) {
        const uint32_t mine = rows_within(c * kRows, begin, end);
        clear_rows<T, W>(a.dx, a.lddx, c * kRows, mine, at.col);
        clear_rows<T, W>(a.dgate, a.lddg, c * kRows, mine, at.col);
    });
}

// A thread takes eight columns of a row.  Bound by memory, or by the call where there is little: 512 x 4,096 bfloat16 6.6 us (the first
// kernel, one column a thread, 8.0), 64 x 40 floats 2.4.
constexpr int kStepColumns = 8;
template <class T, bool SIGMOID>
__global__ __launch_bounds__(256) void k_step(int64_t n, int d, const T* x, int64_t ldx, const T* gate, int64_t ldg, float* state, int64_t lds, T* y,
                                              int64_t ldy) {
    const int64_t groups = (d + kStepColumns - 1) / kStepColumns;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n * groups; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / groups, c = (i - r * groups) * kStepColumns;
        const bool whole = c + kStepColumns <= d;
        Values<T, kStepColumns> u, z, out;
        Values<float, kStepColumns> h;
        u.load(x + r * ldx, c, d, whole), z.load(gate + r * ldg, c, d, whole), h.load(state + r * lds, c, d, whole);
#pragma unroll
        for (int j = 0; j < kStepColumns; ++j) {
            const Terms w = terms_of<SIGMOID>(u.get(j), z.get(j));
            const float v = fmaf(w.a, h.get(j), w.u);
            h.set(j, v), out.set(j, v);
        }
        h.store(state + r * lds, c, d, whole), out.store(y + r * ldy, c, d, whole);
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

// How a call's work is shared out, and where its temporaries lie in the workspace (from 0 on).
struct Layout {
    int width, strips, lanes, groups, shares;
    int64_t rows, chunks;
    int64_t share, chunk, of_row, carry, bytes;
};

// Blocks of a launch: two of 512 threads a CU.  Twice as many split more sequences: 32,768 x 4,096 bfloat16 in 16, both ways, 481 us in place of 454,
// 10,007 x 777 half precision 90 in place of 78, one sequence of 65,537 x 100 36.0 in place of 28.3; the histories alone gain, 131 in place of 134.
constexpr int64_t kBlocks = 512;
// One block a CU where rows are wide, which leaves fewer sequences that go on from share to share and starts each block once.  Both ways,
// microseconds with it and without; "ragged": lengths by a power law.
//   bfloat16, taken:  32,768 x 4,096 in 16 454 and 483, in 8 451 and 620, in 30 ragged 525 and 620; 40,000 rows in 16: 4,096 wide 556 and 557, 6,000
//                     1,081 and 1,196, 8,192 1,087 and 1,109; 5,000 wide in 20 ragged 1,020 and 1,168
//   not taken:        short sequences, whose instructions need the waves (32,768 x 4,096 in 512 702 and 650, ragged 623 and 565); rows below 8 KB,
//                     where it depends on the lengths: 65,000 x 1,000 in 64 ragged 412 and 394, 40,000 x 2,500 in 20 ragged 629 and 625, but
//                     3,500 789 and 855, and in 16 alike 2,048 wide 289 and 381, 2,500 555 and 618, 3,500 723 and 843, 4,000 759 and 777
//   floats, taken:    65,536 x 1,024 in 16 532 and 592, in 500 426 and 454, in 8,000 ragged 498 and 531; 32,768 x 2,048 in 4,000 469 and 475, ragged 493
//                     and 510; 32,768 x 4,096 in 16 796 and 813 (in 512 842 and 828)
//   not taken:        300,000 x 200 in 50 750 and 733; but 65,536 x 512 in 50 288 and 307, 800 wide 486 and 566
bool one_block_a_cu(const ccdpp_scan_t* p) {
    return p->dtype == CCDPP_F32 ? p->d >= 1024 : p->d >= 4096 && p->n / 256 >= p->s;
}
// Bytes of a row that the lanes of a group take at least, where strips are made narrower for more blocks.  With 128 bytes 10,007 x 777 half precision
// takes 36.2 us forward in place of 34.2, 1,000 x 4,096 bfloat16 23.8 in place of 21.9, 4,000 x 200 floats 21.6 in place of 17.1; the fewest rows
// gain (256 x 4,096 bfloat16 11.7 in place of 14.2).
constexpr int kPiece = 256;
// Values from which on the gradients take two columns a thread: 289 us in place of 375 for 32,768 x 4,096 bfloat16, where their instructions
// bound them; one column leaves registers for twice the waves, which wait less: 44.7 in place of 46.3 for 10,007 x 777 half precision.
constexpr int64_t kMuch = 1 << 25;

Layout layout(const ccdpp_scan_t* p, int32_t call) {
    Layout l;
    l.width = p->d >= 2 && (call == CCDPP_SCAN_FORWARD || p->n * p->d >= kMuch) ? 2 : 1;
    const int lanes = (p->d + l.width - 1) / l.width;
    l.chunks = (p->n + kRows - 1) / kRows;
    const int64_t blocks = one_block_a_cu(p) ? kBlocks / 2 : kBlocks;
    int64_t shares = 1;
    for (int widest = kLanes;; widest /= 2) {
        l.strips = (lanes + widest - 1) / widest;
        l.lanes = (lanes + l.strips - 1) / l.strips;
        l.groups = std::min(kThreads / l.lanes, 64);
        shares = std::max<int64_t>(1, std::min(blocks / l.strips, l.chunks / l.groups));
        if (l.strips * shares >= blocks || widest * l.width * (p->dtype == CCDPP_F32 ? 4 : 2) <= kPiece) break;
    }
    l.rows = round_up((std::max<int64_t>(p->n, 1) + shares - 1) / shares, kRows);
    l.shares = (int)((std::max<int64_t>(p->n, 1) + l.rows - 1) / l.rows);
    l.share = 0;
    l.chunk = round_up(l.share + (l.shares + 1) * (int64_t)sizeof(Share), 256);
    l.of_row = round_up(l.chunk + l.chunks * (int64_t)sizeof(Chunk), 256);
    l.carry = round_up(l.of_row + p->n * 4, 256);
    l.bytes = round_up(l.carry + (int64_t)l.shares * p->d * 8, 256);
    return l;
}

int64_t workspace(const ccdpp_scan_t* p, int32_t call) { return layout(p, call).bytes; }

void set(Scan& a, const ccdpp_scan_t* p, const Layout& l, void* ws) {
    a.n = p->n, a.s = p->s, a.ldx = p->ldx, a.ldg = p->ldg, a.d = p->d, a.bits = p->starts_bits;
    a.x = p->x, a.gate = p->gate, a.starts = p->starts, a.initial = p->initial;
    a.strips = l.strips, a.lanes = l.lanes, a.groups = l.groups, a.shares = l.shares, a.rows = l.rows, a.near = l.rows * 3 / 16, a.chunks = l.chunks;
    a.share = (Share*)((char*)ws + l.share), a.chunk = (Chunk*)((char*)ws + l.chunk), a.of_row = (int32_t*)((char*)ws + l.of_row);
    a.carry = (float*)((char*)ws + l.carry);
    a.sums = l.strips * (l.shares - 1);
    a.tables = (int)((l.chunks + kThreads - 1) / kThreads);
    a.marks = (l.shares + 1 + kThreads / 64 - 1) / (kThreads / 64);
}

template <bool GRAD>
int launch(const ccdpp_scan_t* p, const Layout& l, const Scan& a, bool ends, hipStream_t st) {
    const int64_t nones = ends ? (p->s + kThreads - 1) / kThreads : 0;
    const int64_t first = (int64_t)a.sums + a.tables + a.marks + nones;
    typed(p->dtype, p->mode, [&](auto z, auto sigmoid) {
        typedef decltype(z) T;
        constexpr bool S = decltype(sigmoid)::value;
        const auto both = [&](auto w) {
            constexpr int W = decltype(w)::value;
            k_scan_first<T, W, S, GRAD><<<(unsigned)first, kThreads, 0, st>>>(a);
            if (p->n == 0) return;
            if constexpr (GRAD) k_scan_grad<T, W, S><<<(unsigned)(l.strips * l.shares), kThreads, 0, st>>>(a);
            else k_scan<T, W, S><<<(unsigned)(l.strips * l.shares), kThreads, 0, st>>>(a);
        };
        if (l.width == 2) both(std::integral_constant<int, 2>());
        else both(std::integral_constant<int, 1>());
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CCDPP_OK : hip_fail(e, GRAD ? "gated scan gradients" : "gated scan");
}

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
    *bytes = (p->n + kRows - 1) / kRows * p->d * 4;
    return CCDPP_OK;
}

int ccdpp_gated_scan(const ccdpp_scan_t* p, void* y, int64_t ldy, float* last, void* kept, void* ws, int64_t ws_bytes, void* stream) {
    using namespace ccdops;
    if (int rc = check(p)) return rc;
    if (int rc = check_pointers(p, kept, ws, ws_bytes, workspace(p, CCDPP_SCAN_FORWARD))) return rc;
    if (p->n > 0 && !y) return fail(CCDPP_EINVAL, "y must be non-NULL");
    if (ldy < p->d) return fail(CCDPP_EINVAL, "ldy must be at least d");
    if (p->n > 0 && (y == p->x || y == p->gate)) return fail(CCDPP_EINVAL, "an output must not be an input");
    // (Not in place: the block that has a sequence's first row reads its initial state, and the one that has its last row writes the last.)
    if (last && last == p->initial && p->s > 0) return fail(CCDPP_EINVAL, "last must not be initial");
    if (misaligned(y, p->dtype == CCDPP_F32 ? 4 : 2) || misaligned(last, 4)) return fail(CCDPP_EINVAL, "pointers must be aligned to their types");
    if (int rc = check_device()) return rc;
    const Layout l = layout(p, CCDPP_SCAN_FORWARD);
    Scan a = {};
    set(a, p, l, ws);
    a.y = y, a.ldy = ldy, a.last = last, a.keep = (float*)kept;
    return launch<false>(p, l, a, last != nullptr, (hipStream_t)stream);
}

int ccdpp_gated_scan_grad(const ccdpp_scan_t* p, const void* dy, int64_t lddy, const float* dlast, const void* kept, void* dx, int64_t lddx, void* dgate,
                          int64_t lddg, float* dinitial, void* ws, int64_t ws_bytes, void* stream) {
    using namespace ccdops;
    if (int rc = check(p)) return rc;
    if (int rc = check_pointers(p, kept, ws, ws_bytes, workspace(p, CCDPP_SCAN_GRAD))) return rc;
    if (p->n > 0 && (!dy || !kept || !dx || !dgate)) return fail(CCDPP_EINVAL, "dy, kept, dx and dgate must be non-NULL");
    if (lddy < p->d || lddx < p->d || lddg < p->d) return fail(CCDPP_EINVAL, "lddy, lddx and lddg must be at least d");
    if (p->n > 0 && (dx == p->x || dx == p->gate || dx == dy || dgate == p->x || dgate == p->gate || dgate == dy || dx == dgate))
        return fail(CCDPP_EINVAL, "an output must not be an input");
    const uintptr_t es = p->dtype == CCDPP_F32 ? 4 : 2;
    if (misaligned(dy, es) || misaligned(dx, es) || misaligned(dgate, es) || misaligned(dlast, 4) || misaligned(dinitial, 4))
        return fail(CCDPP_EINVAL, "pointers must be aligned to their types");
    if (int rc = check_device()) return rc;
    if (dinitial && dinitial == dlast && p->s > 0) return fail(CCDPP_EINVAL, "dinitial must not be dlast");  // as for last and initial
    const Layout l = layout(p, CCDPP_SCAN_GRAD);
    Scan a = {};
    set(a, p, l, ws);
    a.y = const_cast<void*>(dy), a.ldy = lddy, a.dlast = dlast, a.kept = (const float*)kept;
    a.dx = dx, a.lddx = lddx, a.dgate = dgate, a.lddg = lddg, a.dinitial = dinitial;
    return launch<true>(p, l, a, dinitial != nullptr, (hipStream_t)stream);
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
    const int64_t blocks = (n * ((d + kStepColumns - 1) / kStepColumns) + 255) / 256;
    typed(dtype, mode, [&](auto z, auto sigmoid) {
        typedef decltype(z) T;
        k_step<T, decltype(sigmoid)::value><<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, (hipStream_t)stream>>>(n, d, (const T*)x, ldx, (const T*)gate, ldg,
                                                                                                                       state, lds, (T*)y, ldy);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CCDPP_OK : hip_fail(e, "gated scan step");
}

}  // extern "C"
