// The best continuations of beams, and the beams' states in their order (gfx950).
//
// Beam b continued by item i has the score  s_b + z_bi - L_b,  L_b = log sum_j exp z_bj.  Within a beam the order is that of z, which is
// exact in 32 bits: a row leaves its k greatest keys (z, then the lowest item).  Between beams scores are compared in 64 bits.
//
// Bound by reading the logits once where they are many: 512 rows of 624,961 floats with offsets 248 us (5.2 TB/s, a copy's rate; streams that
// are only read reach 6.5 to 6.8).  Less of them is bound by instructions and rounds to LDS one after another: 128 rows of 131,072 in bfloat16
// 24 us (14 without the selection; 5.2 would be a read from the memory-side cache), then 9 for joining, most of it rounds to memory, and 4 for
// the states.
#include <algorithm>
#include <cmath>

#include "ccdpp_seq.h"
#include "ops_internal.hpp"

namespace ccdops {
namespace {

constexpr int kMost = 64;             // beams of a group, and continuations
constexpr int64_t kGrid = 1 << 20;    // blocks of a launch

// (The kernel before this one, which took a chunk's greatest values out one by one, up to k times a chunk, instead of comparing with a bound: 32
// us for the 128 rows above.)
constexpr int kEach = 32;             // logits of a lane in a chunk
constexpr int kChunk = 64 * kEach;    // of a wave
constexpr int kWaves = 4;             // of a block
constexpr float kLog2e = 1.44269504f;

// Ascending order of values as whole numbers: NaN last.
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t u = __float_as_uint(z);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ uint64_t order_of(double z) {
    if (z != z) return ~0ull;
    const uint64_t u = (uint64_t)__double_as_longlong(z + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// The greatest value of a wave, for all its lanes: lanes of a row of 16 from each other, then the rows' last ones.
template <int CTRL, int ROWS, class V>
__device__ __forceinline__ V from_lane(V v) {
    const int x = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(x, x, CTRL, ROWS, 0xF, false));
}
template <class V>
__device__ __forceinline__ V greater(V a, V b) { return a > b ? a : b; }
__device__ __forceinline__ float greater(float a, float b) { return fmaxf(a, b); }
template <class V>
__device__ __forceinline__ V wave_max(V v) {
    v = greater(v, from_lane<0x111, 0xF>(v));
    v = greater(v, from_lane<0x112, 0xF>(v));
    v = greater(v, from_lane<0x114, 0xF>(v));
    v = greater(v, from_lane<0x118, 0xF>(v));
    v = greater(v, from_lane<0x142, 0xA>(v));
    v = greater(v, from_lane<0x143, 0xC>(v));
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
    const uint32_t hi = wave_max((uint32_t)(v >> 32)), lo = wave_max((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
    return (uint64_t)hi << 32 | lo;
}
template <class V>
__device__ __forceinline__ V lane_of(V v, int lane) { return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }
__device__ __forceinline__ uint64_t lane_of(uint64_t v, int lane) { return (uint64_t)lane_of((uint32_t)(v >> 32), lane) << 32 | lane_of((uint32_t)v, lane); }

// The greatest keys of a wave in descending order, one a lane; 0: none.  A key is a value's order and then the lowest item, so no two are equal.
struct Best {
    uint64_t key;
    __device__ __forceinline__ void insert(uint64_t k) {
        const int at = __popcll(__ballot(key > k)), lane = threadIdx.x & 63;
        const uint32_t hi = from_lane<0x138, 0xF>((uint32_t)(key >> 32)), lo = from_lane<0x138, 0xF>((uint32_t)key);  // of the lane before
        key = lane < at ? key : lane == at ? k : (uint64_t)hi << 32 | lo;
    }
};

struct Beam {
    int64_t groups, v, ld, end;
    int beams, k, shares;
    int64_t each;      // chunks of a share of a row
    const void* logits;
    const float *score, *offset;
    const uint8_t* done;
    float* out_score;
    int64_t *parent, *item;
    uint8_t* out_done;
    double* sums;      // of exponentials over a share, relative to
    float* refs;       // about its greatest logit; inf where that is inf or NaN, -inf where nothing takes part
    uint64_t* keys;    // k of each share, descending; 0: none
};

// A chunk's logits as they are in memory, and their offsets: lane l has V side by side at l V, and again every 64 V.
template <class T, bool OFFSET>
struct Chunk {
    static constexpr int V = 16 / sizeof(T), J = kEach / V;
    Run<T, V> raw[J];
    Run<float, 4> off[OFFSET ? kEach / 4 : 1];
    __device__ __forceinline__ void load(const T* row, const float* offset, int64_t first, int64_t v) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int64_t i = first + j * 64 * V + lane * V;
            if (first + kChunk <= v || i + V <= v) {
                raw[j] = load_run<V>(row + i);
                if constexpr (OFFSET)
#pragma unroll
                    for (int q = 0; q < V / 4; ++q) off[j * V / 4 + q] = load_run<4>(offset + i + 4 * q);
            } else {
#pragma unroll
                for (int w = 0; w < V; ++w) {
                    raw[j].v[w] = i + w < v ? row[i + w] : (T)-INFINITY;
                    if constexpr (OFFSET) off[(j * V + w) / 4].v[w % 4] = i + w < v ? offset[i + w] : 0.f;
                }
            }
        }
    }
    // The logit with its offset; -inf where it takes no part.
    __device__ __forceinline__ float get(int e) const {
        const float z = (float)raw[e / V].v[e % V];
        if constexpr (!OFFSET) return z;
        const float o = off[e / 4].v[e % 4];
        return o < -1e38f ? -INFINITY : z + o;
    }
};

// What a wave has found: keys in no order, of which the k greatest count.  A value is put there if it is above `own`, the k-th greatest of
// those there or less (later items do not go before equal ones that are there), and not below what another wave of the block knows.
constexpr int kFound = 192, kAdded = 128;
struct Found {
    uint64_t* keys;
    int n;
    float own;
    static __device__ __forceinline__ void agree() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    // Leaves the k greatest, in descending order: a key's place is the number of greater ones.
    __device__ __forceinline__ void prune(int k) {
        const int lane = threadIdx.x & 63;
        agree();
        uint64_t mine[kFound / 64];
        int place[kFound / 64];
#pragma unroll
        for (int u = 0; u < kFound / 64; ++u) mine[u] = lane + 64 * u < n ? keys[lane + 64 * u] : 0, place[u] = 0;
#pragma unroll
        for (int v = 0; v < kFound / 64; ++v) {
            const int last = min(n - 64 * v, 64);
            for (int i = 0; i < last; ++i) {
                const uint64_t other = lane_of(mine[v], i);
#pragma unroll
                for (int u = 0; u < kFound / 64; ++u)
                    if (64 * u < n) place[u] += other > mine[u];
            }
        }
        agree();
#pragma unroll
        for (int u = 0; u < kFound / 64; ++u)
            if (lane + 64 * u < n && place[u] < k) keys[place[u]] = mine[u];
        agree();
        if (n >= k) own = fmaxf(own, value_of(__builtin_amdgcn_readfirstlane((uint32_t)(keys[k - 1] >> 32))));
        n = min(n, k);
    }
};

// One block for each share of a row.  Its waves take chunks in turn; a chunk is read once: its exponentials are added up relative to about the
// lane's greatest logit so far (in 32 bits within a chunk, in 64 over them), then what may be among the k best is put aside.
// What they are relative to is raised only where a logit is more than 1 above it, so a term that ends D below it is rounded for D + 3 raises at
// most, however long the row is.  With u = 2^-24 (half a step of 32 bits): 2 u each and 2.3 u for each 1 of D, in the exponential and the
// raises together; 2 u for the exponential, 9 u for its chunk's sum: (4.3 D + 20) u.  Of fewer than 2^28 terms the mean D by weight is below
// 16, so the sum is within 90 u < 2^-17 of itself.  (Raised with every new maximum, the log sum of 2^28 ascending floats was 2^-14 off.)  Of a wave's
// first chunk that is what is not below the k-th greatest of its lanes' greatest values; with values in any order little is found after that.
// Where more than kAdded values pass, a bound is looked for that at least k and no more than kAdded pass; where there is none (many equal
// ones), the k greatest of the chunk are taken out one by one.
// (Registers for four waves a SIMD where a chunk of raw values takes 16.)
template <class T, bool OFFSET>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 2 && !OFFSET ? 4 : 2) void k_beam_rows(Beam a) {
    typedef Chunk<T, OFFSET> C;
    __shared__ uint64_t keys[kWaves][kFound];
    __shared__ double sums[kWaves];
    __shared__ float refs[kWaves];
    __shared__ int counts[kWaves];
    __shared__ uint32_t known;  // the order of a value that k of the block's are not below
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t items = a.groups * a.beams * a.shares;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = item / a.shares;
        if (a.score[row] == -INFINITY || (a.done && a.done[row])) continue;
        const int64_t begin = (item - row * a.shares) * a.each, end = min(begin + a.each, (a.v + kChunk - 1) / kChunk);
        const T* const base = (const T*)a.logits + row * a.ld;
        C next;
        if (begin + wave < end) next.load(base, a.offset, (begin + wave) * kChunk, a.v);
        __syncthreads();
        if (threadIdx.x == 0) known = 0;
        __syncthreads();
        Found found = {keys[wave], 0, -INFINITY};
        float ref = -INFINITY;  // of the lane
        double sum = 0.0;
        for (int64_t c = begin + wave; c < end; c += kWaves) {
            float z[kEach];
#pragma unroll
            for (int e = 0; e < kEach; ++e) z[e] = next.get(e);
            if (c + kWaves < end) next.load(base, a.offset, (c + kWaves) * kChunk, a.v);
            const uint32_t all_know = *(volatile uint32_t*)&known;
            float run[C::J];  // the greatest of a run
            const auto greatest = [&] {
                float m = -INFINITY;
#pragma unroll
                for (int j = 0; j < C::J; ++j) {
                    run[j] = z[j * C::V];
#pragma unroll
                    for (int w = 1; w < C::V; ++w) run[j] = fmaxf(run[j], z[j * C::V + w]);
                    m = fmaxf(m, run[j]);
                }
                return m;
            };
            float m = greatest();
            const float was = ref;
            ref = m > ref + 1.f ? m : ref;
            const float to = ref == -INFINITY ? 0.f : ref;
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < kEach; ++e) part[e & 3] += __builtin_amdgcn_exp2f((z[e] - to) * kLog2e);
            const float parts = (part[0] + part[1]) + (part[2] + part[3]);
            if (__ballot(parts != parts)) {  // NaN (or infinity less infinity): NaN counts as infinity
#pragma unroll
                for (int e = 0; e < kEach; ++e) z[e] = z[e] != z[e] ? INFINITY : z[e];
                m = greatest();
                if (m == INFINITY) ref = m;
            }
            sum = sum * (was == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((was - to) * kLog2e)) + (double)parts;
            // At least `bound`: above own, and not below what others know.
            const auto bound_of = [&] { return value_of(max(order_of(found.own + 0.f) + 1, all_know)); };
            float bound = bound_of();
            uint64_t lanes = __ballot(m >= bound);
            if (!lanes) continue;
            const auto key_of = [&](float v, int at) { return (uint64_t)order_of(v + 0.f) << 32 | (uint32_t)~(uint32_t)(c * kChunk + at); };  // (-0 is 0)
            float raised = -INFINITY;
            if (__popcll(lanes) > a.k) {  // the k-th greatest of the lanes' greatest
                int above = 0;
#pragma unroll
                for (int l = 0; l < 64; ++l) above += lane_of(m, l) > m;
                raised = -wave_max(above < a.k ? -m : -INFINITY);
                bound = fmaxf(bound, raised);
            }
            int passing = __popcll(__ballot(m >= bound)) * kEach;  // at most
            if (passing > kAdded) {
                passing = 0;
#pragma unroll
                for (int e = 0; e < kEach; ++e) passing += __popcll(__ballot(z[e] >= bound));
            }
            if (passing > kAdded) {  // (halving what lies between the bound and the greatest value, up to 32 times)
                uint32_t low = order_of(bound + 0.f), high = order_of(wave_max(m) + 0.f) + 1;  // too many are not below low, none not below high
                while (high - low > 1) {
                    const uint32_t mid = low + (high - low) / 2;
                    const float v = value_of(mid);
                    int n = 0;
#pragma unroll
                    for (int e = 0; e < kEach; ++e) n += __popcll(__ballot(z[e] >= v));
                    if (n > kAdded) low = mid;
                    else if (n < a.k) high = mid;
                    else {
                        bound = raised = v, passing = n;
                        break;
                    }
                }
            }
            if (found.n + min(passing, kAdded) > kFound) found.prune(a.k);
            if (passing <= kAdded) {
                asm("" : "+v"(bound));  // (compared again: 32 masks would not stay in scalar registers)
#pragma unroll
                for (int j = 0; j < C::J; ++j) {
                    if (!__ballot(run[j] >= bound)) continue;
#pragma unroll
                    for (int w = 0; w < C::V; ++w) {
                        const int e = j * C::V + w;
                        const bool pass = z[e] >= bound;
                        const uint64_t those = __ballot(pass);
                        if (!those) continue;
                        const int at = found.n + __builtin_amdgcn_mbcnt_hi((uint32_t)(those >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)those, 0));
                        if (pass) found.keys[at] = key_of(z[e], j * 64 * C::V + lane * C::V + w);
                        found.n += __popcll(those);
                    }
                }
            } else {
                bound = bound_of();
                raised = -INFINITY;
                for (int i = 0; i < a.k && __ballot(m >= bound); ++i) {
                    const float most = wave_max(m);
                    // The lowest item that has it, and out with it.
                    int at = 0;
                    bool there = false;
#pragma unroll
                    for (int j = 0; j < C::J; ++j) {
                        if (there) continue;
                        uint64_t any = 0;
#pragma unroll
                        for (int w = 0; w < C::V; ++w) any |= __ballot(z[j * C::V + w] == most);
                        if (any) {
                            there = true;
                            const int owner = __ffsll((unsigned long long)any) - 1;
                            int which = 0;
#pragma unroll
                            for (int w = C::V - 1; w >= 0; --w)
                                if (__ballot(z[j * C::V + w] == most) >> owner & 1) which = w;
#pragma unroll
                            for (int w = 0; w < C::V; ++w) z[j * C::V + w] = lane == owner && w == which ? -INFINITY : z[j * C::V + w];
                            at = j * 64 * C::V + owner * C::V + which;
                        }
                    }
                    m = greatest();
                    if (lane == 0) found.keys[found.n] = key_of(most, at);
                    ++found.n;
                    if (i + 1 == a.k) raised = most;
                }
            }
            const float before = found.own;
            found.own = fmaxf(before, raised);
            if (found.n >= 2 * a.k) found.prune(a.k);
            if (found.own > before && lane == 0) atomicMax(&known, order_of(found.own + 0.f));
        }
        found.prune(a.k);
        const float all = wave_max(ref);
        if (ref != all) sum *= ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ref - all) * kLog2e);
        for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
        if (lane == 0) sums[wave] = sum, refs[wave] = all, counts[wave] = found.n;
        __syncthreads();
        // Places among all waves' keys.
        const uint64_t mine = lane < found.n ? keys[wave][lane] : 0;
        int place = lane, total = 0;
        uint64_t theirs[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) theirs[w] = keys[w][lane];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const int n = __builtin_amdgcn_readfirstlane(counts[w]);
            total += n;
            if (w == wave) continue;
            for (int i = 0; i < n; ++i) place += lane_of(theirs[w], i) > mine;
        }
        if (lane < found.n && place < a.k) a.keys[item * a.k + place] = mine;
        if (wave == 0) {
            if (lane >= total && lane < a.k) a.keys[item * a.k + lane] = 0;
            if (lane == 0) {
                float t = refs[0];
                for (int w = 1; w < kWaves; ++w) t = fmaxf(t, refs[w]);
                double s = 0.0;
                for (int w = 0; w < kWaves; ++w)
                    if (refs[w] != -INFINITY) s += sums[w] * (double)__builtin_amdgcn_exp2f((refs[w] - t) * kLog2e);
                a.sums[item] = s, a.refs[item] = t;
            }
        }
    }
}

// One block a group: a wave joins the shares of a row, then the first wave goes down the beams' lists, lane b that of beam b.
__global__ __launch_bounds__(1024) void k_beam_join(Beam a) {
    __shared__ uint64_t lists[kMost][kMost];
    __shared__ double logs[kMost];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    for (int64_t g = blockIdx.x; g < a.groups; g += gridDim.x) {
        float my_score = -INFINITY;  // of beam `lane`
        bool my_done = false;
        if (lane < a.beams) my_score = a.score[g * a.beams + lane], my_done = a.done && a.done[g * a.beams + lane];
        for (int b = wave; b < a.beams; b += waves) {
            const int64_t row = g * a.beams + b;
            const int64_t first = row * a.shares;
            // What most rows need is asked for at once: the first lists, references and sums.  (Where the beam is none or done they hold nothing.)
            constexpr int kAtOnce = 8;
            uint64_t other[kAtOnce];
            const auto ask = [&](int s) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) other[u] = lane < a.k && s + u < a.shares ? a.keys[(first + s + u) * a.k + lane] : 0;
            };
            float my_ref = -INFINITY;
            double my_sum = 0.0;
            if (lane < a.shares) my_ref = a.refs[first + lane], my_sum = a.sums[first + lane];
            ask(0);
            if (lane_of(my_score, b) == -INFINITY || __ballot(my_done) >> b & 1) continue;
            Best best = {other[0]};
            other[0] = 0;
            for (int s = 0;;) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    for (int j = 0; j < a.k; ++j) {
                        const uint64_t k = lane_of(other[u], j);
                        if (k <= lane_of(best.key, a.k - 1)) break;
                        best.insert(k);
                    }
                s += kAtOnce;
                if (s >= a.shares) break;
                ask(s);
            }
            for (int s = lane + 64; s < a.shares; s += 64) {
                const float t = a.refs[first + s], more = fmaxf(my_ref, t);
                if (t == -INFINITY) continue;
                my_sum = my_sum * (my_ref == -INFINITY ? 0.0 : exp((double)my_ref - more)) + a.sums[first + s] * exp((double)t - more);
                my_ref = more;
            }
            const float ref = wave_max(my_ref);
            double sum = my_sum;
            if (a.shares > 1) {
                sum = my_ref == -INFINITY ? 0.0 : my_sum * exp((double)my_ref - ref);
                for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
            }
            if (lane < a.k) lists[b][lane] = best.key;
            if (lane == 0) logs[b] = ref == INFINITY ? (double)NAN : ref + log(sum);
        }
        __syncthreads();
        if (wave == 0) {
            const int b = lane;
            const float s = my_score;
            const bool done = my_done;
            const bool live = s != -INFINITY;
            const double sum = live && !done ? logs[b] : 0.0;
            int at = 0;
            for (int j = 0; j < a.k; ++j) {
                double value = -INFINITY;
                int64_t item = -1;
                if (live && done && at == 0) value = s, item = a.end;
                if (live && !done && at < a.k) {
                    const uint64_t key = lists[b][at];
                    if (key) value = s + ((double)value_of((uint32_t)(key >> 32)) - sum), item = (uint32_t)~(uint32_t)key;
                }
                const uint64_t mine = order_of(value), most = wave_max(mine);
                const bool none = most == order_of((double)-INFINITY);
                const int winner = __ffsll((unsigned long long)__ballot(mine == most)) - 1;
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
        __syncthreads();
    }
}

constexpr int kTable = 16;  // tensors a launch

struct Moves {
    const char* in[kTable];
    char* out[kTable];
    int64_t stride[kTable], bytes[kTable];
    const int64_t* parent;
    int64_t rows, pieces;  // groups * k; pieces of a row of all tensors
    int beams, k, n;
};

// Rows of out are cut into pieces of kPiece bytes, one for each block of 256 threads at a time: a run of 16 bytes for each, and the
// bytes that a row has over one by one.
constexpr int64_t kPiece = 4096;
__global__ __launch_bounds__(256) void k_reorder(Moves m) {
    const int64_t items = m.rows * m.pieces;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t at = item / m.pieces;
        const int64_t g = at / m.k, parent = m.parent[at];
        const bool there = parent >= 0 && parent < m.beams;
        int64_t piece = item - at * m.pieces;
        int t = 0;
        while (piece >= (m.bytes[t] + kPiece - 1) / kPiece) piece -= (m.bytes[t] + kPiece - 1) / kPiece, ++t;
        const int64_t lo = piece * kPiece + 16 * threadIdx.x;
        const uint8_t* from = (const uint8_t*)m.in[t] + (g * m.beams + (there ? parent : 0)) * m.stride[t];
        uint8_t* to = (uint8_t*)m.out[t] + at * m.bytes[t];
        typedef words4 loose __attribute__((aligned(1), may_alias));
        if (lo + 16 <= m.bytes[t]) {
            *(loose*)(to + lo) = there ? *(const loose*)(from + lo) : (words4){0, 0, 0, 0};
        } else {
            for (int64_t i = lo; i < m.bytes[t]; ++i) to[i] = there ? from[i] : (uint8_t)0;
        }
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

// How a row is shared out among blocks, and where the shares' results lie in the workspace (from 0 on).  Three blocks a CU are wanted: a wave's
// first chunk costs the most, so fewer shares are better for many rows, but too few leave waits bare.  Whole calls, microseconds with 512, 768 and
// 1,024 blocks wanted:
//   131,072 bfloat16: 128 rows 33.6, 34.3, 32.2 (256 blocks 39.1); 256 46.3, 43.3, 42.3; 384 64.2, 50.0, 49.9; 400 64.1, 64.4, 52.9; 512 65.6, 65.6,
//                     54.3; 768 72.0, 71.9, 71.7
//   624,961 floats:   400 rows 230, 231, 252; 504 247, 247, 261; 512 258, 258, 270
// So 768 is the best for many logits (385 to 767 rows get one share each), and up to a fifth behind 1,024 for as many rows of fewer logits.
struct Layout {
    int64_t shares, each, sums, refs, keys, bytes;
};

Layout layout(const ccdpp_beam_t* p) {
    Layout l;
    const int64_t rows = p->groups * p->beams, chunks = (p->v + kChunk - 1) / kChunk;
    const int64_t wanted = std::max<int64_t>(1, std::min<int64_t>(768 / std::max<int64_t>(rows, 1), 256));
    l.each = std::max<int64_t>(round_up((chunks + wanted - 1) / wanted, kWaves), kWaves);
    l.shares = (chunks + l.each - 1) / l.each;
    l.sums = 0;
    l.refs = round_up(rows * l.shares * 8, 256);
    l.keys = l.refs + round_up(rows * l.shares * 4, 256);
    l.bytes = l.keys + round_up(rows * l.shares * p->k * 8, 256) + 256;
    return l;
}

int64_t workspace(const ccdpp_beam_t* p) { return layout(p).bytes; }

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
    const Layout l = layout(p);
    Beam a = {};
    a.groups = p->groups, a.v = p->v, a.ld = p->ld, a.end = p->end, a.beams = p->beams, a.k = p->k, a.shares = (int)l.shares, a.each = l.each;
    a.logits = p->logits, a.score = p->score, a.offset = p->offset, a.done = p->done;
    a.out_score = out_score, a.parent = parent, a.item = item, a.out_done = out_done;
    a.sums = (double*)((char*)ws + l.sums), a.refs = (float*)((char*)ws + l.refs), a.keys = (uint64_t*)((char*)ws + l.keys);
    hipStream_t st = (hipStream_t)stream;
    const unsigned blocks = (unsigned)std::min<int64_t>(rows * l.shares, kGrid);
    const auto rows_of = [&](auto z) {
        typedef decltype(z) T;
        if (p->offset) k_beam_rows<T, true><<<blocks, 64 * kWaves, 0, st>>>(a);
        else k_beam_rows<T, false><<<blocks, 64 * kWaves, 0, st>>>(a);
    };
    if (p->dtype == CCDPP_F32) rows_of(float());
    else if (p->dtype == CCDPP_BF16) rows_of((__bf16)0.f);
    else rows_of((_Float16)0.f);
    k_beam_join<<<(unsigned)std::min<int64_t>(p->groups, kGrid), 64 * std::min(p->beams, 16), 0, st>>>(a);
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
        if (groups > 0 && row_bytes[i] > 0 && in[i] == out[i]) return fail(CCDPP_EINVAL, "an output must not be an input");
    }
    if (int rc = check_device()) return rc;
    if (groups == 0) return CCDPP_OK;
    Moves m;
    m.parent = parent, m.rows = groups * k, m.beams = beams, m.k = k, m.n = 0, m.pieces = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (row_bytes[i]) m.in[m.n] = (const char*)in[i], m.out[m.n] = (char*)out[i], m.stride[m.n] = in_stride[i], m.bytes[m.n] = row_bytes[i], m.pieces += (row_bytes[i] + kPiece - 1) / kPiece, ++m.n;
        if (!m.n || (m.n < kTable && i + 1 < n)) continue;
        k_reorder<<<(unsigned)std::min<int64_t>(m.rows * m.pieces, kGrid), 256, 0, (hipStream_t)stream>>>(m);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "beam reordering");
        m.n = 0, m.pieces = 0;
    }
    return CCDPP_OK;
}

}  // extern "C"
