// Log probabilities, entropy and the largest of a row of logits, and their gradient.
//
// One pass: with the running maximum M, S = sum exp((z - M) / T) and
// W = sum exp((z - M) / T) (z - M) / T,
//   l_j = (z_j - M) / T - ln S;   entropy = ln S - W / S;
// when the maximum rises by d (in units of T), S becomes S exp(-d) and W exp(-d) (W - d S).
// Two runs' triples join the same way.  HBM bounds large calls (one read of the logits;
// the gradient one read and one write, two reads of rows far from 0), the call small ones.  8192 x 65536 in bf16 179 us (6.0 TB/s,
// 0.88 of a copy's rate), its gradient 312 (6.9 TB/s, 1.01); one row of 131072 with its 8 largest
// 8.3 us on a cluster of 8 blocks.  Two elements to an instruction took the first from 199 to 180 us.
//
// The K largest come from a second look at a small part of the row.  On the way each thread
// notes the largest of its pieces (16 bytes; the lowest column among equals).  Of the
// pieces' maxima, any K that are at hand bound the K-th from below, and every one of the
// row's K largest lies in a piece whose maximum is at or above that bound: only the strips
// of threads that hold such pieces are read again, and what is at or above the bound, a
// few dozen as a rule, is ranked by comparing all with all.  Of the shortest rows' they are found
// one after another, as all rows' are where there is no room for the candidates.  (Each warp keeping a sorted list
// in its lanes took up to five times the whole pass: an insertion is a dozen dependent
// exchanges; 1 x 131072, top 8, 18.2 us, and 8192 x 65536 753, now 8.3 and 268.)
//
// A row goes to a few lanes, to a block of threads, or, where rows are few and long, to a
// cluster of blocks that join through shared memory (1 x 131072: 12.6 us by one block, 4.6 by eight;
// 300 x 131072: 29.9 by one, 19.6 by two, 23.9 by eight).  Rows start anywhere: their aligned
// 16-byte pieces are loaded whole, the up to 14 elements around them singly.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_pair.cuh"
#include "nn_ptx.cuh"

namespace emtk {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostTop = 32, kMostCluster = 8;
// Pieces of a thread in flight: 512 x 131072 with 2, 4 and 8 42, 34 and 31 us, 8192 x 65536 192, 180 and 190, its gradient 324, 312 and 421.
constexpr int kFlight = 4;

constexpr float kFar = -1e4f;  // an exponent whose power is 0, in the place of -infinity where that would meet a 0

__device__ __forceinline__ float minus_infinity() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float not_a_number() { return __int_as_float(0x7fffffff); }

// Elements of each type: TYPE is an emtk_type.
template <int TYPE>
struct Elem {
    using T = uint16_t;
    static constexpr int kPer = 8;  // of 16 bytes
    static __device__ __forceinline__ float value(uint16_t x) { return from16<TYPE == EMTK_TYPE_F16>(x); }
    static __device__ __forceinline__ void values(const uint4 &q, float *v) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = from16<TYPE == EMTK_TYPE_F16>(w[i] & 0xffffu);
            v[2 * i + 1] = TYPE == EMTK_TYPE_F16 ? from16<true>(w[i] >> 16) : __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t r;
        if (TYPE == EMTK_TYPE_F16)
            asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else
            asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float largest(const uint4 &q) {  // NaN only if all are
        const float2 v = values_of<TYPE == EMTK_TYPE_F16>(larger(larger(q.x, q.y), larger(q.z, q.w)));
        return fmaxf(v.x, v.y);
    }
    static __device__ __forceinline__ uint16_t stored(float v) { return (uint16_t)to16<TYPE == EMTK_TYPE_F16>(v); }
    static __device__ __forceinline__ uint4 stored(const float *v) {
        constexpr bool F16 = TYPE == EMTK_TYPE_F16;
        return make_uint4(pack16<F16>(v[0], v[1]), pack16<F16>(v[2], v[3]), pack16<F16>(v[4], v[5]), pack16<F16>(v[6], v[7]));
    }
};
template <>
struct Elem<EMTK_TYPE_F32> {
    using T = float;
    static constexpr int kPer = 4;
    static __device__ __forceinline__ float value(float x) { return x; }
    static __device__ __forceinline__ void values(const uint4 &q, float *v) {
        v[0] = __uint_as_float(q.x), v[1] = __uint_as_float(q.y), v[2] = __uint_as_float(q.z), v[3] = __uint_as_float(q.w);
    }
    static __device__ __forceinline__ float largest(const uint4 &q) {
        return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
    }
    static __device__ __forceinline__ float stored(float v) { return v; }
    static __device__ __forceinline__ uint4 stored(const float *v) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};

// A row's layout: `head` elements, `pieces` of 16 aligned bytes, `tail` elements.
struct Split {
    int head, pieces, tail;
};
template <int TYPE>
__device__ __forceinline__ Split split_row(const void *p, int v) {
    using E = Elem<TYPE>;
    const int to_grid = (int)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(p) % 16)) % 16) / (int)sizeof(typename E::T);
    Split s;
    s.head = min(to_grid, v);
    s.pieces = (v - s.head) / E::kPer;
    s.tail = v - s.head - s.pieces * E::kPer;
    return s;
}

// ---------------------------------------------------------------- forward
// Maximum, S and W of a run of logits; k = log2(e) / T, W in units of log 2.
struct Sums {
    float m, s, w;
    __device__ __forceinline__ void clear() { m = minus_infinity(), s = w = 0.f; }
    // Raises the maximum to at least `to`.  A run without any logit above -infinity has s and
    // w 0 (or NaN, which stays).
    __device__ __forceinline__ void raise(float to, float k) {
        if (!(to > m)) return;
        const float d = m == minus_infinity() ? 0.f : fmaxf((m - to) * k, kFar);
        const float f = exp2_f(d);
        w = f * fmaf(d, s, w);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void join(Sums o, float k) {
        const float top = fmaxf(m, o.m);
        raise(top, k);
        o.raise(top, k);
        s += o.s;
        w += o.w;
    }
};
// A thread's: even and odd elements' sums apart, so that one instruction adds two.
struct Sums2 {
    float m;
    float2 s, w;
    __device__ __forceinline__ void clear() { m = minus_infinity(), s = w = both(0.f); }
    __device__ __forceinline__ void raise(float to, float k) {
        if (!(to > m)) return;
        const float d = m == minus_infinity() ? 0.f : fmaxf((m - to) * k, kFar);
        const float f = exp2_f(d);
        w = fma2(both(d), s, w) * both(f);
        s = s * both(f);
        m = to;
    }
    // N values, none above the maximum, absent ones -infinity.
    template <int N>
    __device__ __forceinline__ void add(const float (&z)[N], float k) {
        const float base = m == minus_infinity() ? 0.f : m;
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 d = (make_float2(z[i], z[i + 1]) - both(base)) * both(k);
            const float2 e = make_float2(exp2_f(d.x), exp2_f(d.y));
            s = s + e;
            w = fma2(e, make_float2(fmaxf(d.x, kFar), fmaxf(d.y, kFar)), w);  // of -infinity: 0
        }
    }
    __device__ __forceinline__ Sums all() const { return {m, s.x + s.y, w.x + w.y}; }
};

// Order of logits; NaN is the least.  Never 0.
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);  // -0 and 0 are equal
    return z != z ? 1u : b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
    return order == 1u ? not_a_number() : __uint_as_float((order & 0x80000000u) ? order & 0x7fffffffu : ~order);
}
// The lowest place first among equals; 0: nothing.
__device__ __forceinline__ uint64_t key_of(uint32_t order, int place) { return ((uint64_t)order << 32) | (uint32_t)~place; }
__device__ __forceinline__ int place_of(uint64_t key) { return (int)~(uint32_t)key; }

// lse is max / T + ln S rounded to fp32: off by up to half a step, and p = exp(z / T - lse) by so much of itself, 2^-20 up to
// 32, where ordinary rows end.  Beyond, up to a row of the type's least values, whose lse holds nothing of ln S any more, the
// gradient takes the row's maximum and S again: 8192 x 65536 in bf16 312 us of ordinary rows, 534 of such.  A row that is cut
// among blocks and overwritten has its sums taken first, by the forward kernel, a block to a row and so in the same order,
// which leaves ordinary rows at once (1 x 131072 in place 2.7 us, 2.0 apart).  With its own code for such rows an ordinary element has no instruction more:
// one for all took 345.
constexpr float kFarLse = 32.f;
__device__ __forceinline__ bool is_far(float lse) { return fabsf(lse) > kFarLse; }

struct LogprobArgs {
    const uint8_t *z;
    int64_t row_bytes;
    const int32_t *tokens;
    float *logprob, *entropy, *lse, *top_logprob;
    int32_t *top_index;
    int m, v, top;
    float k, inverse_t;  // log2(e) / T, 1 / T
    int lanes_log2;      // of a row, in lanes_kernel
    const float *far;    // the gradient's: rows whose lse is far alone, and of them
    float2 *sums;        // the maximum and S
};

// A thread's strip of a row, thread t of `threads` at part `part` of `parts` of it: every
// threads-th piece of the part, and the elements around the pieces, the head (unit 0; pieces
// are units 1 ..) for the first thread and the tail (the last unit) for the last.
template <int TYPE>
struct Strip {
    using E = Elem<TYPE>;
    const typename E::T *p;
    Split split;
    int t, threads, first, end;  // first piece, end of the part's pieces
    bool ends;                   // the part has the row's ends
    __device__ __forceinline__ Strip(const uint8_t *row, int v, int t, int threads, int part, int parts)
        : p(reinterpret_cast<const typename E::T *>(row)), split(split_row<TYPE>(row, v)), t(t), threads(threads) {
        const int each = (split.pieces + parts - 1) / parts;
        first = part * each + t;
        end = min((part + 1) * each, split.pieces);
        ends = part == 0;
    }
    __device__ __forceinline__ int column(int unit) const { return unit == 0 ? 0 : split.head + (unit - 1) * E::kPer; }
    __device__ __forceinline__ int units() const { return split.pieces + 2; }
    // A unit's values, and how many there are; absent ones NaN, which largest() passes over: a unit of NaN alone is as low as
    // its elements.
    __device__ __forceinline__ int values(int unit, float (&z)[E::kPer]) const {
        if (unit > 0 && unit <= split.pieces) {
            E::values(__ldg(reinterpret_cast<const uint4 *>(p + split.head) + unit - 1), z);
            return E::kPer;
        }
        const int n = unit == 0 ? split.head : split.tail;
#pragma unroll
        for (int i = 0; i < E::kPer; ++i) z[i] = i < n ? E::value(p[column(unit) + i]) : not_a_number();
        return n;
    }
};

// The largest of a strip's units, by its largest value.
struct Best {
    uint32_t order = 0u;
    int unit = 0;
    __device__ __forceinline__ void offer(uint32_t o, int u) {
        if (o > order) order = o, unit = u;
    }
    __device__ __forceinline__ uint64_t key() const { return order ? key_of(order, unit) : 0u; }
};

template <int N>
__device__ __forceinline__ float largest(const float (&z)[N]) {  // NaN only if all are
    float top = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, z[i]);
    return top;
}

// WRITTEN: the kernel may write where the logits are, so they do not take the read-only path.
template <int TYPE, bool TOP, bool WRITTEN = false, int FLIGHT = kFlight>
__device__ __forceinline__ Sums take_strip(const Strip<TYPE> &s, float k, Best &best) {
    using E = Elem<TYPE>;
    Sums2 sums;
    sums.clear();
    auto take = [&](const float (&z)[E::kPer], float top, int unit) {
        sums.raise(top, k);
        sums.add(z, k);
        if (TOP) best.offer(order_of(top), unit);
    };
    float z[E::kPer];
    auto take_some = [&](int unit) {  // of the row's ends
        const int n = s.values(unit, z);
        const float top = largest(z);
#pragma unroll
        for (int i = 0; i < E::kPer; ++i) z[i] = i < n ? z[i] : minus_infinity();
        take(z, top, unit);
    };
    if (s.ends && s.t == 0 && s.split.head > 0) take_some(0);
    const uint4 *const q = reinterpret_cast<const uint4 *>(s.p + s.split.head);
    for (int at = s.first; at < s.end; at += FLIGHT * s.threads) {
        uint4 w[FLIGHT];
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i)
            if (at + i * s.threads < s.end) w[i] = WRITTEN ? q[at + i * s.threads] : __ldg(q + at + i * s.threads);
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            if (at + i * s.threads >= s.end) continue;
            E::values(w[i], z);
            take(z, E::largest(w[i]), at + i * s.threads + 1);
        }
    }
    if (s.ends && s.t == s.threads - 1 && s.split.tail > 0) take_some(s.units() - 1);
    return sums.all();
}

// ---- the largest: candidates in shared memory
struct Found {
    uint64_t *keys;
    int *count;
    int room;
    __device__ __forceinline__ void add(uint64_t key) const {
        const int at = atomicAdd(count, 1);  // in any order: they are ranked
        if (at < room) keys[at] = key;
    }
};
// A unit's elements at or above the bound, if the unit is.
template <int TYPE>
__device__ __forceinline__ void offer_unit(const Strip<TYPE> &s, int unit, uint64_t bound, const Found &found) {
    float z[Elem<TYPE>::kPer];
    const int n = s.values(unit, z);
    if (n == 0 || key_of(order_of(largest(z)), unit) < bound) return;
#pragma unroll
    for (int i = 0; i < Elem<TYPE>::kPer; ++i) {
        const uint32_t o = order_of(z[i]);
        if (i < n && o >= (uint32_t)(bound >> 32)) found.add(key_of(o, s.column(unit) + i));
    }
}
// The strip of thread t again, by itself or (lanes = 32) by a warp.
template <int TYPE>
__device__ __forceinline__ void offer_strip(const Strip<TYPE> &s, int t, int lane, int lanes, uint64_t bound, const Found &found) {
    if (s.ends && t == 0 && lane == 0 && s.split.head > 0) offer_unit(s, 0, bound, found);
    for (int at = s.first - s.t + t + lane * s.threads; at < s.end; at += lanes * s.threads) offer_unit(s, at + 1, bound, found);
    if (s.ends && t == s.threads - 1 && lane == 0 && s.split.tail > 0) offer_unit(s, s.units() - 1, bound, found);
}
// The strip's largest unit below `limit`.
template <int TYPE>
__device__ __forceinline__ uint64_t next_unit(const Strip<TYPE> &s, uint64_t limit) {
    uint64_t best = 0u;
    auto look = [&](int unit) {
        float z[Elem<TYPE>::kPer];
        const uint64_t key = s.values(unit, z) ? key_of(order_of(largest(z)), unit) : 0u;
        if (key < limit && key > best) best = key;
    };
    if (s.ends && s.t == 0) look(0);
    for (int at = s.first; at < s.end; at += s.threads) look(at + 1);
    if (s.ends && s.t == s.threads - 1) look(s.units() - 1);
    return best;
}
// Where there was no room for all: the strip's largest element below `limit`.
template <int TYPE>
__device__ __forceinline__ uint64_t next_below(const Strip<TYPE> &s, uint64_t limit) {
    uint64_t best = 0u;
    auto look = [&](int unit) {
        float z[Elem<TYPE>::kPer];
        const int n = s.values(unit, z);
        for (int i = 0; i < n; ++i) {
            const uint64_t key = key_of(order_of(z[i]), s.column(unit) + i);
            if (key < limit && key > best) best = key;
        }
    };
    if (s.ends && s.t == 0) look(0);
    for (int at = s.first; at < s.end; at += s.threads) look(at + 1);
    if (s.ends && s.t == s.threads - 1) look(s.units() - 1);
    return best;
}
__device__ __forceinline__ uint64_t warp_max(uint64_t key) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
    return ((uint64_t)hi << 32) | lo;
}
// How many of n keys are larger.
__device__ __forceinline__ int rank_of(uint64_t key, const uint64_t *keys, int n) {
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < n; ++i) rank += keys[i] > key ? 1 : 0;
    return rank;
}
// The key of a rank among the warp's; 0 if there is none.
__device__ __forceinline__ uint64_t ranked(uint64_t key, int rank, int which) {
    const uint32_t has = __ballot_sync(0xffffffffu, key != 0u && rank == which);
    return has ? __shfl_sync(0xffffffffu, key, __ffs(has) - 1) : 0u;
}

// l of a logit, from the row's sums.  By halves: the type's least value less a large one may be beyond fp32 where l is not.
__device__ __forceinline__ float logprob_of(float z, const Sums &x, float log_s, float inverse_t) {
    return x.m == minus_infinity() && x.s == 0.f ? minus_infinity() : fmaf((0.5f * z - 0.5f * x.m) * inverse_t, 2.f, -log_s);
}

// A row's results; `z` is its token's logit.
__device__ __forceinline__ void finish_row(const LogprobArgs &a, int64_t row, const Sums &x, int token, float z) {
    const bool empty = x.m == minus_infinity() && x.s == 0.f;
    const float log_s = logf(x.s);
    if (a.logprob)
        a.logprob[row] = token < 0 ? 0.f : token >= a.v ? not_a_number() : logprob_of(z, x, log_s, a.inverse_t);
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - x.w * kLn2 / x.s;
    if (a.lse) a.lse[row] = empty ? minus_infinity() : fmaf(x.m, a.inverse_t, log_s);
    if (a.sums) a.sums[row] = make_float2(x.m, x.s);
}
__device__ __forceinline__ void finish_top(const LogprobArgs &a, int64_t row, const Sums &x, uint64_t key, int rank) {
    a.top_logprob[row * a.top + rank] = logprob_of(value_of((uint32_t)(key >> 32)), x, logf(x.s), a.inverse_t);
    a.top_index[row * a.top + rank] = place_of(key);
}
template <int TYPE>
__device__ __forceinline__ float token_logit(const LogprobArgs &a, const uint8_t *row, int token) {
    using E = Elem<TYPE>;
    return token >= 0 && token < a.v ? E::value(reinterpret_cast<const typename E::T *>(row)[token]) : 0.f;
}

// Room for a warp's candidates: where fewer lanes than K have a piece, all elements are.
constexpr int kWarpRoom = 32 * 8 + 16;
constexpr int kTopOfMaxima = 20;  // 32768 x 1000: the 32 largest 186 us from 32 maxima (no room), 88 from 64
// Short rows: 2^lanes_log2 lanes to a row; fewer than a warp look for the largest one after another.
template <int TYPE, bool TOP>
__global__ void __launch_bounds__(kThreads) logprob_lanes_kernel(const __grid_constant__ LogprobArgs a) {
    __shared__ uint64_t keys[TOP ? kWarps : 1][kWarpRoom];
    __shared__ int counts[kWarps];
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> a.lanes_log2;
    const bool in = row < a.m;
    const uint8_t *const p = a.z + row * a.row_bytes;
    Best best;
    pdl_trigger();
    pdl_wait();
    const int token = in && a.tokens ? a.tokens[row] : -1;
    const float z = in ? token_logit<TYPE>(a, p, token) : 0.f;
    const Strip<TYPE> strip(p, in ? a.v : 0, lane, lanes, 0, 1);
    Sums sums = take_strip<TYPE, TOP>(strip, a.k, best);
    for (int d = lanes >> 1; d > 0; d >>= 1) {
        Sums o;
        o.m = __shfl_xor_sync(0xffffffffu, sums.m, d);
        o.s = __shfl_xor_sync(0xffffffffu, sums.s, d);
        o.w = __shfl_xor_sync(0xffffffffu, sums.w, d);
        sums.join(o, a.k);
    }
    if (in && lane == 0) finish_row(a, row, sums, token, z);
    if (TOP && a.lanes_log2 < 5) {  // the largest one after another
        uint64_t limit = ~0ull;
        for (int i = 0; i < a.top; ++i) {
            uint64_t key = next_below(strip, limit);
            for (int d = lanes >> 1; d > 0; d >>= 1) {
                const uint64_t other = __shfl_xor_sync(0xffffffffu, key, d);
                key = other > key ? other : key;
            }
            limit = key;
            if (in && lane == 0) finish_top(a, row, sums, key, i);
        }
        return;
    }
    if (!in) return;
    if constexpr (TOP) {
        const int warp = threadIdx.x / 32;
        const Found found{keys[warp], counts + warp, kWarpRoom};
        if (lane == 0) counts[warp] = 0;
        keys[warp][lane] = best.key();
        __syncwarp();
        uint64_t bound;
        if (a.top <= kTopOfMaxima) {
            bound = ranked(best.key(), rank_of(best.key(), keys[warp], 32), a.top - 1);
        } else {  // from the low end of 32 maxima much would be above it: of two pieces of each lane
            const uint64_t second = next_unit(strip, best.key());
            keys[warp][32 + lane] = second;
            __syncwarp();
            bound = max(ranked(best.key(), rank_of(best.key(), keys[warp], 64), a.top - 1), ranked(second, rank_of(second, keys[warp], 64), a.top - 1));
        }
        __syncwarp();
        if (best.key() && best.key() >= bound) offer_strip(strip, lane, 0, 1, bound, found);
        __syncwarp();
        const int n = counts[warp];
        if (n <= kWarpRoom) {
            for (int i = lane; i < n; i += 32) {
                const uint64_t key = keys[warp][i];
                const int rank = rank_of(key, keys[warp], n);
                if (rank < a.top) finish_top(a, row, sums, key, rank);
            }
        } else {
            uint64_t limit = ~0ull;
            for (int i = 0; i < a.top; ++i) {
                limit = warp_max(next_below(strip, limit));
                if (lane == 0) finish_top(a, row, sums, limit, i);
            }
        }
    }
}

// What a block leaves for the join: its sums and its largest keys, in order.
struct Joined {
    Sums sums;
    uint64_t key[kMostTop];
};
constexpr int kBlockRoom = 512;  // for candidates

// A row to a block, or, in a cluster, to its blocks.
template <int TYPE, bool TOP>
__global__ void __launch_bounds__(kThreads) logprob_block_kernel(const __grid_constant__ LogprobArgs a, int cluster) {
    __shared__ Sums warps[kWarps];
    __shared__ Joined blocks[kMostCluster];
    __shared__ Joined all;
    __shared__ uint64_t keys[TOP ? kBlockRoom : 1];
    __shared__ uint64_t bounds[kWarps][2];
    __shared__ int count;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int64_t row = blockIdx.x / (unsigned)cluster;
    const uint8_t *const p = a.z + row * a.row_bytes;
    Best best;
    if (cluster > 1) cluster_arrive();  // it has started
    pdl_trigger();
    pdl_wait();
    if (a.far && !is_far(a.far[row])) return;  // (without a cluster)
    const int token = a.tokens ? a.tokens[row] : -1;
    const float z = threadIdx.x == 0 ? token_logit<TYPE>(a, p, token) : 0.f;
    const Strip<TYPE> strip(p, a.v, threadIdx.x, kThreads, rank, cluster);
    Sums sums = take_strip<TYPE, TOP>(strip, a.k, best);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        Sums o;
        o.m = __shfl_xor_sync(0xffffffffu, sums.m, d);
        o.s = __shfl_xor_sync(0xffffffffu, sums.s, d);
        o.w = __shfl_xor_sync(0xffffffffu, sums.w, d);
        sums.join(o, a.k);
    }
    if (lane == 0) warps[warp] = sums;
    if constexpr (TOP) {
        // K pieces at or above it: as many of every warp whose lanes all have one, or all of one
        keys[threadIdx.x] = best.key();
        if (threadIdx.x == 0) count = 0;
        __syncwarp();
        const int mine = rank_of(best.key(), keys + 32 * warp, 32);
        const int full = max(1, min(kWarps, (strip.end - strip.first + (int)threadIdx.x) / 32));
        const uint64_t few = ranked(best.key(), mine, (a.top + full - 1) / full - 1), many = ranked(best.key(), mine, a.top - 1);
        if (lane == 0) bounds[warp][0] = warp < full ? few : ~0ull, bounds[warp][1] = many;
    }
    __syncwarp();
    if (cluster > 1) cluster_wait();
    __syncthreads();
    if (threadIdx.x == 0) {
        sums = warps[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) sums.join(warps[w], a.k);
        all.sums = sums;
    }
    if constexpr (TOP) {
        uint64_t few = bounds[0][0], bound = bounds[0][1];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) {
            few = min(few, bounds[w][0]);
            bound = max(bound, bounds[w][1]);
        }
        bound = max(bound, few);
        const Found found{keys, &count, kBlockRoom};
        const uint32_t again = __ballot_sync(0xffffffffu, best.key() && best.key() >= bound);
        int width = 4;  // lanes of a strip: a piece each, if it is short
        while (width < 32 && width * kThreads < strip.end - strip.first + (int)threadIdx.x) width *= 2;
        for (int i = lane / width; i < __popc(again); i += 32 / width)
            offer_strip(strip, 32 * warp + (int)__fns(again, 0, i + 1), lane % width, width, bound, found);
        __syncthreads();
        const int n = count;
        if (n <= kBlockRoom) {
            for (int i = threadIdx.x; i < n; i += kThreads) {
                const uint64_t key = keys[i];
                const int at = rank_of(key, keys, n);
                if (at < a.top) all.key[at] = key;
            }
        } else {  // many at or above every bound: one after another
            uint64_t limit = ~0ull;
            for (int i = 0; i < a.top; ++i) {
                const uint64_t best_of = warp_max(next_below(strip, limit));
                if (lane == 0) bounds[warp][i & 1] = best_of;
                __syncthreads();
                limit = bounds[0][i & 1];
                for (int w = 1; w < kWarps; ++w) limit = max(limit, bounds[w][i & 1]);
                if (threadIdx.x == 0) all.key[i] = limit;
            }
        }
    }
    __syncthreads();
    if (cluster > 1) {
        if (warp == 0) {
            const uint32_t to = cluster_addr(smem_u32(&blocks[rank]), 0);
            const Sums &x = all.sums;
            if (lane < 3) store_cluster(to + 4 * lane, __float_as_uint(lane == 0 ? x.m : lane == 1 ? x.s : x.w));
            if (TOP && lane < a.top) store_cluster(to + (uint32_t)offsetof(Joined, key) + 8 * lane, all.key[lane]);
        }
        __syncwarp();
        cluster_sync();
        if (rank != 0) return;
        if (threadIdx.x == 0) {
            sums = blocks[0].sums;
            for (int b = 1; b < cluster; ++b) sums.join(blocks[b].sums, a.k);
            all.sums = sums;
        }
        if constexpr (TOP) {
            const int n = cluster * a.top;
            const int b = threadIdx.x / a.top;
            uint64_t key = 0u;
            if ((int)threadIdx.x < n) key = keys[threadIdx.x] = blocks[b].key[threadIdx.x - b * a.top];
            __syncthreads();
            const int at = (int)threadIdx.x < n ? rank_of(key, keys, n) : n;
            if (at < a.top) all.key[at] = key;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) finish_row(a, row, all.sums, token, z);
    if (TOP && (int)threadIdx.x < a.top) finish_top(a, row, all.sums, all.key[threadIdx.x], threadIdx.x);
}

// ---------------------------------------------------------------- gradient
struct LogprobGradArgs {
    const uint8_t *z;
    uint8_t *dz;
    int64_t row_bytes, d_row_bytes;
    const int32_t *tokens;
    const float *lse, *entropy, *d_logprob, *d_entropy;
    int m, v;
    float k, inverse_t;  // log2(e) / T, 1 / T
    int lanes_log2;      // threads of a row, in a block
    const float2 *sums;  // far rows' maximum and S; null: the row's threads take them
};

// A row's maximum and S by its `lanes` threads (a power of two, to kThreads), of which this is t; in each of them.
template <int TYPE>
__device__ __forceinline__ float2 sums_again(const uint8_t *row, int v, float k, int t, int lanes) {
    __shared__ Sums warps[kWarps];
    const Strip<TYPE> strip(row, v, t, lanes, 0, 1);
    Best none;
    Sums sums = take_strip<TYPE, false, true, 1>(strip, k, none);
    const int lane = threadIdx.x & 31, width = min(lanes, 32);
    const uint32_t mask = (0xffffffffu >> (32 - width)) << (lane & ~(width - 1));
    for (int d = width >> 1; d > 0; d >>= 1) {
        Sums o;
        o.m = __shfl_xor_sync(mask, sums.m, d);
        o.s = __shfl_xor_sync(mask, sums.s, d);
        o.w = 0.f;
        sums.join(o, k);
    }
    if (lanes > 32) {
        if (lane == 0) warps[threadIdx.x / 32] = sums;
        switch ((int)threadIdx.x / lanes) {  // (by number: with one that is computed a block would hold all 16)
            case 0: asm volatile("bar.sync 1, %0;" ::"r"(lanes) : "memory"); break;
            case 1: asm volatile("bar.sync 2, %0;" ::"r"(lanes) : "memory"); break;
            case 2: asm volatile("bar.sync 3, %0;" ::"r"(lanes) : "memory"); break;
            default: asm volatile("bar.sync 4, %0;" ::"r"(lanes) : "memory");
        }
        const int first = (int)threadIdx.x / lanes * (lanes / 32);
        sums = warps[first];
        for (int w = 1; w < lanes / 32; ++w) sums.join(warps[first + w], k);
    }
    return make_float2(sums.m, sums.s);
}

// What a row's elements share.
struct RowGrad {
    float base, lse, inverse_t, dl, dh, dh_h;  // d_logprob, d_entropy, d_entropy * entropy; FAR: the maximum, and ln S as lse
    int token;
    bool empty;  // FAR, and of -infinity alone: nothing to change
    template <bool FAR>
    __device__ __forceinline__ float of(float z, int column) const {
        if (FAR && empty) return 0.f;
        const float l = fmaf(FAR ? z - base : z, inverse_t, -lse), p = exp2_f(l * kLog2E);
        float g = p == 0.f ? 0.f : -p * (dl + fmaf(dh, l, dh_h));
        if (column == token) g += dl;
        return g * inverse_t;
    }
};

// A row's gradient by `threads` threads, of which this is t.
template <int TYPE, bool FAR>
__device__ __forceinline__ void write_row(const RowGrad &g, const typename Elem<TYPE>::T *z, typename Elem<TYPE>::T *dz, int v, int t, int threads) {
    using E = Elem<TYPE>;
    // pieces where both rows lie alike on 16 bytes, else elements
    const bool alike = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15u) == 0;
    Split s = split_row<TYPE>(z, v);
    if (!alike) s = {v, 0, 0};
    for (int e = t; e < s.head + s.tail; e += threads) {
        const int column = e < s.head ? e : s.pieces * E::kPer + e;
        dz[column] = E::stored(g.of<FAR>(E::value(z[column]), column));
    }
    const uint4 *const q = reinterpret_cast<const uint4 *>(z + s.head);
    uint4 *const to = reinterpret_cast<uint4 *>(dz + s.head);
    for (int at = t; at < s.pieces; at += kFlight * threads) {
        uint4 w[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (at + i * threads < s.pieces) w[i] = q[at + i * threads];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (at + i * threads >= s.pieces) continue;
            float v[E::kPer];
            E::values(w[i], v);
#pragma unroll
            for (int j = 0; j < E::kPer; ++j) v[j] = g.of<FAR>(v[j], s.head + (at + i * threads) * E::kPer + j);
            to[at + i * threads] = E::stored(v);
        }
    }
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads, 5) logprob_grad_kernel(const __grid_constant__ LogprobGradArgs a) {
    using T = typename Elem<TYPE>::T;
    const int lanes = 1 << a.lanes_log2, threads = lanes * gridDim.y;
    const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> a.lanes_log2;
    const int lane = threadIdx.x & (lanes - 1), t = blockIdx.y * lanes + lane;
    pdl_trigger();
    pdl_wait();
    if (row >= a.m) return;
    const T *const z = reinterpret_cast<const T *>(a.z + row * a.row_bytes);
    T *const dz = reinterpret_cast<T *>(a.dz + row * a.d_row_bytes);
    RowGrad g;
    g.lse = a.lse[row];
    g.inverse_t = a.inverse_t;
    g.token = a.tokens ? a.tokens[row] : -1;
    g.dl = a.d_logprob && g.token >= 0 && g.token < a.v ? a.d_logprob[row] : 0.f;
    g.dh = a.d_entropy ? a.d_entropy[row] : 0.f;
    g.dh_h = a.d_entropy ? g.dh * a.entropy[row] : 0.f;
    if (!is_far(g.lse)) return write_row<TYPE, false>(g, z, dz, a.v, t, threads);
    const float2 x = a.sums ? a.sums[row] : sums_again<TYPE>(reinterpret_cast<const uint8_t *>(z), a.v, a.k, lane, lanes);
    g.base = x.x;
    g.lse = logf(x.y);
    g.empty = x.x == minus_infinity() && x.y == 0.f;
    write_row<TYPE, true>(g, z, dz, a.v, t, threads);
}

template <int TYPE, bool TOP>
cudaError_t run(LogprobArgs &a, int sms, cudaStream_t s) {
    const int pieces = a.v / Elem<TYPE>::kPer;
    // A few lanes to a row where rows are many: a warp waits for no other.  Lanes and a block to a row, the sums alone:
    // 32768 x 1000 21.8 and 112 us, 8192 x 32768 99 and 105, 2000 x 8192 12.8 and 12.3, 64 x 2048 3.5 and 2.8.  With the 8
    // largest: 8192 x 8192 59 and 90, 8192 x 16384 116 and 114, 600 x 4096 10.2 and 9.3; the 32 largest: 8192 x 8192 94 and
    // 109, 8192 x 16384 186 and 143.
    const int most = !TOP ? 4096 : a.top <= kTopOfMaxima ? 2048 : 1024;
    if (pieces <= 64 || (pieces <= most && (TOP ? 4 : 2) * (int64_t)pieces <= a.m)) {
        while (a.lanes_log2 < 5 && (2 << a.lanes_log2) < pieces) ++a.lanes_log2;
        // The largest one after another or with a warp to a row: 20000 rows of 8, top 5, 4.9 and 19.9 us; 32768 of 64, top 5,
        // 14.8 and 32.5; 20000 of 33 (fp32), top 8, 20.6 and 22.6, top 16 37.8 and 27.8; 32768 of 200, top 2, 25.5 and 30.6, top 5
        // 47.9 and 32.2.
        if (TOP && a.top * a.v > 320) a.lanes_log2 = 5;
        const int64_t rows = kThreads >> a.lanes_log2;
        return launch_pdl(logprob_lanes_kernel<TYPE, TOP>, dim3((unsigned)((a.m + rows - 1) / rows)), dim3(kThreads), 0, s, a);
    }
    // blocks for every SM, each with a round of pieces at least
    int cluster = 1;
    while (cluster < kMostCluster && (int64_t)a.m * cluster < 2 * sms && pieces >= 2 * cluster * kThreads * kFlight) cluster *= 2;
    if (cluster == 1)
        return launch_pdl(logprob_block_kernel<TYPE, TOP>, dim3((unsigned)a.m), dim3(kThreads), 0, s, a, cluster);
    return launch_cluster(logprob_block_kernel<TYPE, TOP>, dim3((unsigned)(a.m * cluster)), dim3(kThreads), 0, cluster, s, a, cluster);
}
template <int TYPE>
cudaError_t run(LogprobArgs &a, int sms, cudaStream_t s) {
    return a.top ? run<TYPE, true>(a, sms, s) : run<TYPE, false>(a, sms, s);
}

}  // namespace

cudaError_t launch_logprobs(const emtk_logprobs_args &p, int sms, cudaStream_t s) {
    if (p.m == 0) return cudaSuccess;
    LogprobArgs a{};
    a.z = static_cast<const uint8_t *>(p.logits.d);
    a.row_bytes = p.logits.ld * (p.type == EMTK_TYPE_F32 ? 4 : 2);
    a.tokens = p.tokens;
    a.logprob = p.logprob;
    a.entropy = p.entropy;
    a.lse = p.lse;
    a.top_logprob = p.top_logprob;
    a.top_index = p.top_index;
    a.m = p.m;
    a.v = p.v;
    a.top = p.top;
    a.inverse_t = 1.f / p.temperature;
    a.k = kLog2E * a.inverse_t;
    if (p.type == EMTK_TYPE_F32) return run<EMTK_TYPE_F32>(a, sms, s);
    return p.type == EMTK_TYPE_F16 ? run<EMTK_TYPE_F16>(a, sms, s) : run<EMTK_TYPE_BF16>(a, sms, s);
}

cudaError_t launch_logprobs_grad(const emtk_logprobs_grad_args &p, const emtk_nn *nn, cudaStream_t s) {
    if (p.m == 0 || p.v == 0) return cudaSuccess;
    LogprobGradArgs a{};
    const int elem = p.type == EMTK_TYPE_F32 ? 4 : 2;
    a.z = static_cast<const uint8_t *>(p.logits.d);
    a.dz = static_cast<uint8_t *>(p.d_logits.d);
    a.row_bytes = p.logits.ld * elem;
    a.d_row_bytes = p.d_logits.ld * elem;
    a.tokens = p.tokens;
    a.lse = p.lse;
    a.entropy = p.entropy;
    a.d_logprob = p.d_logprob;
    a.d_entropy = p.d_entropy;
    a.m = p.m;
    a.v = p.v;
    a.inverse_t = 1.f / p.temperature;
    a.k = kLog2E * a.inverse_t;
    const int sms = nn->sm_count;
    const int64_t pieces = std::max<int64_t>(1, (int64_t)p.v * elem / 16);
    // Up to 8 pieces a thread, as long as threads are left for the SMs: 32768 x 1000 with 1, 4 and 8 pieces a thread 49, 25 and
    // 23 us, 4000 x 1000 with 1, 2 and 8 5.3, 4.0 and 4.6, 64 x 1000 1.6, 1.8 and 2.8.
    int each = 1;
    while (each < 8 && p.m * pieces >= 2 * each * 1024ll * sms) each *= 2;
    while (a.lanes_log2 < 8 && ((int64_t)each << a.lanes_log2) < pieces) ++a.lanes_log2;
    const int64_t rows = kThreads >> a.lanes_log2;
    // long rows are cut where there are too few for every SM
    const int64_t blocks = (p.m + rows - 1) / rows, rounds = (pieces + kThreads * kFlight - 1) / (kThreads * kFlight);
    const unsigned cut = (unsigned)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(rounds, 65535), 2ll * kCutRows * sms / blocks));
    void (*kernel)(const LogprobGradArgs) = p.type == EMTK_TYPE_F32   ? logprob_grad_kernel<EMTK_TYPE_F32>
                                            : p.type == EMTK_TYPE_F16 ? logprob_grad_kernel<EMTK_TYPE_F16>
                                                                      : logprob_grad_kernel<EMTK_TYPE_BF16>;
    if (cut > 1 && a.dz == a.z) {  // a block would write while another of the row still reads
        LogprobArgs f{};
        f.z = a.z;
        f.row_bytes = a.row_bytes;
        f.m = p.m;
        f.v = p.v;
        f.k = a.k;
        f.inverse_t = a.inverse_t;
        f.far = p.lse;
        a.sums = f.sums = nn->far_sums;
        void (*sums)(const LogprobArgs, int) = p.type == EMTK_TYPE_F32   ? logprob_block_kernel<EMTK_TYPE_F32, false>
                                               : p.type == EMTK_TYPE_F16 ? logprob_block_kernel<EMTK_TYPE_F16, false>
                                                                         : logprob_block_kernel<EMTK_TYPE_BF16, false>;
        const cudaError_t e = launch_pdl(sums, dim3((unsigned)p.m), dim3(kThreads), 0, s, f, 1);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, dim3((unsigned)blocks, cut), dim3(kThreads), 0, s, a);
}

}  // namespace emtk
