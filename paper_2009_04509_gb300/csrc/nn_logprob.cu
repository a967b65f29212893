// Log probabilities, entropy and the largest of a row of logits, and their gradient.
//
// One pass: with the running maximum M, S = sum exp((z - M) / T) and
// W = sum exp((z - M) / T) (z - M) / T,
//   l_j = (z_j - M) / T - ln S;   entropy = ln S - W / S;
// when the maximum rises by d (in units of T), S becomes S exp(-d) and W exp(-d) (W - d S).
// Two runs' triples join the same way.  HBM bounds large calls (one read of the logits;
// the gradient one read and one write), the call small ones.
//
// A row goes to a few lanes, to a block of threads, or, where rows are few and long, to a
// cluster of blocks that join through shared memory.  Rows start anywhere: their aligned
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
constexpr int kFlight = 4;  // pieces of a thread in flight

constexpr float kFar = -1e4f;  // an exponent whose power is 0, in the place of -infinity where that would meet a 0

__device__ __forceinline__ float minus_infinity() { return __int_as_float(0xff800000); }

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
    __device__ __forceinline__ void add(float z, float k) {
        const float base = m == minus_infinity() ? 0.f : m;
        const float d = (z - base) * k, e = exp2_f(d);
        s += e;
        w = fmaf(e, fmaxf(d, kFar), w);
    }
    __device__ __forceinline__ void join(Sums o, float k) {
        const float top = fmaxf(m, o.m);
        raise(top, k);
        o.raise(top, k);
        s += o.s;
        w += o.w;
    }
};

// Order of logits, and the lowest index first among equals; NaN is the least.  Never 0.
__device__ __forceinline__ uint64_t key_of(float z, int column) {
    const uint32_t b = __float_as_uint(z + 0.f);  // -0 and 0 are equal
    const uint32_t u = z != z ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return ((uint64_t)u << 32) | (uint32_t)~column;
}
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    if (u == 0u) return __int_as_float(0x7fffffff);
    return __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint64_t warp_max(uint64_t key) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
    return ((uint64_t)hi << 32) | lo;
}

// A warp's largest keys, descending over its lanes; 0: none yet.
struct TopList {
    uint64_t mine, least;  // this lane's, and the one at `top`, which all know
    float bar;             // value of `least`; NaN while there is none
    __device__ __forceinline__ void clear() { mine = least = 0u, bar = __int_as_float(0x7fffffff); }
    __device__ __forceinline__ void insert(uint64_t key, int top, int lane) {
        const int at = __popc(__ballot_sync(0xffffffffu, mine > key));
        const uint64_t up = __shfl_up_sync(0xffffffffu, mine, 1);
        mine = lane < at ? mine : lane == at ? key : up;
        least = __shfl_sync(0xffffffffu, mine, top - 1);
        bar = least ? value_of(least) : __int_as_float(0x7fffffff);
    }
    // N values of each lane, the first `valid` of them from `column` on.
    template <int N>
    __device__ __forceinline__ void push(const float (&z)[N], int valid, int column, int top, int lane) {
        bool some = false;
#pragma unroll
        for (int i = 0; i < N; ++i) some = some || (i < valid && !(z[i] < bar));
        if (!__any_sync(0xffffffffu, some)) return;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t key = i < valid ? key_of(z[i], column + i) : 0u;
            uint32_t mask = __ballot_sync(0xffffffffu, key > least);
            while (mask) {
                const int from = __ffs(mask) - 1;
                insert(__shfl_sync(0xffffffffu, key, from), top, lane);
                mask &= mask - 1;
                mask &= __ballot_sync(0xffffffffu, key > least);
            }
        }
    }
};

struct LogprobArgs {
    const uint8_t *z;
    int64_t row_bytes;
    const int32_t *tokens;
    float *logprob, *entropy, *lse, *top_logprob;
    int32_t *top_index;
    int m, v, top;
    float k, inverse_t;  // log2(e) / T, 1 / T
    int lanes_log2;      // of a row, in lanes_kernel
};

// The row's logits that thread `t` of `threads` takes, part `part` of `parts` of the row.
// All threads of a warp run this together.
template <int TYPE, bool TOP>
__device__ __forceinline__ void take_row(const LogprobArgs &a, const uint8_t *row, bool in, int t, int threads, int part,
                                         int parts, Sums &sums, TopList &list) {
    using E = Elem<TYPE>;
    const typename E::T *const p = reinterpret_cast<const typename E::T *>(row);
    const Split s = split_row<TYPE>(row, in ? a.v : 0);
    const int lane = threadIdx.x & 31;
    // a part's pieces; the elements around them go with the first
    const int each = (s.pieces + parts - 1) / parts, begin = part * each, end = min(begin + each, s.pieces);
    const int singles = part == 0 ? s.head + s.tail : 0;
    for (int e = t; TOP ? __any_sync(0xffffffffu, e < singles) : e < singles; e += threads) {
        const int column = e < s.head ? e : s.pieces * E::kPer + e;
        float z[1] = {0.f};
        if (e < singles) {
            z[0] = E::value(p[column]);
            sums.raise(z[0], a.k);
            sums.add(z[0], a.k);
        }
        if (TOP) list.push(z, e < singles ? 1 : 0, column, a.top, lane);
    }
    const uint4 *const q = reinterpret_cast<const uint4 *>(p + s.head);
    for (int at = begin + t; TOP ? __any_sync(0xffffffffu, at < end) : at < end; at += kFlight * threads) {
        uint4 w[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (at + i * threads < end) w[i] = __ldg(q + at + i * threads);
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const bool has = at + i * threads < end;
            float z[E::kPer];
            if (has) {
                E::values(w[i], z);
                float top = z[0];
#pragma unroll
                for (int j = 1; j < E::kPer; ++j) top = fmaxf(top, z[j]);
                sums.raise(top, a.k);
#pragma unroll
                for (int j = 0; j < E::kPer; ++j) sums.add(z[j], a.k);
            } else {
#pragma unroll
                for (int j = 0; j < E::kPer; ++j) z[j] = 0.f;
            }
            if (TOP) list.push(z, has ? E::kPer : 0, s.head + (at + i * threads) * E::kPer, a.top, lane);
        }
    }
}

// l of a logit, from the row's sums.
__device__ __forceinline__ float logprob_of(float z, const Sums &x, float log_s, float inverse_t) {
    return x.m == minus_infinity() && x.s == 0.f ? minus_infinity() : (z - x.m) * inverse_t - log_s;
}

// A row's results; `z` is its token's logit.
__device__ __forceinline__ void finish_row(const LogprobArgs &a, int64_t row, const Sums &x, int token, float z) {
    const bool empty = x.m == minus_infinity() && x.s == 0.f;
    const float log_s = logf(x.s);
    if (a.logprob)
        a.logprob[row] = token < 0 ? 0.f : token >= a.v ? __int_as_float(0x7fffffff) : logprob_of(z, x, log_s, a.inverse_t);
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - x.w * kLn2 / x.s;
    if (a.lse) a.lse[row] = empty ? minus_infinity() : fmaf(x.m, a.inverse_t, log_s);
}
__device__ __forceinline__ void finish_top(const LogprobArgs &a, int64_t row, const Sums &x, uint64_t key, int lane) {
    if (lane >= a.top) return;
    a.top_logprob[row * a.top + lane] = logprob_of(value_of(key), x, logf(x.s), a.inverse_t);
    a.top_index[row * a.top + lane] = (int)~(uint32_t)key;
}
template <int TYPE>
__device__ __forceinline__ float token_logit(const LogprobArgs &a, const uint8_t *row, int token) {
    using E = Elem<TYPE>;
    return token >= 0 && token < a.v ? E::value(reinterpret_cast<const typename E::T *>(row)[token]) : 0.f;
}

// Short rows: 2^lanes_log2 lanes to a row (a warp where the largest are wanted).
template <int TYPE, bool TOP>
__global__ void __launch_bounds__(kThreads) logprob_lanes_kernel(const __grid_constant__ LogprobArgs a) {
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> a.lanes_log2;
    const bool in = row < a.m;
    const uint8_t *const p = a.z + row * a.row_bytes;
    Sums sums;
    TopList list;
    sums.clear();
    list.clear();
    pdl_trigger();
    pdl_wait();
    const int token = in && a.tokens ? a.tokens[row] : -1;
    const float z = in ? token_logit<TYPE>(a, p, token) : 0.f;
    take_row<TYPE, TOP>(a, p, in, lane, lanes, 0, 1, sums, list);
    for (int d = lanes >> 1; d > 0; d >>= 1) {
        Sums o;
        o.m = __shfl_xor_sync(0xffffffffu, sums.m, d);
        o.s = __shfl_xor_sync(0xffffffffu, sums.s, d);
        o.w = __shfl_xor_sync(0xffffffffu, sums.w, d);
        sums.join(o, a.k);
    }
    if (!in) return;
    if (lane == 0) finish_row(a, row, sums, token, z);
    if (TOP) finish_top(a, row, sums, list.mine, lane);
}

// What a block leaves for the join: its sums and its largest keys.
struct Joined {
    Sums sums;
    uint64_t key[kMostTop];
};

// The largest `top` of up to 32 descending lists, key i in lane i: each round takes the
// largest head.
__device__ __forceinline__ uint64_t merge_lists(const uint64_t *mine, int top, int lane) {
    uint64_t out = 0u, head = mine ? mine[0] : 0u;
    int at = 0;
    for (int i = 0; i < top; ++i) {
        const uint64_t best = warp_max(head);
        if (lane == i) out = best;
        if (best && head == best) head = ++at < top ? mine[at] : 0u;  // keys are unlike: they hold the column
    }
    return out;
}

// A row to a block, or, in a cluster, to its blocks.
template <int TYPE, bool TOP>
__global__ void __launch_bounds__(kThreads) logprob_block_kernel(const __grid_constant__ LogprobArgs a, int cluster) {
    __shared__ Joined warps[kWarps];
    __shared__ Joined blocks[kMostCluster];
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int64_t row = blockIdx.x / (unsigned)cluster;
    const uint8_t *const p = a.z + row * a.row_bytes;
    Sums sums;
    TopList list;
    sums.clear();
    list.clear();
    if (cluster > 1) cluster_arrive();  // it has started
    pdl_trigger();
    pdl_wait();
    const int token = a.tokens ? a.tokens[row] : -1;
    const float z = threadIdx.x == 0 ? token_logit<TYPE>(a, p, token) : 0.f;
    take_row<TYPE, TOP>(a, p, true, threadIdx.x, kThreads, rank, cluster, sums, list);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        Sums o;
        o.m = __shfl_xor_sync(0xffffffffu, sums.m, d);
        o.s = __shfl_xor_sync(0xffffffffu, sums.s, d);
        o.w = __shfl_xor_sync(0xffffffffu, sums.w, d);
        sums.join(o, a.k);
    }
    if (lane == 0) warps[warp].sums = sums;
    if (TOP && lane < a.top) warps[warp].key[lane] = list.mine;
    __syncwarp();
    if (cluster > 1) cluster_wait();
    __syncthreads();
    uint64_t key = 0u;
    if (warp == 0) {
        sums = warps[0].sums;
#pragma unroll
        for (int w = 1; w < kWarps; ++w) sums.join(warps[w].sums, a.k);
        if (TOP) key = merge_lists(lane < kWarps ? warps[lane].key : nullptr, a.top, lane);
    }
    if (cluster > 1) {
        if (warp == 0) {
            const uint32_t to = cluster_addr(smem_u32(&blocks[rank]), 0);
            if (lane < 3) store_cluster(to + 4 * lane, __float_as_uint(lane == 0 ? sums.m : lane == 1 ? sums.s : sums.w));
            if (TOP && lane < a.top) store_cluster(to + (uint32_t)offsetof(Joined, key) + 8 * lane, key);
        }
        __syncwarp();
        cluster_sync();
        if (rank != 0) return;
        if (warp == 0) {
            sums = blocks[0].sums;
            for (int b = 1; b < cluster; ++b) sums.join(blocks[b].sums, a.k);
            if (TOP) key = merge_lists(lane < cluster ? blocks[lane].key : nullptr, a.top, lane);
        }
    }
    if (threadIdx.x == 0) finish_row(a, row, sums, token, z);
    if (TOP && warp == 0) finish_top(a, row, sums, key, lane);
}

// ---------------------------------------------------------------- gradient
struct LogprobGradArgs {
    const uint8_t *z;
    uint8_t *dz;
    int64_t row_bytes, d_row_bytes;
    const int32_t *tokens;
    const float *lse, *entropy, *d_logprob, *d_entropy;
    int m, v;
    float inverse_t;
    int lanes_log2;  // threads of a row
};

// What a row's elements share.
struct RowGrad {
    float lse, inverse_t, dl, dh, dh_h;  // d_logprob, d_entropy, d_entropy * entropy
    int token;
    __device__ __forceinline__ float of(float z, int column) const {
        const float l = fmaf(z, inverse_t, -lse), p = exp2_f(l * kLog2E);
        float g = p == 0.f ? 0.f : -p * (dl + fmaf(dh, l, dh_h));
        if (column == token) g += dl;
        return g * inverse_t;
    }
};

template <int TYPE>
__global__ void __launch_bounds__(kThreads) logprob_grad_kernel(const __grid_constant__ LogprobGradArgs a) {
    using E = Elem<TYPE>;
    using T = typename E::T;
    const int lanes = 1 << a.lanes_log2, threads = lanes * gridDim.y;
    const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> a.lanes_log2;
    const int t = blockIdx.y * lanes + (threadIdx.x & (lanes - 1));
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
    const bool empty = g.lse == minus_infinity();  // nothing to change
    // pieces where both rows lie alike on 16 bytes, else elements
    const bool alike = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15u) == 0;
    Split s = split_row<TYPE>(z, a.v);
    if (!alike) s = {a.v, 0, 0};
    for (int e = t; e < s.head + s.tail; e += threads) {
        const int column = e < s.head ? e : s.pieces * E::kPer + e;
        dz[column] = E::stored(empty ? 0.f : g.of(E::value(z[column]), column));
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
            for (int j = 0; j < E::kPer; ++j)
                v[j] = empty ? 0.f : g.of(v[j], s.head + (at + i * threads) * E::kPer + j);
            to[at + i * threads] = E::stored(v);
        }
    }
}

template <int TYPE, bool TOP>
cudaError_t run(LogprobArgs &a, int sms, cudaStream_t s) {
    const int pieces = a.v / Elem<TYPE>::kPer;
    if (pieces <= 256) {  // up to 8 pieces a lane
        a.lanes_log2 = TOP ? 5 : 0;
        while (a.lanes_log2 < 5 && (2 << a.lanes_log2) < pieces) ++a.lanes_log2;
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

cudaError_t launch_logprobs_grad(const emtk_logprobs_grad_args &p, int sms, cudaStream_t s) {
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
    const int64_t pieces = std::max(1, p.v * elem / 16);
    while (a.lanes_log2 < 8 && (1 << a.lanes_log2) < pieces) ++a.lanes_log2;
    const int64_t rows = kThreads >> a.lanes_log2;
    // long rows are cut where there are too few for every SM
    const int64_t blocks = (p.m + rows - 1) / rows, rounds = (pieces + kThreads * kFlight - 1) / (kThreads * kFlight);
    const unsigned cut = (unsigned)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(rounds, 65535), 8ll * sms / blocks));
    void (*kernel)(const LogprobGradArgs) = p.type == EMTK_TYPE_F32   ? logprob_grad_kernel<EMTK_TYPE_F32>
                                            : p.type == EMTK_TYPE_F16 ? logprob_grad_kernel<EMTK_TYPE_F16>
                                                                      : logprob_grad_kernel<EMTK_TYPE_BF16>;
    return launch_pdl(kernel, dim3((unsigned)blocks, cut), dim3(kThreads), 0, s, a);
}

}  // namespace emtk
