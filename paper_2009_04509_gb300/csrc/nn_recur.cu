// The gated linear recurrence along sequences, and its gradients.
//
//   b = 1 / (1 + exp(f));  h_t = h_(t-1) + b_t (x_t - h_(t-1));  y = act(o) h
//
// A run of steps maps the state before it to the one after it, linearly: h becomes H + A h,
// with H the state that the run makes of 0 and A = prod(1 - b).  A factor is held as q:
// itself where it is below a half, else as its complement with the sign changed, A - 1, so
// that neither what is kept for long nor what is nearly forgotten loses its low bits: at
// f = 8 a rounding of 1 - b in fp32 alone is 10^-4 of the state it settles to.
//
// A block takes 32 columns and goes along a sequence in tiles of 128 steps: each half
// warp a run of 8 steps, two columns to a lane.  The runs' (q, H) meet in shared memory, each
// half warp joins those before its own and goes over its 8 steps once more, from
// registers: everything is read once and written once.  Where columns and sequences are
// too few for the SMs, a cluster of blocks takes neighbouring tiles of a sequence and
// exchanges its tiles' (q, H) through shared memory.  Orders are fixed: the same call gives
// the same bits.
//
// Backwards, g_t = u_t + (1 - b_(t+1)) g_(t+1) with u = act(o) dy: passing p = (1 - b) g down,
// a run makes p of R + A p, with the same A.  A tile's states come from the one
// before it, which the forward pass kept.
//
// HBM bounds it: 8 bytes a value forward, 14 backward (16 bits, with o).
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_math.cuh"
#include "nn_ptx.cuh"

namespace emtk {
namespace {

constexpr int kCols = 32, kRuns = 16, kLen = 8, kTile = kRuns * kLen, kThreads = 16 * kRuns;
constexpr int kMostCluster = 8;
constexpr int kShort = 8;  // steps up to which a thread takes a whole sequence
static_assert(kTile == EMTK_RECURRENCE_STEP, "states are kept once a tile");

struct Plane {  // a 16-bit matrix
    uint8_t *p;
    int64_t row_bytes;
};
Plane plane_of(const emtk_matrix &m) { return {static_cast<uint8_t *>(m.d), 2 * m.ld}; }

struct Sequences {
    const int32_t *offsets;
    int rows, n, seqs, length;  // length: of each, without offsets
    __device__ __forceinline__ void rows_of(int s, int &r0, int &r1) const {
        if (offsets) {
            r0 = min(max(__ldg(offsets + s), 0), rows);
            r1 = min(max(__ldg(offsets + s + 1), r0), rows);
        } else {
            r0 = s * length;
            r1 = r0 + length;
        }
    }
};

struct RecurArgs {
    Plane f, x, o, y;
    Sequences at;
    const float *state;
    float *last, *states;
    int col_tiles, words;  // words: every row starts on 4 bytes
};
struct RecurGradArgs {
    Plane dy, f, x, o, df, dx, d_o;
    Sequences at;
    const float *states, *d_last;
    float *d_state;
    int col_tiles, words;
};

// Two neighbouring columns, of which `valid` exist.
__device__ __forceinline__ uint32_t load_pair(const Plane &a, int64_t r, int c, int valid, bool words) {
    const uint16_t *const p = reinterpret_cast<const uint16_t *>(a.p + r * a.row_bytes) + c;
    if (words && valid == 2) return __ldg(reinterpret_cast<const uint32_t *>(p));
    uint32_t v = 0;
    if (valid > 0) v = __ldg(p);
    if (valid > 1) v |= (uint32_t)__ldg(p + 1) << 16;
    return v;
}
__device__ __forceinline__ void store_pair(const Plane &a, int64_t r, int c, int valid, bool words, uint32_t v) {
    uint16_t *const p = reinterpret_cast<uint16_t *>(a.p + r * a.row_bytes) + c;
    if (words && valid == 2) {
        *reinterpret_cast<uint32_t *>(p) = v;
        return;
    }
    if (valid > 0) p[0] = (uint16_t)v;
    if (valid > 1) p[1] = (uint16_t)(v >> 16);
}
template <bool F16>
__device__ __forceinline__ float half_of(uint32_t w, int which) {
    return which ? (F16 ? from16<F16>(w >> 16) : __uint_as_float(w & 0xffff0000u)) : from16<F16>(F16 ? w & 0xffffu : w);
}
// fp32 states [..][n]
__device__ __forceinline__ void load_state(const float *p, int64_t row, int n, int c, int valid, float (&v)[2]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) v[j] = p && j < valid ? p[row * n + c + j] : 0.f;
}
__device__ __forceinline__ void store_state(float *p, int64_t row, int n, int c, int valid, const float (&v)[2]) {
    if (!p) return;
#pragma unroll
    for (int j = 0; j < 2; ++j)
        if (j < valid) p[row * n + c + j] = v[j];
}

// Factors held as q (above); -0 is the complement 0.
__device__ __forceinline__ bool is_complement(float q) { return __float_as_int(q) < 0; }
// a step's: of exp(f), beyond 80 of which 1 - a is 0 already
__device__ __forceinline__ float factor_of(float f) {
    const float e = exp_f(f > 80.f ? 80.f : f), b = reciprocal_f(1.f + e);
    return e > 1.f ? -b : e * b;
}
__device__ __forceinline__ float times(float q, float v) { return fmaf(q, v, is_complement(q) ? v : 0.f); }  // a v
__device__ __forceinline__ float complement(float q) { return is_complement(q) ? -q : 1.f - q; }            // 1 - a
// a h + (1 - a) x
__device__ __forceinline__ float step(float q, float h, float x) { return fmaf(q, h - x, is_complement(q) ? h : x); }
// of a run, from its product and its complement
__device__ __forceinline__ float factor_of(float product, float complement) { return complement < 0.5f ? -complement : product; }
__device__ __forceinline__ float product_of(float p, float q) {  // of two runs
    if (!is_complement(p) || !is_complement(q)) return is_complement(p) ? times(p, q) : times(q, p);
    const float c = fmaf(-p, 1.f + q, -q);  // both complements: 1 - (1 - c1)(1 - c2)
    return c < 0.5f ? -c : 1.f - c;
}

// Runs of two columns: (q0, H0, q1, H1).
__device__ __forceinline__ void then(float (&state)[2], const float4 &run) {
    state[0] = run.y + times(run.x, state[0]);
    state[1] = run.w + times(run.z, state[1]);
}
__device__ __forceinline__ void join(float4 &a, const float4 &b) {  // a, then b
    a.y = b.y + times(b.x, a.y);
    a.w = b.w + times(b.z, a.w);
    a.x = product_of(a.x, b.x);
    a.z = product_of(a.z, b.z);
}

// The cluster's tiles of this round: each block's run is written to every block.
__device__ __forceinline__ void share(float4 (*slots)[16], const float4 &run, int rank, int cluster, int lane) {
    const uint32_t mine = smem_u32(&slots[rank][lane]);
    for (int other = 0; other < cluster; ++other) {
        const uint32_t to = cluster_addr(mine, other);
        store_cluster(to, __float_as_uint(run.x));
        store_cluster(to + 4, __float_as_uint(run.y));
        store_cluster(to + 8, __float_as_uint(run.z));
        store_cluster(to + 12, __float_as_uint(run.w));
    }
}

// A half warp's run from state 0, and its steps' factors; steps from `count` on change nothing.
template <bool F16>
__device__ __forceinline__ float4 local_run(const uint32_t (&wf)[kLen], const uint32_t (&wx)[kLen], int count,
                                            float (&q)[kLen][2]) {
    float h[2] = {0.f, 0.f}, product[2] = {1.f, 1.f}, rest[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kLen; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            q[i][j] = i < count ? factor_of(half_of<F16>(wf[i], j)) : -0.f;
            h[j] = step(q[i][j], h[j], half_of<F16>(wx[i], j));
            rest[j] = step(q[i][j], rest[j], 1.f);
            product[j] = times(q[i][j], product[j]);
        }
    return make_float4(factor_of(product[0], rest[0]), h[0], factor_of(product[1], rest[1]), h[1]);
}

template <bool F16, int ACT>
__global__ void __launch_bounds__(kThreads) recur_kernel(const __grid_constant__ RecurArgs a, int cluster) {
    __shared__ float4 runs[2][kRuns][16];
    __shared__ float4 tiles[2][kMostCluster][16];
    const int run = threadIdx.x / 16, lane = threadIdx.x % 16;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int unit = blockIdx.x / cluster, s = unit / a.col_tiles;
    const int col = (unit - s * a.col_tiles) * kCols + 2 * lane, n = a.at.n;
    const int valid = min(max(n - col, 0), 2);
    const bool words = a.words != 0, gated = a.o.p != nullptr;
    if (cluster > 1) cluster_arrive();
    pdl_trigger();
    pdl_wait();
    int r0, r1;
    a.at.rows_of(s, r0, r1);
    float carry[2];
    load_state(a.state, s, n, col, valid, carry);
    if (cluster > 1) cluster_wait();
    const int all = (r1 - r0 + kTile - 1) / kTile;
    int turn = 0;
    for (int first = 0; first < all; first += cluster, turn ^= 1) {
        const int tile = first + rank;
        const int64_t row = (int64_t)r0 + (int64_t)tile * kTile + run * kLen;
        const int count = (int)min((int64_t)kLen, r1 - row);  // of this run; none if negative
        uint32_t wf[kLen], wx[kLen], wo[kLen];
#pragma unroll
        for (int i = 0; i < kLen; ++i) {
            wf[i] = wx[i] = wo[i] = 0u;
            if (i >= count) continue;
            wf[i] = load_pair(a.f, row + i, col, valid, words);
            wx[i] = load_pair(a.x, row + i, col, valid, words);
            if (gated) wo[i] = load_pair(a.o, row + i, col, valid, words);
        }
        float q[kLen][2], h[2];
        runs[turn][run][lane] = local_run<F16>(wf, wx, count, q);
        __syncthreads();
        if (cluster > 1) {
            if (run == 0) {
                float4 sum = runs[turn][0][lane];
#pragma unroll
                for (int r = 1; r < kRuns; ++r) join(sum, runs[turn][r][lane]);
                share(tiles[turn], sum, rank, cluster, lane);
            }
            __syncwarp();
            cluster_sync();
            for (int other = 0; other < cluster; ++other) {
                if (other == rank) h[0] = carry[0], h[1] = carry[1];
                then(carry, tiles[turn][other][lane]);
            }
            if (run == 0 && tile < all) store_state(a.states, (int64_t)r0 / kTile + tile + s, n, col, valid, h);
            for (int r = 0; r < run; ++r) then(h, runs[turn][r][lane]);
        } else {
            if (run == 0) store_state(a.states, (int64_t)r0 / kTile + tile + s, n, col, valid, carry);
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                if (r == run) h[0] = carry[0], h[1] = carry[1];
                then(carry, runs[turn][r][lane]);
            }
        }
#pragma unroll
        for (int i = 0; i < kLen; ++i) {
            if (i >= count) continue;
            float y[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                h[j] = step(q[i][j], h[j], half_of<F16>(wx[i], j));
                y[j] = gated ? h[j] * act_of<ACT>(half_of<F16>(wo[i], j)) : h[j];
            }
            store_pair(a.y, row + i, col, valid, words, pack16<F16>(y[0], y[1]));
        }
    }
    if (rank == 0 && run == 0) store_state(a.last, s, n, col, valid, carry);
}

template <bool F16, int ACT>
__global__ void __launch_bounds__(kThreads) recur_grad_kernel(const __grid_constant__ RecurGradArgs a, int cluster) {
    __shared__ float4 runs[2][kRuns][16];  // q and H of the runs
    __shared__ float2 back[2][kRuns][16];  // R
    __shared__ float4 tiles[2][kMostCluster][16];  // q and R of the tiles
    const int run = threadIdx.x / 16, lane = threadIdx.x % 16;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int unit = blockIdx.x / cluster, s = unit / a.col_tiles;
    const int col = (unit - s * a.col_tiles) * kCols + 2 * lane, n = a.at.n;
    const int valid = min(max(n - col, 0), 2);
    const bool words = a.words != 0, gated = a.o.p != nullptr;
    if (cluster > 1) cluster_arrive();
    pdl_trigger();
    pdl_wait();
    int r0, r1;
    a.at.rows_of(s, r0, r1);
    float carry[2];
    load_state(a.d_last, s, n, col, valid, carry);
    if (cluster > 1) cluster_wait();
    const int all = (r1 - r0 + kTile - 1) / kTile;
    int turn = 0;
    for (int first = 0; first < all; first += cluster, turn ^= 1) {
        const int tile = all - 1 - (first + rank);  // negative: nothing is left for this block
        const int64_t row = (int64_t)r0 + (int64_t)tile * kTile + run * kLen;
        const int count = tile < 0 ? 0 : (int)min((int64_t)kLen, r1 - row);
        uint32_t wf[kLen], wx[kLen], wo[kLen], wd[kLen];
#pragma unroll
        for (int i = 0; i < kLen; ++i) {
            wf[i] = wx[i] = wo[i] = wd[i] = 0u;
            if (i >= count) continue;
            wf[i] = load_pair(a.f, row + i, col, valid, words);
            wx[i] = load_pair(a.x, row + i, col, valid, words);
            wd[i] = load_pair(a.dy, row + i, col, valid, words);
            if (gated) wo[i] = load_pair(a.o, row + i, col, valid, words);
        }
        float h[2] = {0.f, 0.f};
        if (tile >= 0) load_state(a.states, (int64_t)r0 / kTile + tile + s, n, col, valid, h);
        float q[kLen][2], p[2] = {0.f, 0.f};
        runs[turn][run][lane] = local_run<F16>(wf, wx, count, q);
#pragma unroll
        for (int i = kLen - 1; i >= 0; --i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float dy = half_of<F16>(wd[i], j);
                const float g = p[j] + (gated ? dy * act_of<ACT>(half_of<F16>(wo[i], j)) : dy);
                p[j] = times(q[i][j], g);
            }
        back[turn][run][lane] = make_float2(p[0], p[1]);
        __syncthreads();
        auto down = [&](float (&v)[2], int r) {  // p past the run r
            const float4 c = runs[turn][r][lane];
            const float2 d = back[turn][r][lane];
            v[0] = d.x + times(c.x, v[0]);
            v[1] = d.y + times(c.z, v[1]);
        };
        if (cluster > 1) {
            if (run == 0) {
                float4 sum = runs[turn][kRuns - 1][lane];
                sum.y = back[turn][kRuns - 1][lane].x;
                sum.w = back[turn][kRuns - 1][lane].y;
#pragma unroll
                for (int r = kRuns - 2; r >= 0; --r) {
                    const float4 c = runs[turn][r][lane];
                    const float2 d = back[turn][r][lane];
                    join(sum, make_float4(c.x, d.x, c.z, d.y));
                }
                share(tiles[turn], sum, rank, cluster, lane);
            }
            __syncwarp();
            cluster_sync();
            for (int other = 0; other < cluster; ++other) {
                if (other == rank) p[0] = carry[0], p[1] = carry[1];
                then(carry, tiles[turn][other][lane]);
            }
            for (int r = kRuns - 1; r > run; --r) down(p, r);
        } else {
#pragma unroll
            for (int r = kRuns - 1; r >= 0; --r) {
                if (r == run) p[0] = carry[0], p[1] = carry[1];
                down(carry, r);
            }
        }
        for (int r = 0; r < run; ++r) then(h, runs[turn][r][lane]);
        float before[kLen][2];  // the state before each step
#pragma unroll
        for (int i = 0; i < kLen; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                before[i][j] = h[j];
                h[j] = step(q[i][j], h[j], half_of<F16>(wx[i], j));
            }
#pragma unroll
        for (int i = kLen - 1; i >= 0; --i) {
            if (i >= count) continue;
            float df[2], dx[2], d_o[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float dy = half_of<F16>(wd[i], j), x = half_of<F16>(wx[i], j);
                float act = 1.f, slope = 0.f;
                if (gated) act_slope<ACT>(half_of<F16>(wo[i], j), act, slope);
                const float g = fmaf(dy, act, p[j]), size = fabsf(q[i][j]);  // a or 1 - a, the smaller
                dx[j] = complement(q[i][j]) * g;
                df[j] = g * (before[i][j] - x) * fmaf(-size, size, size);
                d_o[j] = dy * slope * step(q[i][j], before[i][j], x);
                p[j] = times(q[i][j], g);
            }
            if (a.df.p) store_pair(a.df, row + i, col, valid, words, pack16<F16>(df[0], df[1]));
            if (a.dx.p) store_pair(a.dx, row + i, col, valid, words, pack16<F16>(dx[0], dx[1]));
            if (a.d_o.p) store_pair(a.d_o, row + i, col, valid, words, pack16<F16>(d_o[0], d_o[1]));
        }
    }
    if (rank == 0 && run == 0) store_state(a.d_state, s, n, col, valid, carry);
}

// Sequences of up to kShort steps, all of one length: two columns of one to a thread.
template <bool F16, int ACT>
__global__ void __launch_bounds__(256) recur_short_kernel(const __grid_constant__ RecurArgs a) {
    const int pairs = (a.at.n + 1) / 2, n = a.at.n;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t s = at / pairs;
    const int col = (int)(at - s * pairs) * 2, valid = min(n - col, 2);
    const bool words = a.words != 0, gated = a.o.p != nullptr;
    pdl_trigger();
    pdl_wait();
    if (s >= a.at.seqs) return;
    const int64_t r0 = s * a.at.length;
    float h[2];
    load_state(a.state, s, n, col, valid, h);
    store_state(a.states, r0 / kTile + s, n, col, valid, h);
#pragma unroll
    for (int i = 0; i < kShort; ++i) {
        if (i >= a.at.length) break;
        const uint32_t f = load_pair(a.f, r0 + i, col, valid, words), x = load_pair(a.x, r0 + i, col, valid, words);
        const uint32_t o = gated ? load_pair(a.o, r0 + i, col, valid, words) : 0u;
        float y[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            h[j] = step(factor_of(half_of<F16>(f, j)), h[j], half_of<F16>(x, j));
            y[j] = gated ? h[j] * act_of<ACT>(half_of<F16>(o, j)) : h[j];
        }
        store_pair(a.y, r0 + i, col, valid, words, pack16<F16>(y[0], y[1]));
    }
    store_state(a.last, s, n, col, valid, h);
}

// ---------------------------------------------------------------- host
bool on_words(const emtk_matrix &m, int rows) {
    return !m.d || (reinterpret_cast<uintptr_t>(m.d) % 4 == 0 && (rows <= 1 || m.ld % 2 == 0));
}

// Blocks of a unit (32 columns of a sequence): as many as its tiles occupy, until there
// are three for each SM.
int cluster_of(int64_t units, int rows, int seqs, int sms) {
    const int64_t tiles = ((int64_t)rows + (int64_t)seqs * kTile - 1) / ((int64_t)seqs * kTile);
    int c = 1;
    while (c < kMostCluster && units * c < 3 * sms && 2 * c <= tiles) c *= 2;
    return c;
}

template <typename Kernel, typename Args>
cudaError_t run_tiles(Kernel kernel, const Args &a, int sms, cudaStream_t s) {
    const int64_t units = (int64_t)a.at.seqs * a.col_tiles;
    const int cluster = cluster_of(units, a.at.rows, a.at.seqs, sms);
    if (units * cluster > INT32_MAX) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)(units * cluster)), block(kThreads);
    return cluster == 1 ? launch_pdl(kernel, grid, block, 0, s, a, cluster) : launch_cluster(kernel, grid, block, cluster, s, a, cluster);
}

template <bool F16, int ACT>
cudaError_t run(const RecurArgs &a, int sms, cudaStream_t s) {
    if (!a.at.offsets && a.at.length <= kShort) {
        const int64_t blocks = ((int64_t)a.at.seqs * ((a.at.n + 1) / 2) + 255) / 256;
        if (blocks > INT32_MAX) return cudaErrorInvalidValue;
        return launch_pdl(recur_short_kernel<F16, ACT>, dim3((unsigned)blocks), dim3(256), 0, s, a);
    }
    return run_tiles(recur_kernel<F16, ACT>, a, sms, s);
}
template <bool F16, int ACT>
cudaError_t run(const RecurGradArgs &a, int sms, cudaStream_t s) {
    return run_tiles(recur_grad_kernel<F16, ACT>, a, sms, s);
}
template <bool F16, typename Args>
cudaError_t run(const Args &a, int act, int sms, cudaStream_t s) {
    switch (act) {
        case EMTK_ACT_RELU: return run<F16, EMTK_ACT_RELU>(a, sms, s);
        case EMTK_ACT_GELU: return run<F16, EMTK_ACT_GELU>(a, sms, s);
        case EMTK_ACT_SILU: return run<F16, EMTK_ACT_SILU>(a, sms, s);
        case EMTK_ACT_SIGMOID: return run<F16, EMTK_ACT_SIGMOID>(a, sms, s);
        default: return run<F16, EMTK_ACT_NONE>(a, sms, s);
    }
}
template <typename Args>
cudaError_t run(const Args &a, int type, int act, int sms, cudaStream_t s) {
    return type == EMTK_TYPE_F16 ? run<true>(a, act, sms, s) : run<false>(a, act, sms, s);
}

}  // namespace

cudaError_t launch_recurrence(const emtk_recurrence_args &p, int sms, cudaStream_t s) {
    if (p.n == 0 || p.seqs == 0) return cudaSuccess;
    RecurArgs a{};
    a.f = plane_of(p.f);
    a.x = plane_of(p.x);
    a.o = plane_of(p.o);
    a.y = plane_of(p.y);
    a.at = {p.offsets, p.rows, p.n, p.seqs, p.offsets ? 0 : p.rows / p.seqs};
    a.state = p.state;
    a.last = p.last;
    a.states = p.states;
    a.col_tiles = (p.n + kCols - 1) / kCols;
    a.words = on_words(p.f, p.rows) && on_words(p.x, p.rows) && on_words(p.o, p.rows) && on_words(p.y, p.rows);
    return run(a, p.type, p.act, sms, s);
}

cudaError_t launch_recurrence_grad(const emtk_recurrence_grad_args &p, int sms, cudaStream_t s) {
    if (p.n == 0 || p.seqs == 0) return cudaSuccess;
    RecurGradArgs a{};
    a.dy = plane_of(p.dy);
    a.f = plane_of(p.f);
    a.x = plane_of(p.x);
    a.o = plane_of(p.o);
    a.df = plane_of(p.df);
    a.dx = plane_of(p.dx);
    a.d_o = plane_of(p.d_o);
    a.at = {p.offsets, p.rows, p.n, p.seqs, p.offsets ? 0 : p.rows / p.seqs};
    a.states = p.states;
    a.d_last = p.d_last;
    a.d_state = p.d_state;
    a.col_tiles = (p.n + kCols - 1) / kCols;
    a.words = on_words(p.dy, p.rows) && on_words(p.f, p.rows) && on_words(p.x, p.rows) && on_words(p.o, p.rows) &&
              on_words(p.df, p.rows) && on_words(p.dx, p.rows) && on_words(p.d_o, p.rows);
    return run(a, p.type, p.act, sms, s);
}

}  // namespace emtk
