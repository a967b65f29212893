// The gated linear recurrence along sequences, and its gradients.
//
//   b = 1 / (1 + exp(f));  h_t = h_(t-1) + b_t (x_t - h_(t-1));  y = act(o) h
//
// A run of steps maps the state before it to the one after it, linearly: h becomes H + A h,
// with H the state that the run makes of 0 and A = prod(1 - b).  A run's factor is held as q:
// itself where it is below a half, else as its complement with the sign changed, A - 1, so
// that neither what is kept for long nor what is nearly forgotten loses its low bits: at
// f = 8 a rounding of 1 - b in fp32 alone is 10^-4 of the state it settles to.  A step's is
// held as -b and used as h + b (x - h), off by 2^-24 of the state before it at most.
//
// A block takes 32 columns and goes along a sequence in tiles of 128 steps: each half
// warp a run of 16 steps, two columns to a lane.  The runs' (q, H) meet in shared memory, each
// half warp joins those before its own and goes over its steps once more, from shared
// memory, where TMA brought the tile: everything is read once and written once.
//
// Where equal sequences and their columns are too few for the SMs, or lengths are unlike,
// tiles are made independent in three kernels: the first leaves each tile's (q, H), the second
// goes along those (a 128th of the data) to each tile's state, the third makes each
// tile's outputs.  f and x are read twice then; HBM or L2 is kept busy whatever the
// sequences are.  (Clusters of blocks that exchange their tiles' (q, H) round by round were
// slower: a round waits 1.4 us for the exchange, as long as a tile takes.)  Orders are fixed:
// the same call gives the same bits.
//
// Backwards, g_t = u_t + (1 - b_(t+1)) g_(t+1) with u = act(o) dy: passing p = (1 - b) g down,
// a run makes p of R + A p, with the same A.  A tile's states come from the one
// before it, which the forward pass kept.
//
// HBM bounds it: 8 bytes a value forward, 14 backward (16 bits, with o).  800 sequences of 1000
// steps of 64 columns in bf16: 71 us forward (5.7 TB/s), 154 backward (4.7 TB/s; 142 registers leave 12
// warps an SM, which wait for their own arithmetic); 20011 steps of 2048 in 4 sequences, as independent tiles, 104 and 195.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_pair.cuh"
#include "nn_ptx.cuh"

namespace emtk {
namespace {

constexpr int kLanes = 16, kCols = 2 * kLanes;  // two columns a lane
constexpr int kRuns = 8, kLen = 16, kTile = kRuns * kLen, kThreads = kLanes * kRuns;
// A thread takes a whole sequence below kLong steps, in lots of kLot, where sequences are short on average.
constexpr int kLot = 8, kLong = 64;
static_assert(kTile == EMTK_RECURRENCE_STEP, "states are kept once a tile");

// Where what is kept of a sequence's tile lies: tiles of different sequences, in order and with gaps.
__device__ __forceinline__ int64_t place_of(int r0, int tile, int seq) { return (int64_t)(r0 / kTile) + tile + seq; }

struct Plane {  // a 16-bit matrix
    uint8_t *p;
    int64_t row_bytes;
};
Plane plane_of(const emtk_matrix &m) { return {static_cast<uint8_t *>(m.d), 2 * m.ld}; }

struct Sequences {
    const int32_t *offsets;
    int rows, n, seqs, length;  // length: of each, without offsets
    int long_only;              // blocks are to sequences of kLong steps and more alone
    __device__ __forceinline__ void rows_of(int s, int &r0, int &r1) const {
        if (offsets) {
            r0 = min(max(__ldg(offsets + s), 0), rows);
            r1 = min(max(__ldg(offsets + s + 1), r0), rows);
        } else {
            r0 = s * length;
            r1 = r0 + length;
        }
    }
    // The sequence whose tiles' places include this one, if any's do: the last that begins
    // at it or before (or, of rows, the one that has this row).  All lanes of a warp look together.
    template <bool ROW>
    __device__ __forceinline__ int at_place(int place) const {
        int low = 0, high = seqs;  // it is in low .. high - 1
        const int lane = threadIdx.x & 31;
        while (high - low > 1) {
            const int step = (high - low + 31) / 32, s = low + lane * step;
            int r0 = 0, r1;
            if (s < high) rows_of(s, r0, r1);
            const uint32_t before = __ballot_sync(0xffffffffu, s < high && (lane == 0 || (ROW ? r0 : place_of(r0, 0, s)) <= place));
            low += (31 - __clz(before)) * step;
            high = min(low + step, high);
        }
        return low;
    }
};

struct Waits {  // of the kernels' bounded waits
    int *status;
    int64_t timeout_ns;
};
constexpr int kMostIn = 4;  // matrices of a tile: f, x, o and dy, in this order
struct Tiles {
    CUtensorMap in[kMostIn], out[3];  // out: y, or df, dx, d_o; of what is there
    int store;                        // whole tiles of results leave by TMA
    Waits waits;
};

// `starts`: what comes into each tile (its state, or backwards its p), at place_of; null
// where a block goes along a whole sequence.
struct RecurArgs {
    Plane f, x, o, y;
    Sequences at;
    const float *state, *starts;
    float *last, *states;
    int col_tiles, words;  // words: every row starts on 4 bytes
};
struct RecurGradArgs {
    Plane f, x, o, dy, df, dx, d_o;
    Sequences at;
    const float *states, *d_last, *starts;
    float *d_state;
    int col_tiles, words;
};

template <int ACT>
__device__ __forceinline__ float2 act2(float2 z) {
    return make_float2(act_of<ACT>(z.x), act_of<ACT>(z.y));
}

// Two neighbouring columns, of which `valid` exist.
__device__ __forceinline__ uint32_t load_pair(const uint8_t *p, int valid, bool words) {
    if (words && valid == 2) return __ldg(reinterpret_cast<const uint32_t *>(p));
    const uint16_t *const h = reinterpret_cast<const uint16_t *>(p);
    uint32_t v = 0;
    if (valid > 0) v = __ldg(h);
    if (valid > 1) v |= (uint32_t)__ldg(h + 1) << 16;
    return v;
}
__device__ __forceinline__ void store_pair(uint8_t *p, int valid, bool words, uint32_t v) {
    uint16_t *const h = reinterpret_cast<uint16_t *>(p);
    if (words && valid == 2) {
        *reinterpret_cast<uint32_t *>(p) = v;
        return;
    }
    if (valid > 0) h[0] = (uint16_t)v;
    if (valid > 1) h[1] = (uint16_t)(v >> 16);
}
__device__ __forceinline__ uint8_t *place(const Plane &a, int64_t row, int col) { return a.p + row * a.row_bytes + 2 * (int64_t)col; }

// fp32 states [..][n]
__device__ __forceinline__ float2 load_state(const float *p, int64_t row, int n, int c, int valid) {
    p += row * n + c;
    return make_float2(valid > 0 ? p[0] : 0.f, valid > 1 ? p[1] : 0.f);
}
__device__ __forceinline__ void store_state(float *p, int64_t row, int n, int c, int valid, float2 v) {
    p += row * n + c;
    if (valid > 0) p[0] = v.x;
    if (valid > 1) p[1] = v.y;
}

// ---- a step's factor, as m = a - 1 = -1 / (1 + exp(f))
template <bool F16>
__device__ __forceinline__ float2 minus_rest(uint32_t w) {
    const float2 z = values_of<F16>(w) * both(kLog2E);
    const float2 d = fma2(make_float2(exp2_f(z.x), exp2_f(z.y)), both(-1.f), both(-1.f));  // -infinity: keeps all
    return make_float2(reciprocal_f(d.x), reciprocal_f(d.y));
}
constexpr uint32_t kKeepAll16 = 0x7c007c00u, kKeepAll = 0x7f807f80u;  // f of a step that is not there: infinity
__device__ __forceinline__ float2 step(float2 m, float2 h, float2 x) { return fma2(m, h - x, h); }  // a h + (1 - a) x
__device__ __forceinline__ float2 kept(float2 m, float2 v) { return fma2(m, v, v); }                // a v
// a (1 - a): a = exp(f) (1 - a), right to its last bits where it is small too; beyond 80, where exp(f) may be infinity, it is 1
__device__ __forceinline__ float slope_of(float f, float m) {
    const float b = -m;
    return (f > 80.f ? 1.f : exp2_f(f * kLog2E) * b) * b;
}

// ---- a run's factor, held as q (above); -0 is the complement 0
__device__ __forceinline__ bool is_complement(float q) { return __float_as_int(q) < 0; }
__device__ __forceinline__ float times(float q, float v) { return fmaf(q, v, is_complement(q) ? v : 0.f); }
__device__ __forceinline__ float2 times(float2 q, float2 v) {
    return fma2(q, v, make_float2(is_complement(q.x) ? v.x : 0.f, is_complement(q.y) ? v.y : 0.f));
}
__device__ __forceinline__ float factor_of(float product, float complement) { return complement < 0.5f ? -complement : product; }
__device__ __forceinline__ float product_of(float p, float q) {  // of two runs
    if (!is_complement(p) || !is_complement(q)) return is_complement(p) ? times(p, q) : times(q, p);
    const float c = fmaf(-p, 1.f + q, -q);  // both complements: 1 - (1 - c1)(1 - c2)
    return c < 0.5f ? -c : 1.f - c;
}

// Runs of two columns: (q0, q1, H0, H1).
__device__ __forceinline__ float2 then(float2 state, const float4 &run) {
    return make_float2(run.z, run.w) + times(make_float2(run.x, run.y), state);
}
__device__ __forceinline__ float4 join(const float4 &a, const float4 &b) {  // a, then b
    const float2 h = then(make_float2(a.z, a.w), b);
    return make_float4(product_of(a.x, b.x), product_of(a.y, b.y), h.x, h.y);
}

// ---- a tile in shared memory: kTile rows of 32 columns to a matrix
constexpr int kPlane = kTile * kLanes;  // words
// The words of a thread's run: word i is its step i.
__device__ __forceinline__ uint32_t *run_of(uint32_t *plane, int run, int lane) { return plane + run * kLen * kLanes + lane; }

// Rows row .. row + kTile - 1 into `plane`, those from `end` on as `fill`, by all threads; a
// thread's loads together.
__device__ __forceinline__ void fill_plane(uint32_t *plane, const Plane &a, int64_t row, int64_t end, int col, int valid, bool words,
                                           uint32_t fill) {
    const int lane = threadIdx.x % kLanes, r0 = threadIdx.x / kLanes;
    const uint8_t *p = place(a, row + r0, col);
    const int left = (int)min((int64_t)kTile, end - row) - r0;  // rows from the thread's first on
    uint32_t v[kLen];
    if (words && valid == 2) {
#pragma unroll
        for (int i = 0; i < kLen; ++i, p += kRuns * a.row_bytes) v[i] = i * kRuns < left ? __ldg(reinterpret_cast<const uint32_t *>(p)) : fill;
    } else {
#pragma unroll
        for (int i = 0; i < kLen; ++i, p += kRuns * a.row_bytes) {
            const uint16_t *const h = reinterpret_cast<const uint16_t *>(p);
            const uint32_t lo = i * kRuns < left && valid > 0 ? __ldg(h) : fill & 0xffffu;
            const uint32_t hi = i * kRuns < left && valid > 1 ? __ldg(h + 1) : fill >> 16;
            v[i] = lo | hi << 16;
        }
    }
#pragma unroll
    for (int i = 0; i < kLen; ++i) plane[(r0 + i * kRuns) * kLanes + lane] = v[i];
}
__device__ __forceinline__ void empty_plane(const uint32_t *plane, const Plane &a, int64_t row, int64_t end, int col, int valid, bool words) {
    const int lane = threadIdx.x % kLanes;
    int r = threadIdx.x / kLanes;
    uint8_t *p = place(a, row + r, col);
#pragma unroll 8
    for (int i = 0; i < kLen; ++i, r += kRuns, p += kRuns * a.row_bytes)
        if (row + r < end) store_pair(p, valid, words, plane[r * kLanes + lane]);
}

// The steps of a thread's run that the sequence does not have, in each of N planes.
template <int N>
__device__ __forceinline__ void mask_run(uint32_t *planes, int run, int lane, int count, uint32_t keep_all) {
    for (int i = count; i < kLen; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) run_of(planes + k * kPlane, run, lane)[i * kLanes] = k == 0 ? keep_all : 0u;
}

// A half warp's run from state 0, and its steps' factors.
template <bool F16>
__device__ __forceinline__ float4 local_run(const uint32_t *f, const uint32_t *x, float2 (&m)[kLen]) {
    float2 h = both(0.f), product = both(1.f), rest = both(0.f);
#pragma unroll
    for (int i = 0; i < kLen; ++i) {
        m[i] = minus_rest<F16>(f[i * kLanes]);
        h = step(m[i], h, values_of<F16>(x[i * kLanes]));
        rest = step(m[i], rest, both(1.f));
        product = kept(m[i], product);
    }
    return make_float4(factor_of(product.x, rest.x), factor_of(product.y, rest.y), h.x, h.y);
}

// Of a run without steps: it keeps all and makes nothing.
__device__ __forceinline__ float4 no_run() { return make_float4(-0.f, -0.f, 0.f, 0.f); }
// The same from its end, for p.
template <bool F16, int ACT>
__device__ __forceinline__ float2 local_back(const float2 (&m)[kLen], const uint32_t *d, const uint32_t *o, bool gated) {
    float2 p = both(0.f);
#pragma unroll
    for (int i = kLen - 1; i >= 0; --i) {
        const float2 dy = values_of<F16>(d[i * kLanes]);
        p = kept(m[i], gated ? fma2(dy, act2<ACT>(values_of<F16>(o[i * kLanes])), p) : p + dy);
    }
    return p;
}

// Where a block works: a sequence's columns, all of its tiles or the one at a place.  Long
// sequences among short ones are found by the first of the rows 0, kLong, 2 kLong .. that they have.
struct Unit {
    int run, lane, seq, col0, col, valid;
    bool any;  // false: a row that no long sequence is found by
    int r0, r1, tile, tiles;  // the sequence's rows; the tiles to do, from `tile` on (or from its end)
    __device__ __forceinline__ Unit(const Sequences &at, int col_tiles, bool one_tile)
        : run(threadIdx.x / kLanes), lane(threadIdx.x % kLanes) {
        const int unit = blockIdx.x / col_tiles;
        col0 = ((int)blockIdx.x - unit * col_tiles) * kCols;
        col = col0 + 2 * lane;
        valid = min(max(at.n - col, 0), 2);
        seq = one_tile ? at.at_place<false>(unit) : at.long_only ? at.at_place<true>(unit * kLong) : unit;
        at.rows_of(seq, r0, r1);
        any = !at.long_only || (r1 - r0 >= kLong && (r0 + kLong - 1) / kLong == unit);
        tiles = (r1 - r0 + kTile - 1) / kTile;
        tile = 0;
        if (one_tile) {
            tile = unit - (int)place_of(r0, 0, seq);
            tiles = tile >= 0 && tile < tiles ? 1 : 0;
        }
    }
};

// Tiles on their way: two stages of planes, filled by TMA a tile ahead, one barrier each.
// A stage's results take its inputs' places and leave by TMA too, where they lie on its
// grid and rows are whole pieces of 16 bytes (at 31 columns a store wrote the 32nd, the
// caller's padding); it is filled again once they are read, in the middle of the next tile.
struct Pipe {
    uint32_t *stages;  // [2][planes][kPlane]
    uint64_t *full;    // [2]
    int planes;
    Guard guard;
    bool ok = true;

    __device__ __forceinline__ void start() {
        if (threadIdx.x == 0) {
            mbar_init(smem_u32(full), 1);
            mbar_init(smem_u32(full + 1), 1);
            *guard.abort = 0;
            fence_mbar_init();
        }
        __syncthreads();
    }
    __device__ __forceinline__ uint32_t *stage(int s) const { return stages + s * planes * kPlane; }
    // One thread: the tile of rows row .. into stage s.
    __device__ __forceinline__ void load(const Tiles &t, const bool (&has)[kMostIn], int s, int col, int row) const {
        const uint32_t bar = smem_u32(full + s);
        int bytes = 0;
#pragma unroll
        for (int k = 0; k < kMostIn; ++k) bytes += has[k] ? 4 * kPlane : 0;
        mbar_expect_tx(bar, bytes);
#pragma unroll
        for (int k = 0; k < kMostIn; ++k)
            if (has[k]) tma_load_2d(smem_u32(stage(s) + k * kPlane), &t.in[k], bar, col, row);
    }
    __device__ __forceinline__ void wait(int s, uint32_t parity) {
        if (ok) ok = wait_bounded(smem_u32(full + s), parity, guard);
    }
};

// Results in flight have been read when a block leaves; copies in flight after a wait
// that gave up land within microseconds: they are left a millisecond.
__device__ __forceinline__ void pipe_end(const Pipe &pipe) {
    if (threadIdx.x == 0) bulk_wait_read();
    if (pipe.ok) return;
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 1000000u) {
    }
}

// The tiles of a sequence one after another, or (a.starts) a tile.
template <bool F16, int ACT, bool TMA>
__global__ void __launch_bounds__(kThreads, 4) recur_kernel(const __grid_constant__ RecurArgs a, const __grid_constant__ Tiles maps) {
    extern __shared__ __align__(128) uint32_t planes[];
    __shared__ float4 runs[2][kRuns][kLanes];
    __shared__ uint64_t full[2];
    __shared__ uint32_t abort_flag;
    const int n = a.at.n;
    const bool words = a.words != 0, gated = a.o.p != nullptr;
    constexpr uint32_t kFill = F16 ? kKeepAll16 : kKeepAll;
    Pipe pipe{planes, full, 3, {&abort_flag, maps.waits.status, maps.waits.timeout_ns}};
    if (TMA) pipe.start();
    pdl_trigger();
    pdl_wait();
    const Unit u(a.at, a.col_tiles, a.starts != nullptr);
    if (!u.any) return;
    const bool has[kMostIn] = {true, true, gated, false};
    auto fetch = [&](int i, int s) {  // the i-th tile
        if (TMA && threadIdx.x == 0 && i < u.tiles) pipe.load(maps, has, s, u.col0, u.r0 + (u.tile + i) * kTile);
    };
    fetch(0, 0);
    fetch(1, 1);
    float2 carry = both(0.f);
    if (a.starts) {
        if (u.tiles > 0) carry = load_state(a.starts, place_of(u.r0, u.tile, u.seq), n, u.col, u.valid);
    } else if (a.state) {
        carry = load_state(a.state, u.seq, n, u.col, u.valid);
    }
    int turn = 0, parity = 0;
    for (int i = 0; i < u.tiles; ++i) {
        const int64_t row = (int64_t)u.r0 + (int64_t)(u.tile + i) * kTile;
        const int count = (int)max(min((int64_t)kLen, u.r1 - row - u.run * kLen), (int64_t)0);  // steps of this run
        uint32_t *const stage = TMA ? pipe.stage(turn) : planes;
        if (TMA) {
            pipe.wait(turn, parity);
        } else {
            __syncthreads();  // the results of the tile before have left
            fill_plane(stage, a.f, row, u.r1, u.col, u.valid, words, kFill);
            fill_plane(stage + kPlane, a.x, row, u.r1, u.col, u.valid, words, 0u);
            if (gated) fill_plane(stage + 2 * kPlane, a.o, row, u.r1, u.col, u.valid, words, 0u);
            __syncthreads();
        }
        const bool work = __any_sync(0xffffffffu, count > 0);  // of the warp's two runs
        if (work && count < kLen) mask_run<3>(stage, u.run, u.lane, count, kFill);
        const uint32_t *const f = run_of(stage, u.run, u.lane), *const o = run_of(stage + 2 * kPlane, u.run, u.lane);
        uint32_t *const x = run_of(stage + kPlane, u.run, u.lane);
        float2 m[kLen], h;
        runs[turn][u.run][u.lane] = work ? local_run<F16>(f, x, m) : no_run();
        __syncthreads();
        if (TMA && i > 0) {  // the other stage's results have been read: its next tile
            if (threadIdx.x == 0) bulk_wait_read();
            fetch(i + 1, turn ^ 1);
        }
        if (a.states && u.run == 0) store_state(a.states, place_of(u.r0, u.tile + i, u.seq), n, u.col, u.valid, carry);
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
            if (r == u.run) h = carry;
            carry = then(carry, runs[turn][r][u.lane]);
        }
        if (work) {
#pragma unroll
            for (int j = 0; j < kLen; ++j) {
                h = step(m[j], h, values_of<F16>(x[j * kLanes]));
                const float2 y = gated ? h * act2<ACT>(values_of<F16>(o[j * kLanes])) : h;
                x[j * kLanes] = pack16<F16>(y.x, y.y);
            }
        }
        if (TMA) bulk_fence();
        __syncthreads();
        if (TMA && maps.store && row + kTile <= u.r1) {
            if (threadIdx.x == 0) bulk_store(&maps.out[0], smem_u32(stage + kPlane), u.col0, (int)row);
        } else {
            empty_plane(stage + kPlane, a.y, row, u.r1, u.col, u.valid, words);
        }
        parity ^= turn;
        turn ^= 1;
    }
    if (a.last && !a.starts && u.run == 0) store_state(a.last, u.seq, n, u.col, u.valid, carry);
    if (TMA) pipe_end(pipe);
}

// A step's gradients, from the states before and after it and the p that comes into it, which
// becomes the one that leaves it.
struct Slopes {
    float2 df, dx;
};
template <bool F16, int ACT>
__device__ __forceinline__ Slopes slopes(float2 m, float2 before, float2 after, uint32_t wf, uint32_t wx, uint32_t wo, uint32_t wd, bool gated,
                                         float2 &p, float2 &d_o) {
    const float2 dy = values_of<F16>(wd);
    float2 g = p + dy;
    if (gated) {
        const float2 o = values_of<F16>(wo);
        float2 act, slope;
        act_slope<ACT>(o.x, act.x, slope.x);
        act_slope<ACT>(o.y, act.y, slope.y);
        g = fma2(dy, act, p);
        d_o = dy * slope * after;
    }
    const float2 f = values_of<F16>(wf), slope_f = make_float2(slope_of(f.x, m.x), slope_of(f.y, m.y));
    p = kept(m, g);
    return {g * (before - values_of<F16>(wx)) * slope_f, -m * g};
}

// Backwards: the tiles of a sequence from its last, or (a.starts) a tile.
template <bool F16, int ACT, bool TMA>
__global__ void __launch_bounds__(kThreads, 3) recur_grad_kernel(const __grid_constant__ RecurGradArgs a,
                                                                 const __grid_constant__ Tiles maps) {
    extern __shared__ __align__(128) uint32_t planes[];
    __shared__ float4 runs[2][kRuns][kLanes];  // q and H of the runs
    __shared__ float2 back[2][kRuns][kLanes];  // R
    __shared__ uint64_t full[2];
    __shared__ uint32_t abort_flag;
    const int n = a.at.n;
    const bool words = a.words != 0, gated = a.o.p != nullptr;
    constexpr uint32_t kFill = F16 ? kKeepAll16 : kKeepAll;
    Pipe pipe{planes, full, 4, {&abort_flag, maps.waits.status, maps.waits.timeout_ns}};
    if (TMA) pipe.start();
    pdl_trigger();
    pdl_wait();
    const Unit u(a.at, a.col_tiles, a.starts != nullptr);
    if (!u.any) return;
    const bool has[kMostIn] = {true, true, gated, true};
    auto fetch = [&](int i, int s) {
        if (TMA && threadIdx.x == 0 && i < u.tiles) pipe.load(maps, has, s, u.col0, u.r0 + (u.tile + u.tiles - 1 - i) * kTile);
    };
    fetch(0, 0);
    fetch(1, 1);
    float2 carry = both(0.f);
    if (a.starts) {
        if (u.tiles > 0) carry = load_state(a.starts, place_of(u.r0, u.tile, u.seq), n, u.col, u.valid);
    } else if (a.d_last) {
        carry = load_state(a.d_last, u.seq, n, u.col, u.valid);
    }
    int turn = 0, parity = 0;
    for (int i = 0; i < u.tiles; ++i) {
        const int tile = u.tile + u.tiles - 1 - i;
        const int64_t row = (int64_t)u.r0 + (int64_t)tile * kTile;
        const int count = (int)max(min((int64_t)kLen, u.r1 - row - u.run * kLen), (int64_t)0);
        uint32_t *const stage = TMA ? pipe.stage(turn) : planes;
        float2 h = load_state(a.states, place_of(u.r0, tile, u.seq), n, u.col, u.valid);
        if (TMA) {
            pipe.wait(turn, parity);
        } else {
            __syncthreads();  // the results of the tile before have left
            fill_plane(stage, a.f, row, u.r1, u.col, u.valid, words, kFill);
            fill_plane(stage + kPlane, a.x, row, u.r1, u.col, u.valid, words, 0u);
            if (gated) fill_plane(stage + 2 * kPlane, a.o, row, u.r1, u.col, u.valid, words, 0u);
            fill_plane(stage + 3 * kPlane, a.dy, row, u.r1, u.col, u.valid, words, 0u);
            __syncthreads();
        }
        const bool work = __any_sync(0xffffffffu, count > 0);
        if (work && count < kLen) mask_run<4>(stage, u.run, u.lane, count, kFill);
        uint32_t *const f = run_of(stage, u.run, u.lane), *const x = run_of(stage + kPlane, u.run, u.lane),
                 *const o = run_of(stage + 2 * kPlane, u.run, u.lane);
        const uint32_t *const d = run_of(stage + 3 * kPlane, u.run, u.lane);
        float2 m[kLen], p;
        runs[turn][u.run][u.lane] = work ? local_run<F16>(f, x, m) : no_run();
        back[turn][u.run][u.lane] = work ? local_back<F16, ACT>(m, d, o, gated) : both(0.f);
        __syncthreads();
        if (TMA && i > 0) {
            if (threadIdx.x == 0) bulk_wait_read();
            fetch(i + 1, turn ^ 1);
        }
#pragma unroll
        for (int r = kRuns - 1; r >= 0; --r) {
            if (r == u.run) p = carry;
            const float4 c = runs[turn][r][u.lane];
            carry = back[turn][r][u.lane] + times(make_float2(c.x, c.y), carry);
        }
        if (work) {
            for (int r = 0; r < u.run; ++r) h = then(h, runs[turn][r][u.lane]);
            float2 before[kLen + 1];  // the state before each step, and after the last
            before[0] = h;
#pragma unroll
            for (int j = 0; j < kLen; ++j) before[j + 1] = step(m[j], before[j], values_of<F16>(x[j * kLanes]));
#pragma unroll
            for (int j = kLen - 1; j >= 0; --j) {
                float2 d_o;
                const Slopes g = slopes<F16, ACT>(m[j], before[j], before[j + 1], f[j * kLanes], x[j * kLanes], gated ? o[j * kLanes] : 0u,
                                                  d[j * kLanes], gated, p, d_o);
                f[j * kLanes] = pack16<F16>(g.df.x, g.df.y);
                x[j * kLanes] = pack16<F16>(g.dx.x, g.dx.y);
                if (gated) o[j * kLanes] = pack16<F16>(d_o.x, d_o.y);
            }
        }
        if (TMA) bulk_fence();
        __syncthreads();
        const Plane *const out[3] = {&a.df, &a.dx, &a.d_o};
        if (TMA && maps.store && row + kTile <= u.r1) {
            if (threadIdx.x == 0) {
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (out[k]->p) bulk_store(&maps.out[k], smem_u32(stage + k * kPlane), u.col0, (int)row);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (out[k]->p) empty_plane(stage + k * kPlane, *out[k], row, u.r1, u.col, u.valid, words);
        }
        parity ^= turn;
        turn ^= 1;
    }
    if (a.d_state && !a.starts && u.run == 0) store_state(a.d_state, u.seq, n, u.col, u.valid, carry);
    if (TMA) pipe_end(pipe);
}

// ---- independent tiles
// What a tile makes of what comes into it: [place][n] of q and of H (or backwards of R).
struct Sum {
    float *factor, *made;
};
// BACK: R from f, o and dy; else H from f and x.
template <bool F16, int ACT, bool BACK, bool TMA>
__global__ void __launch_bounds__(kThreads) tile_sum_kernel(const __grid_constant__ RecurGradArgs a, const __grid_constant__ Tiles maps,
                                                            const Sum sum) {
    __shared__ __align__(128) uint32_t planes[(BACK ? kMostIn : 2) * kPlane];
    __shared__ float4 runs[kRuns][kLanes];
    __shared__ uint64_t full[2];
    __shared__ uint32_t abort_flag;
    const bool words = a.words != 0, gated = BACK && a.o.p != nullptr;
    constexpr uint32_t kFill = F16 ? kKeepAll16 : kKeepAll;
    constexpr int kX = BACK ? 3 : 1;  // the plane of x or dy
    Pipe pipe{planes, full, 0, {&abort_flag, maps.waits.status, maps.waits.timeout_ns}};
    if (TMA) pipe.start();
    pdl_trigger();
    pdl_wait();
    const Unit u(a.at, a.col_tiles, true);
    if (u.tiles == 0) return;
    const int64_t row = (int64_t)u.r0 + (int64_t)u.tile * kTile;
    if (TMA) {
        const bool has[kMostIn] = {true, !BACK, gated, BACK};
        if (threadIdx.x == 0) pipe.load(maps, has, 0, u.col0, (int)row);
        pipe.wait(0, 0);
    } else {
        fill_plane(planes, a.f, row, u.r1, u.col, u.valid, words, kFill);
        fill_plane(planes + kX * kPlane, BACK ? a.dy : a.x, row, u.r1, u.col, u.valid, words, 0u);
        if (gated) fill_plane(planes + 2 * kPlane, a.o, row, u.r1, u.col, u.valid, words, 0u);
        __syncthreads();
    }
    const int count = (int)max(min((int64_t)kLen, u.r1 - row - u.run * kLen), (int64_t)0);
    const bool work = __any_sync(0xffffffffu, count > 0);
    if (work && count < kLen) mask_run<BACK ? 4 : 2>(planes, u.run, u.lane, count, kFill);
    float2 m[kLen];
    const uint32_t *const x = run_of(planes + kX * kPlane, u.run, u.lane);
    float4 mine = work ? local_run<F16>(run_of(planes, u.run, u.lane), x, m) : no_run();
    if (BACK && work) {
        const float2 p = local_back<F16, ACT>(m, x, run_of(planes + 2 * kPlane, u.run, u.lane), gated);
        mine.z = p.x;
        mine.w = p.y;
    }
    runs[u.run][u.lane] = mine;
    __syncthreads();
    if (u.run == 0) {
        float4 all = runs[BACK ? kRuns - 1 : 0][u.lane];
#pragma unroll
        for (int r = 1; r < kRuns; ++r) all = join(all, runs[BACK ? kRuns - 1 - r : r][u.lane]);
        const int64_t place = place_of(u.r0, u.tile, u.seq);
        store_state(sum.factor, place, a.at.n, u.col, u.valid, make_float2(all.x, all.y));
        store_state(sum.made, place, a.at.n, u.col, u.valid, make_float2(all.z, all.w));
    }
    if (TMA) pipe_end(pipe);
}

// Along a sequence's tiles, a column to a lane: what comes into each (starts) and what comes
// out in the end.  Each warp takes a few neighbouring tiles in registers and joins them, the
// warps meet in shared memory, and each goes along its own from what those before it make.
constexpr int kScanWarps = 32, kScanTiles = 8;
template <bool BACK>
__global__ void __launch_bounds__(32 * kScanWarps) tile_scan_kernel(const __grid_constant__ Sequences at, const Sum sum, const float *begin,
                                                                    float *starts, float *end, int col_tiles) {
    __shared__ float2 shares[2][kScanWarps][32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const int seq = blockIdx.x / col_tiles, n = at.n, col = ((int)blockIdx.x - seq * col_tiles) * 32 + lane;
    pdl_trigger();
    pdl_wait();
    int r0, r1;
    at.rows_of(seq, r0, r1);
    const int tiles = (r1 - r0 + kTile - 1) / kTile;
    const bool in = col < n;
    // (`end` may be `begin`: it is written after every thread's last barrier, or by the one that reads it)
    float carry = begin && in ? begin[(int64_t)seq * n + col] : 0.f;
    int turn = 0;
    for (int t0 = 0; t0 < tiles; t0 += kScanWarps * kScanTiles, turn ^= 1) {
        // tile t of the order that is gone along
        auto index = [&](int t) { return place_of(r0, BACK ? tiles - 1 - t : t, seq) * n + col; };
        const int first = t0 + warp * kScanTiles;
        float q[kScanTiles], made[kScanTiles];
#pragma unroll
        for (int i = 0; i < kScanTiles; ++i) {
            q[i] = -0.f;  // keeps all, makes nothing
            made[i] = 0.f;
            if (in && first + i < tiles) {
                q[i] = sum.factor[index(first + i)];
                made[i] = sum.made[index(first + i)];
            }
        }
        float factor = -0.f, all = 0.f;
#pragma unroll
        for (int i = 0; i < kScanTiles; ++i) {
            all = made[i] + times(q[i], all);
            factor = product_of(factor, q[i]);
        }
        shares[turn][warp][lane] = make_float2(factor, all);
        __syncthreads();
        float v = carry;
#pragma unroll 8
        for (int w = 0; w < kScanWarps; ++w) {
            if (w == warp) v = carry;
            const float2 share = shares[turn][w][lane];
            carry = share.y + times(share.x, carry);
        }
#pragma unroll
        for (int i = 0; i < kScanTiles; ++i) {
            if (in && first + i < tiles) starts[index(first + i)] = v;
            v = made[i] + times(q[i], v);
        }
    }
    if (end && in && warp == 0) end[(int64_t)seq * n + col] = carry;
}

// Short sequences: two columns of one to a thread, step by step, kLot steps' loads together.
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
    int r0, r1;
    a.at.rows_of((int)s, r0, r1);
    if (r1 - r0 >= kLong) return;
    float2 h = a.state ? load_state(a.state, s, n, col, valid) : both(0.f);
    if (a.states && r1 > r0) store_state(a.states, place_of(r0, 0, (int)s), n, col, valid, h);
    for (int first = r0; first < r1; first += kLot) {
        uint32_t f[kLot], x[kLot], o[kLot];
#pragma unroll
        for (int i = 0; i < kLot; ++i) {
            if (first + i >= r1) break;
            f[i] = load_pair(place(a.f, first + i, col), valid, words);
            x[i] = load_pair(place(a.x, first + i, col), valid, words);
            if (gated) o[i] = load_pair(place(a.o, first + i, col), valid, words);
        }
#pragma unroll
        for (int i = 0; i < kLot; ++i) {
            if (first + i >= r1) break;
            h = step(minus_rest<F16>(f[i]), h, values_of<F16>(x[i]));
            const float2 y = gated ? h * act2<ACT>(values_of<F16>(o[i])) : h;
            store_pair(place(a.y, first + i, col), valid, words, pack16<F16>(y.x, y.y));
        }
    }
    if (a.last) store_state(a.last, s, n, col, valid, h);
}

// The same backwards: along the lots once for the state before each, then from the last to the first.
template <bool F16, int ACT>
__global__ void __launch_bounds__(256) recur_short_grad_kernel(const __grid_constant__ RecurGradArgs a) {
    const int pairs = (a.at.n + 1) / 2, n = a.at.n;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t s = at / pairs;
    const int col = (int)(at - s * pairs) * 2, valid = min(n - col, 2);
    const bool words = a.words != 0, gated = a.o.p != nullptr;
    pdl_trigger();
    pdl_wait();
    if (s >= a.at.seqs) return;
    int r0, r1;
    a.at.rows_of((int)s, r0, r1);
    if (r1 - r0 >= kLong) return;
    float2 p = a.d_last ? load_state(a.d_last, s, n, col, valid) : both(0.f);
    float2 starts[kLong / kLot];
    uint32_t wf[kLot], wx[kLot];
    const int last = (r1 - r0 - 1) / kLot;  // the last lot
    if (r1 > r0) starts[0] = load_state(a.states, place_of(r0, 0, (int)s), n, col, valid);
    for (int lot = 0; lot < last; ++lot) {
        const int first = r0 + lot * kLot;
#pragma unroll
        for (int i = 0; i < kLot; ++i) {
            wf[i] = load_pair(place(a.f, first + i, col), valid, words);
            wx[i] = load_pair(place(a.x, first + i, col), valid, words);
        }
        float2 h = starts[lot];
#pragma unroll
        for (int i = 0; i < kLot; ++i) h = step(minus_rest<F16>(wf[i]), h, values_of<F16>(wx[i]));
        starts[lot + 1] = h;
    }
    for (int lot = last; r1 > r0 && lot >= 0; --lot) {
        const int first = r0 + lot * kLot;
        uint32_t wo[kLot], wd[kLot];
#pragma unroll
        for (int i = 0; i < kLot; ++i) {
            if (first + i >= r1) break;
            wf[i] = load_pair(place(a.f, first + i, col), valid, words);
            wx[i] = load_pair(place(a.x, first + i, col), valid, words);
            wd[i] = load_pair(place(a.dy, first + i, col), valid, words);
            if (gated) wo[i] = load_pair(place(a.o, first + i, col), valid, words);
        }
        float2 m[kLot], before[kLot + 1];
        before[0] = starts[lot];
#pragma unroll
        for (int i = 0; i < kLot; ++i) {
            if (first + i >= r1) break;
            m[i] = minus_rest<F16>(wf[i]);
            before[i + 1] = step(m[i], before[i], values_of<F16>(wx[i]));
        }
#pragma unroll
        for (int i = kLot - 1; i >= 0; --i) {
            if (first + i >= r1) continue;
            float2 d_o;
            const Slopes g = slopes<F16, ACT>(m[i], before[i], before[i + 1], wf[i], wx[i], wo[i], wd[i], gated, p, d_o);
            if (a.df.p) store_pair(place(a.df, first + i, col), valid, words, pack16<F16>(g.df.x, g.df.y));
            if (a.dx.p) store_pair(place(a.dx, first + i, col), valid, words, pack16<F16>(g.dx.x, g.dx.y));
            if (a.d_o.p) store_pair(place(a.d_o, first + i, col), valid, words, pack16<F16>(d_o.x, d_o.y));
        }
    }
    if (a.d_state) store_state(a.d_state, s, n, col, valid, p);
}

// ---------------------------------------------------------------- host
bool on_words(const emtk_matrix &m, int rows) {
    return !m.d || (reinterpret_cast<uintptr_t>(m.d) % 4 == 0 && (rows <= 1 || m.ld % 2 == 0));
}

// Whether blocks go along whole sequences: three units (32 columns of one) to every two
// SMs, and all of one length, or not so long that one of them would keep the others
// waiting.  20000 rows of 2048 columns, forward and backward: 256 units 107 and 187 us, as
// independent tiles 103 and 212; 64 units 281 and 535, independent 95 and 202; 1024 units (of 1250 rows)
// 59 and 134, independent as with 64.  16896 rows of 498 columns in 88 sequences of unlike lengths:
// both passes 410 us as independent tiles, most of whose places are empty.  Sequences of four tiles
// at most are done before three kernels would be.
// Off TMA's grid a block has no tile ahead: three units to every SM (4 x 5000 steps of 2048 columns in rows
// of 2050: along 206 and 379 us, independent 160 and 368; 10 x 2000: 165 and 317, 9 x 2222 independent 170 and 383).
bool along(bool uniform, bool tma, int rows, int seqs, int col_tiles, int sms) {
    if ((uniform ? rows / seqs : rows) <= 4 * kTile) return true;
    const int64_t units = (int64_t)seqs * col_tiles;
    return (tma ? 2 * units >= 3 * sms : units >= 3 * sms) && (uniform || rows / seqs <= 4 * kTile);
}
// Whether a thread takes a whole sequence, as a tile would be nearly empty: of unlike ones those below
// kLong steps where that is so on average, the others are left to blocks that go along them.  Forward and
// backward, 320 sequences of 1024 columns, of 0 - 8 steps 8.2 and 12.4 us, a tile to each 48 and 128; of
// 0 - 120 steps 64 and 139, 66 and 163; one of 8192 steps and 800 single steps of 2048 columns 142 and 322,
// 273 and 739.  Equal ones: 64 of 16 steps of 2048 columns 5.8 and 10.8 us, a tile to each 20.7 and 57;
// where blocks are no more than the SMs hold at once, tiles are as fast (16 of 16 of 1024: 4.9 and 8.6, 4.2
// and 12.7) and faster for more steps (16 of 32: 8.5 and 16.3, 4.0 and 12.6).
bool step_by_step(bool uniform, int rows, int seqs, int n, int sms) {
    const int length = rows / seqs;
    const bool many = (int64_t)seqs * ((n + kCols - 1) / kCols) > 4 * sms;
    return length <= kLot || (uniform ? length < kLong && many : length <= kLong);
}
int64_t places(int rows, int seqs) { return (int64_t)rows / kTile + seqs; }

// Workspace of independent tiles: (q, H) and, where they are not kept anyway, the starts.
Sum sums_in(void *workspace, int64_t places, int n) {
    float *const p = static_cast<float *>(workspace);
    return {p, p + places * n};
}

constexpr size_t shared_bytes(int planes, bool tma, bool along) { return (size_t)(tma && along ? 2 : 1) * planes * kPlane * 4; }

bool grid_ok(int64_t blocks) { return blocks <= INT32_MAX; }

template <typename Kernel, typename Args>
cudaError_t run_tiles(Kernel kernel, int planes, bool tma, const Args &a, const Tiles &maps, cudaStream_t s) {
    const bool whole = a.starts == nullptr;
    const int64_t blocks =
        (!whole ? places(a.at.rows, a.at.seqs) : a.at.long_only ? (a.at.rows + kLong - 1) / kLong : a.at.seqs) * (int64_t)a.col_tiles;
    if (!grid_ok(blocks)) return cudaErrorInvalidValue;
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3(kThreads), shared_bytes(planes, tma, whole), s, a, maps);
}

// Whether no sequence is left to blocks, with short ones step by step.
bool no_long(const int32_t *offsets, int rows) { return !offsets || rows < kLong; }
// The short sequences; `a` is left with the long ones, `done` if there can be none.
template <typename Args>
cudaError_t run_short(void (*kernel)(const Args), Args &a, bool &done, cudaStream_t s) {
    const int64_t blocks = ((int64_t)a.at.seqs * ((a.at.n + 1) / 2) + 255) / 256;
    if (!grid_ok(blocks)) return cudaErrorInvalidValue;
    const cudaError_t e = launch_pdl(kernel, dim3((unsigned)blocks), dim3(256), 0, s, a);
    done = e != cudaSuccess || no_long(a.at.offsets, a.at.rows);
    a.at.long_only = 1;
    return e;
}

// Each tile's start, by the first two kernels.
template <bool F16, int ACT, bool BACK>
cudaError_t run_starts(const RecurGradArgs &a, const Tiles *maps, void *workspace, const float *begin, float *starts, float *end,
                       cudaStream_t s) {
    const int64_t all = places(a.at.rows, a.at.seqs), blocks = all * a.col_tiles;
    if (!grid_ok(blocks)) return cudaErrorInvalidValue;
    const Sum sum = sums_in(workspace, all, a.at.n);
    const dim3 grid((unsigned)blocks), block(kThreads);
    const cudaError_t e = maps ? launch_pdl(tile_sum_kernel<F16, ACT, BACK, true>, grid, block, 0, s, a, *maps, sum)
                               : launch_pdl(tile_sum_kernel<F16, ACT, BACK, false>, grid, block, 0, s, a, Tiles{}, sum);
    if (e != cudaSuccess) return e;
    return launch_pdl(tile_scan_kernel<BACK>, dim3((unsigned)(a.at.seqs * (int64_t)a.col_tiles)), dim3(32 * kScanWarps), 0, s, a.at, sum,
                      begin, starts, end, a.col_tiles);
}

template <bool F16, int ACT>
cudaError_t run(RecurArgs a, const Tiles *maps, void *workspace, int sms, cudaStream_t s) {
    if (step_by_step(!a.at.offsets, a.at.rows, a.at.seqs, a.at.n, sms)) {
        bool done;
        const cudaError_t e = run_short(recur_short_kernel<F16, ACT>, a, done, s);
        if (done) return e;
    } else if (!along(!a.at.offsets, maps != nullptr, a.at.rows, a.at.seqs, a.col_tiles, sms)) {
        RecurGradArgs g{};
        g.f = a.f;
        g.x = a.x;
        g.at = a.at;
        g.col_tiles = a.col_tiles;
        g.words = a.words;
        float *const starts = a.states ? a.states : sums_in(workspace, places(a.at.rows, a.at.seqs), a.at.n).made + places(a.at.rows, a.at.seqs) * a.at.n;
        const cudaError_t e = run_starts<F16, EMTK_ACT_NONE, false>(g, maps, workspace, a.state, starts, a.last, s);
        if (e != cudaSuccess) return e;
        a.starts = starts;
        a.states = nullptr;
    }
    return maps ? run_tiles(recur_kernel<F16, ACT, true>, 3, true, a, *maps, s) : run_tiles(recur_kernel<F16, ACT, false>, 3, false, a, Tiles{}, s);
}
template <bool F16, int ACT>
cudaError_t run(RecurGradArgs a, const Tiles *maps, void *workspace, int sms, cudaStream_t s) {
    if (step_by_step(!a.at.offsets, a.at.rows, a.at.seqs, a.at.n, sms)) {
        bool done;
        const cudaError_t e = run_short(recur_short_grad_kernel<F16, ACT>, a, done, s);
        if (done) return e;
    } else if (!along(!a.at.offsets, maps != nullptr, a.at.rows, a.at.seqs, a.col_tiles, sms)) {
        float *const starts = sums_in(workspace, places(a.at.rows, a.at.seqs), a.at.n).made + places(a.at.rows, a.at.seqs) * a.at.n;
        const cudaError_t e = run_starts<F16, ACT, true>(a, maps, workspace, a.d_last, starts, a.d_state, s);
        if (e != cudaSuccess) return e;
        a.starts = starts;
    }
    return maps ? run_tiles(recur_grad_kernel<F16, ACT, true>, 4, true, a, *maps, s)
                : run_tiles(recur_grad_kernel<F16, ACT, false>, 4, false, a, Tiles{}, s);
}
template <bool F16, typename Args>
cudaError_t run(const Args &a, const Tiles *maps, void *workspace, int act, int sms, cudaStream_t s) {
    switch (act) {
        case EMTK_ACT_RELU: return run<F16, EMTK_ACT_RELU>(a, maps, workspace, sms, s);
        case EMTK_ACT_GELU: return run<F16, EMTK_ACT_GELU>(a, maps, workspace, sms, s);
        case EMTK_ACT_SILU: return run<F16, EMTK_ACT_SILU>(a, maps, workspace, sms, s);
        case EMTK_ACT_SIGMOID: return run<F16, EMTK_ACT_SIGMOID>(a, maps, workspace, sms, s);
        default: return run<F16, EMTK_ACT_NONE>(a, maps, workspace, sms, s);
    }
}

// Tensor maps of the matrices that are there; `tma`: those that are read lie on TMA's grid.
template <int IN, int OUT>
cudaError_t make_maps(bool &tma, const emtk_nn *nn, Tiles &t, const emtk_matrix *const (&in)[IN], const emtk_matrix *const (&out)[OUT], int rows, int n) {
    t.waits = {nn->status, nn->timeout_ns};
    tma = true;
    for (const emtk_matrix *m : in) tma = tma && (!m->d || mm_operand_ok(m->d, m->ld, rows));
    if (!tma) return cudaSuccess;
    t.store = n % 8 == 0;
    for (const emtk_matrix *m : out) t.store = t.store && (!m->d || mm_operand_ok(m->d, m->ld, rows));
    for (int i = 0; i < IN; ++i)
        if (in[i]->d && !encode_rows(nn, &t.in[i], *in[i], rows, n, kCols, kTile)) return cudaErrorInvalidValue;
    for (int i = 0; t.store && i < OUT; ++i)
        if (out[i]->d && !encode_rows(nn, &t.out[i], *out[i], rows, n, kCols, kTile)) return cudaErrorInvalidValue;
    return cudaSuccess;
}

template <bool F16, int ACT>
cudaError_t init_kernels() {
    cudaError_t e = cudaFuncSetAttribute(recur_kernel<F16, ACT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared_bytes(3, true, true));
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(recur_grad_kernel<F16, ACT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared_bytes(4, true, true));
    return e;
}
template <bool F16>
cudaError_t init_kernels() {
    for (const cudaError_t e : {init_kernels<F16, EMTK_ACT_NONE>(), init_kernels<F16, EMTK_ACT_RELU>(), init_kernels<F16, EMTK_ACT_GELU>(),
                                init_kernels<F16, EMTK_ACT_SILU>(), init_kernels<F16, EMTK_ACT_SIGMOID>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

}  // namespace

cudaError_t init_recur_kernels() {
    const cudaError_t e = init_kernels<false>();
    return e == cudaSuccess ? init_kernels<true>() : e;
}

// An input that only loads of two bytes reach is copied to rows that TMA reads, but for short
// sequences.  An element off the grid, forward and backward, as they lie and copied: 800 x 1000 steps
// of 64 columns 294 and 603 us, 195 and 377; 8 x 512 of 136 24 and 54, 13 and 33; 88 x 192 of 498 43 and
// 129, 44 and 91; 400 x 200 of 32 14 and 22, 15 and 24.  Two elements off it they are read as they lie: the
// first 147 and 351, 189 and 345.
bool recurrence_copies(const emtk_matrix &m, int rows, int n, int seqs, bool uniform, int sms) {
    const bool odd = (reinterpret_cast<uintptr_t>(m.d) | (uintptr_t)m.ld * 2) & 3;
    return seqs > 0 && m.d && odd && !step_by_step(uniform, rows, seqs, n, sms);
}

size_t recurrence_workspace(int rows, int n, int seqs, bool uniform, bool tma, int sms) {
    if (n == 0 || seqs == 0 || step_by_step(uniform, rows, seqs, n, sms)) return 0;
    const bool whole = along(uniform, tma, rows, seqs, (n + kCols - 1) / kCols, sms);
    return whole ? 0 : 3 * sizeof(float) * places(rows, seqs) * n;
}

cudaError_t launch_recurrence(const emtk_recurrence_args &p, void *workspace, const emtk_nn *nn, cudaStream_t s) {
    if (p.n == 0 || p.seqs == 0) return cudaSuccess;
    RecurArgs a{};
    a.f = plane_of(p.f);
    a.x = plane_of(p.x);
    a.o = plane_of(p.o);
    a.y = plane_of(p.y);
    a.at = {p.offsets, p.rows, p.n, p.seqs, p.offsets ? 0 : p.rows / p.seqs, 0};
    a.state = p.state;
    a.last = p.last;
    a.states = p.states;
    a.col_tiles = (p.n + kCols - 1) / kCols;
    a.words = on_words(p.f, p.rows) && on_words(p.x, p.rows) && on_words(p.o, p.rows) && on_words(p.y, p.rows);
    Tiles maps;
    const emtk_matrix *const in[] = {&p.f, &p.x, &p.o}, *const out[] = {&p.y};
    bool tma = false;
    if (!(step_by_step(!p.offsets, p.rows, p.seqs, p.n, nn->sm_count) && no_long(p.offsets, p.rows))) {
        const cudaError_t e = make_maps(tma, nn, maps, in, out, p.rows, p.n);
        if (e != cudaSuccess) return e;
    }
    return p.type == EMTK_TYPE_F16 ? run<true>(a, tma ? &maps : nullptr, workspace, p.act, nn->sm_count, s)
                                   : run<false>(a, tma ? &maps : nullptr, workspace, p.act, nn->sm_count, s);
}

cudaError_t launch_recurrence_grad(const emtk_recurrence_grad_args &p, void *workspace, const emtk_nn *nn, cudaStream_t s) {
    if (p.n == 0 || p.seqs == 0) return cudaSuccess;
    RecurGradArgs a{};
    a.f = plane_of(p.f);
    a.x = plane_of(p.x);
    a.o = plane_of(p.o);
    a.dy = plane_of(p.dy);
    a.df = plane_of(p.df);
    a.dx = plane_of(p.dx);
    a.d_o = plane_of(p.d_o);
    a.at = {p.offsets, p.rows, p.n, p.seqs, p.offsets ? 0 : p.rows / p.seqs, 0};
    a.states = p.states;
    a.d_last = p.d_last;
    a.d_state = p.d_state;
    a.col_tiles = (p.n + kCols - 1) / kCols;
    a.words = on_words(p.dy, p.rows) && on_words(p.f, p.rows) && on_words(p.x, p.rows) && on_words(p.o, p.rows) &&
              on_words(p.df, p.rows) && on_words(p.dx, p.rows) && on_words(p.d_o, p.rows);
    Tiles maps;
    const emtk_matrix *const in[] = {&p.f, &p.x, &p.o, &p.dy}, *const out[] = {&p.df, &p.dx, &p.d_o};
    bool tma = false;
    if (!(step_by_step(!p.offsets, p.rows, p.seqs, p.n, nn->sm_count) && no_long(p.offsets, p.rows))) {
        const cudaError_t e = make_maps(tma, nn, maps, in, out, p.rows, p.n);
        if (e != cudaSuccess) return e;
    }
    return p.type == EMTK_TYPE_F16 ? run<true>(a, tma ? &maps : nullptr, workspace, p.act, nn->sm_count, s)
                                   : run<false>(a, tma ? &maps : nullptr, workspace, p.act, nn->sm_count, s);
}

}  // namespace emtk
