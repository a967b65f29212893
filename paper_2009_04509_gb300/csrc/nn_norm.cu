// Residual norms: the seam between two blocks, and its gradients.
//
//   v = D post(b);  y = s r + g v;  h = pre(y)
//   post(b) = (b - mean) / sqrt(mean((b - mean)^2) + eps) w + c   (mean 0 for RMS)
//
// A row is held in the registers of a group of threads, eight neighbouring columns to a
// piece, so each matrix is read once and every output written once; variances are of the
// centred values.  HBM bounds the forward pass (8 bytes a value in 16 bits), the call a
// single row: 16384 x 4096 in bf16 with both norms and a gate 85.9 us, 6.25 TB/s (0.92 of a
// copy's rate); one row 3.4 us.
//
// Gradients.  With x^ = (x - mean) / std and q = w d of an output's gradient d, a norm's
// input has the gradient (q - mean(q) - x^ mean(q x^)) / std (mean(q) not for RMS).  One kernel
// goes along rows and writes the inputs' gradients (12 bytes a value) and a few numbers of each
// row, from which another, along columns, adds the parameters' and the gate's (up to 8 bytes a
// value again; in one kernel, each thread adding its columns row by row, the four barriers
// of a row and its sums in shared memory took three times as long).  Sums of slices of
// rows are joined in order, so results do not depend on timing.  16384 x 4096, both norms' and
// the gate's sums: 159 us of rows (5.1 TB/s) and 126 of sums; 8192 x 5461, off the grid, where
// shifting pieces into place bounds both: 189 and 108 (8192 x 5464: 115 and 92).
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_pieces.cuh"
#include "nn_ptx.cuh"

namespace emtk {
namespace {

constexpr int kMaxWarps = 32, kMostGroups = 8, kGroupThreads = 128;

struct NormArgs {
    int kind;
    float eps;
    Param weight, bias;
};
NormArgs norm_args(const emtk_norm &n) {
    const int f32 = n.param_type == EMTK_TYPE_F32;
    return {n.kind, n.eps, param_of(n.weight, f32), param_of(n.bias, f32)};
}

// The sums of K (1, 2 or 4) values over a group's threads, in every thread.  In a warp
// each exchange halves the values that a lane still holds, and then the lanes; the warps'
// sums are read back with one value to a lane and added the same way: a sum costs a third
// of the shuffles that one tree for each value would.  `turn` alternates between two
// buffers, so that one barrier a call is enough.
// A group: the threads of a row, blockDim.x of them, blockDim.y groups to a block (one,
// where a row has more than kGroupThreads).
struct Reduction {
    float *buffer;  // [2][4 * kMaxWarps] of the block, from the group's place on
    int tid, warps, turn, width;  // width: lanes of a row, if it has less than a warp
    bool grouped;
    __device__ __forceinline__ void sync() const {
        if (grouped)
            asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.y + 1), "r"(32 * warps) : "memory");
        else
            __syncthreads();
    }
};
template <int K>
__device__ __forceinline__ void row_sum(float (&v)[K], Reduction &b) {
    const int lane = b.tid & 31;
    float x = v[0];
    if constexpr (K == 4) {  // lane & 3 keeps its value
        const bool upper = (lane & 2) != 0;
        const float k0 = upper ? v[2] : v[0], k1 = upper ? v[3] : v[1];
        const float s0 = upper ? v[0] : v[2], s1 = upper ? v[1] : v[3];
        const float a = k0 + __shfl_xor_sync(0xffffffffu, s0, 2), c = k1 + __shfl_xor_sync(0xffffffffu, s1, 2);
        const bool odd = (lane & 1) != 0;
        x = (odd ? c : a) + __shfl_xor_sync(0xffffffffu, odd ? a : c, 1);
    } else if constexpr (K == 2) {
        const bool odd = (lane & 1) != 0;
        x = (odd ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, odd ? v[0] : v[1], 1);
    }
#pragma unroll
    for (int d = K; d < 32; d *= 2)
        if (d < b.width) x += __shfl_xor_sync(0xffffffffu, x, d);
    if (b.warps > 1) {
        float *const buffer = b.buffer + b.turn * 4 * kMaxWarps;
        if (lane < K) buffer[b.tid / 32 * K + lane] = x;
        b.sync();
        x = 0.f;
        for (int i = lane; i < b.warps * K; i += 32) x += buffer[i];
#pragma unroll
        for (int d = K; d < 32; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
        b.turn ^= 1;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = K == 1 ? x : __shfl_sync(0xffffffffu, x, k, b.width);
}

__device__ __forceinline__ float sum_of(const Eight &e) {
    const float2 a = (e.v[0] + e.v[1]) + (e.v[2] + e.v[3]);
    return a.x + a.y;
}
__device__ __forceinline__ float dot(const Eight &a, const Eight &b) {
    float2 s = a.v[0] * b.v[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) s = fma2(a.v[i], b.v[i], s);
    return s.x + s.y;
}
// e - mean, in the columns that are there.
__device__ __forceinline__ void centre(Eight &e, float mean, int c, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) e.v[i] = e.v[i] - both(mean);
    if (c + kPiece > n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) e.v[i] = make_float2(c + 2 * i < n ? e.v[i].x : 0.f, c + 2 * i + 1 < n ? e.v[i].y : 0.f);
    }
}
__device__ __forceinline__ Eight operator*(const Eight &a, const Eight &b) {
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = a.v[i] * b.v[i];
    return r;
}
__device__ __forceinline__ Eight operator*(const Eight &a, float b) {
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = a.v[i] * both(b);
    return r;
}
__device__ __forceinline__ Eight operator+(const Eight &a, const Eight &b) {
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = a.v[i] + b.v[i];
    return r;
}

constexpr int kMostInputs = 4, kMostStages = 2;
struct Inputs {
    Rows16 in[kMostInputs];
    int m, n;
    int row_bytes, stages;  // of kBulk: room for one row in shared memory, rows on their way
};
// Room for a row: up to 14 bytes before it, whole pieces, and the one after the last.
int bulk_row_bytes(int n) { return (2 * n + 14 + 15) / 16 * 16 + 16; }

struct Waits {  // of the kernels' bounded waits
    int *status;
    int64_t timeout_ns;
};

// How a group of threads has its row.
//   kDirect   one of a block's, two pieces a thread, on the 16-byte grid and of whole pieces
//   kDirectAny the same, anywhere
//   kSmall    several to a block (and to a warp, where they are short), a piece a thread, on the
//             grid and of whole pieces
//   kSmallAny the same, anywhere
//   kBulk     (the gradients) a block goes from row to row, two pieces a thread: a row of each matrix is copied
//             to shared memory, a row or two ahead, so that many rows are on their way
//             without a register
//   kBulkAny  the same, anywhere: in the aligned 16-byte pieces that it lies in, shifted into
//             place from there.  Rows whose outer pieces would reach beyond the matrix
//             are copied by elements.
// A thread's pieces are tid and tid + threads; but for the last of a thread, they are whole.
enum Kind : int { kDirect, kDirectAny, kSmall, kSmallAny, kBulk, kBulkAny };
constexpr bool is_bulk(Kind k) { return k == kBulk || k == kBulkAny; }

template <bool F16, Kind KIND, int COUNT>  // COUNT: matrices
struct RowIo {
    static constexpr int C = KIND == kSmall || KIND == kSmallAny ? 1 : 2;
    static constexpr bool ODD = KIND == kDirectAny || KIND == kSmallAny || KIND == kBulkAny;
    const Inputs &a;
    int64_t row;
    int tid, threads;
    bool last;  // the last piece is this thread's, or beyond the row
    bool live;  // false: a row that is not there, in a warp of rows that are
    // kBulk; unset elsewhere
    uint8_t *stages;
    uint64_t *full;
    Guard guard;
    uint32_t phases = 0;
    int stage = 0;
    bool ok = true;

    __device__ __forceinline__ explicit RowIo(const Inputs &inputs) : a(inputs) {
        tid = threadIdx.x;
        threads = blockDim.x;
        row = KIND == kSmall || KIND == kSmallAny ? (int64_t)blockIdx.x * blockDim.y + threadIdx.y : (int64_t)blockIdx.x;
        last = column(C - 1) + kPiece > a.n;
        live = row < a.m;
        if (C == 1 && threads < 32) row = min(row, (int64_t)a.m - 1);  // its warp's exchanges need all lanes
    }
    // What kBulk has besides.
    __device__ __forceinline__ RowIo(const Inputs &inputs, uint8_t *shared, uint64_t *bars, uint32_t *abort_flag, const Waits &w) : RowIo(inputs) {
        stages = shared;
        full = bars;
        guard = {abort_flag, w.status, w.timeout_ns};
        if (is_bulk(KIND)) {
            if (tid == 0) {
                for (int i = 0; i < kMostStages; ++i) mbar_init(smem_u32(full + i), 1);
                *abort_flag = 0;
                fence_mbar_init();
            }
            __syncthreads();
        }
    }
    __device__ __forceinline__ int column(int k) const { return (k * threads + tid) * kPiece; }

    // ---- kBulk: rows on their way
    __device__ __forceinline__ int head(int i, int64_t r) const { return ODD ? (int)(reinterpret_cast<uintptr_t>(a.in[i].row(r)) % 16) : 0; }
    __device__ __forceinline__ int bytes(int i, int64_t r) const { return (head(i, r) + 2 * a.n + 15) / 16 * 16; }
    __device__ __forceinline__ uint8_t *place(int s, int i) const { return stages + (s * COUNT + i) * a.row_bytes; }
    __device__ __forceinline__ bool by_elements(int64_t r) const {
        if constexpr (ODD) {
            if (r >= kPiece && r < a.m - kPiece) return false;  // the 14 bytes around are of rows between
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                if (!a.in[i].p) continue;
                const int64_t first = r * a.in[i].row_bytes - head(i, r), end = (a.m - 1) * a.in[i].row_bytes + 2 * (int64_t)a.n;
                if (first < 0 || first + bytes(i, r) > end) return true;
            }
        }
        return false;
    }
    __device__ __forceinline__ void fetch(int64_t r, int s) const {  // one thread
        if (r >= a.m || by_elements(r)) return;
        const uint32_t bar = smem_u32(full + s);
        uint32_t all = 0;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) all += a.in[i].p ? (uint32_t)bytes(i, r) : 0u;
        mbar_expect_tx(bar, all);
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (a.in[i].p)
                bulk_load(smem_u32(place(s, i)), reinterpret_cast<const uint8_t *>(a.in[i].row(r)) - head(i, r), bytes(i, r), bar);
    }
    __device__ __forceinline__ void begin() const {
        if (is_bulk(KIND) && tid == 0)
            for (int i = 0; i < a.stages; ++i) fetch(row + (int64_t)i * gridDim.x, i);
    }
    // The row's arrival; all threads.
    __device__ __forceinline__ void wait() {
        if (!is_bulk(KIND)) return;
        if (by_elements(row)) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                if (!a.in[i].p) continue;
                uint16_t *const to = reinterpret_cast<uint16_t *>(place(stage, i) + head(i, row));
                for (int c = tid; c < a.n; c += threads) to[c] = a.in[i].row(row)[c];
            }
            bulk_fence();
            __syncthreads();
        } else {
            if (ok) ok = wait_bounded(smem_u32(full + stage), (phases >> stage) & 1u, guard);
            phases ^= 1u << stage;
        }
    }
    // Every thread has taken its pieces, and met the others since: the stage may be filled again.
    __device__ __forceinline__ void release() {
        if (!is_bulk(KIND)) return;
        if (tid == 0) fetch(row + (int64_t)a.stages * gridDim.x, stage);
        if (++stage == a.stages) stage = 0;
    }
    __device__ __forceinline__ bool next() {  // to the block's next row
        if (!is_bulk(KIND)) return false;
        row += gridDim.x;
        return row < a.m;
    }
    __device__ __forceinline__ void end() const {
        if (!is_bulk(KIND) || ok) return;
        const uint64_t t0 = global_timer_ns();  // copies in flight land within microseconds: leave them a millisecond
        while (global_timer_ns() - t0 < 1000000u) {
        }
    }

    // A matrix' pieces, columns from n on 0.
    __device__ __forceinline__ void load(int which, uint32_t (&w)[C][4]) const {
#pragma unroll
        for (int k = 0; k < C; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[k][i] = 0u;
        if (!a.in[which].p) return;
        if constexpr (KIND == kBulk) {
            const uint4 *const p = reinterpret_cast<const uint4 *>(place(stage, which)) + tid;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (k == C - 1 && last) continue;
                const uint4 x = p[k * threads];
                w[k][0] = x.x, w[k][1] = x.y, w[k][2] = x.z, w[k][3] = x.w;
            }
        } else if constexpr (KIND == kBulkAny) {
            const uint4 *const base = reinterpret_cast<const uint4 *>(place(stage, which));
            const int halves = head(which, row) / 2, most = (a.n - 1) / kPiece;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const uint4 *const p = base + min(k * threads + tid, most);
                const uint4 lo = p[0];
                if (halves) {
                    const uint4 hi = p[1];
                    const uint32_t x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                    shift_words(x, halves, w[k]);
                } else {
                    w[k][0] = lo.x, w[k][1] = lo.y, w[k][2] = lo.z, w[k][3] = lo.w;
                }
            }
            if (last) {
                const int left = a.n - column(C - 1);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[C - 1][i] &= (2 * i < left ? 0xffffu : 0u) | (2 * i + 1 < left ? 0xffff0000u : 0u);
            }
        } else if constexpr (ODD) {
            Piece16<true> x[C];
#pragma unroll
            for (int k = 0; k < C; ++k) {
                x[k].clear();
                if (column(k) < a.n) x[k].load(a.in[which], row, column(k), a.m, a.n);
            }
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (x[k].halves) {
                    shift_words(x[k].x, x[k].halves, w[k]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[k][i] = x[k].x[i];
                }
            }
        } else {
            const uint4 *const p = reinterpret_cast<const uint4 *>(a.in[which].row(row)) + tid;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (k == C - 1 && last) continue;
                const uint4 x = p[k * threads];
                w[k][0] = x.x, w[k][1] = x.y, w[k][2] = x.z, w[k][3] = x.w;
            }
        }
    }
    // A vector's columns of piece k; 0 from n on.
    __device__ __forceinline__ Eight param(const Param &p, int k) const {
        return param8<F16>(p, column(k), a.n, k < C - 1 || !last);
    }
    __device__ __forceinline__ void store(const Rows16 &to, int k, const Eight &e) const {
        uint32_t w[4];
        words8<F16>(e, w);
        if constexpr (C == 1 && ODD) {
            const int lanes = min(32, threads), run = tid / lanes * lanes * kPiece;
            store_run<true>(to.row(row) + run, live ? max(0, min(a.n - run, lanes * kPiece)) : 0, w, lanes, tid & (lanes - 1));
        } else if constexpr (ODD) {
            const int run = (k * threads + (tid & ~31)) * kPiece;
            store_run<true>(to.row(row) + run, max(0, min(a.n - run, 32 * kPiece)), w, 32, tid & 31);
        } else if ((k < C - 1 || !last) && live) {
            reinterpret_cast<uint4 *>(to.row(row))[k * threads + tid] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

// x becomes norm(x) weight + bias.
template <bool F16, typename Io>
__device__ __forceinline__ void normalise(const NormArgs &a, Eight (&x)[Io::C], const Io &io, float inverse_n, Reduction &b) {
    if (a.kind == EMTK_NORM_LAYER) {
        float sum[1] = {sum_of(x[0])};
        if (Io::C > 1) sum[0] += sum_of(x[Io::C - 1]);
        row_sum(sum, b);
#pragma unroll
        for (int k = 0; k < Io::C; ++k) centre(x[k], sum[0] * inverse_n, k < Io::C - 1 ? 0 : io.column(k), io.a.n);
    }
    float square[1] = {dot(x[0], x[0])};
    if (Io::C > 1) square[0] += dot(x[Io::C - 1], x[Io::C - 1]);
    row_sum(square, b);
    const float r = rsqrtf(fmaf(square[0], inverse_n, a.eps));
#pragma unroll
    for (int k = 0; k < Io::C; ++k) {
        x[k] = x[k] * r;
        if (a.weight.p) x[k] = x[k] * io.param(a.weight, k);
        if (a.bias.p) x[k] = x[k] + io.param(a.bias, k);
    }
}

enum SeamInput : int { kInResidual, kInBlock };
struct SeamArgs {
    Inputs in;
    Rows16 gate, y, h;
    NormArgs post, pre;
    Drop drop;
    float scale, inverse_n;
    int gate_every, gate_vec;  // gate_vec: its rows are on 16 bytes
};

template <bool F16, Kind KIND, int THREADS>
__global__ void __launch_bounds__(THREADS) residual_norm_kernel(const __grid_constant__ SeamArgs a) {
    __shared__ float buffer[2 * 4 * kMaxWarps];
    using Io = RowIo<F16, KIND, 2>;
    constexpr int C = Io::C;
    const Io io(a.in);
    constexpr bool kGrouped = KIND == kSmall || KIND == kSmallAny;
    Reduction reduction{buffer + (kGrouped ? threadIdx.y * (io.threads / 32) * 4 : 0), io.tid, io.threads / 32, 0,
                        kGrouped ? min(32, io.threads) : 32, kGrouped};
    pdl_trigger();
    pdl_wait();
    if (io.row >= a.in.m) return;  // (a whole warp)
    const uint64_t offset = a.drop.below ? drop_offset(a.drop) : 0u;
    uint32_t wb[C][4], wr[C][4];
    io.load(kInBlock, wb);
    io.load(kInResidual, wr);
    Eight v[C];
#pragma unroll
    for (int k = 0; k < C; ++k) v[k] = values8<F16>(wb[k]);
    if (a.post.kind != EMTK_NORM_NONE) normalise<F16>(a.post, v, io, a.inverse_n, reduction);
    const Param gate{a.gate.p ? a.gate.row((int)io.row / a.gate_every) : nullptr, 0, a.gate_vec};
#pragma unroll
    for (int k = 0; k < C; ++k) {
        if (a.drop.below) dropped(a.drop, offset, (uint32_t)io.row, (uint32_t)(k * io.threads + io.tid), v[k]);
        if (a.gate.p) v[k] = v[k] * io.param(gate, k);
        const Eight r = values8<F16>(wr[k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[k].v[i] = fma2(r.v[i], both(a.scale), v[k].v[i]);
        if (a.y.p) io.store(a.y, k, v[k]);
    }
    if (a.pre.kind != EMTK_NORM_NONE) {
        normalise<F16>(a.pre, v, io, a.inverse_n, reduction);
#pragma unroll
        for (int k = 0; k < C; ++k) io.store(a.h, k, v[k]);
    }
}

// ---------------------------------------------------------------- gradients
enum GradInput : int { kInY, kInDh, kInOut, kInDy };  // kInOut: the block's output

// What the columns' kernel needs of a row: of y and of the block's output the mean and
// 1 / std, and of q = weight * dh the mean and, over std, the mean of q y^.
struct RowStats {
    float mean_y, ry, q_mean, qy, mean_b, rb, unused[2];
};

struct SeamGradArgs {
    Inputs in;  // y, dh, block, dy
    Rows16 gate, d_residual, d_block;
    NormArgs post, pre;
    Drop drop;
    float scale, inverse_n;
    int gate_every, gate_vec;  // gate_vec: its rows are on 16 bytes
    RowStats *stats;  // null: no sums are wanted
};

template <bool F16, Kind KIND, int THREADS, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS) residual_norm_grad_kernel(const __grid_constant__ SeamGradArgs a, const Waits waits) {
    extern __shared__ __align__(128) uint8_t rows[];
    __shared__ float buffer[2 * 4 * kMaxWarps];
    __shared__ uint64_t full[kMostStages];
    __shared__ uint32_t abort_flag;
    using Io = RowIo<F16, KIND, 4>;
    constexpr int C = Io::C;
    Io io(a.in, rows, full, &abort_flag, waits);
    constexpr bool kGrouped = KIND == kSmall || KIND == kSmallAny;
    Reduction reduction{buffer + (kGrouped ? threadIdx.y * (io.threads / 32) * 4 : 0), io.tid, io.threads / 32, 0,
                        kGrouped ? min(32, io.threads) : 32, kGrouped};
    const bool pre = a.pre.kind != EMTK_NORM_NONE, post = a.post.kind != EMTK_NORM_NONE;
    const bool pre_mean = a.pre.kind == EMTK_NORM_LAYER, post_mean = a.post.kind == EMTK_NORM_LAYER;
    const int n = a.in.n;
    pdl_trigger();
    pdl_wait();
    if (io.row >= a.in.m) return;  // (a whole warp)
    io.begin();
    const uint64_t offset = a.drop.below ? drop_offset(a.drop) : 0u;
    do {
        io.wait();
        uint32_t w[C][4], wt[C][4];
        Eight y[C], q[C], b[C];
        io.load(kInY, w);
#pragma unroll
        for (int k = 0; k < C; ++k) y[k] = values8<F16>(w[k]);
        io.load(kInDh, w);
#pragma unroll
        for (int k = 0; k < C; ++k) q[k] = values8<F16>(w[k]);
        io.load(kInOut, w);
#pragma unroll
        for (int k = 0; k < C; ++k) b[k] = values8<F16>(w[k]);
        io.load(kInDy, wt);
        if (is_bulk(KIND)) {
            __syncthreads();
            io.release();
        }
        RowStats stats{};
        stats.rb = 1.f;
        if (pre_mean || post_mean) {
            float v[2] = {};
#pragma unroll
            for (int k = 0; k < C; ++k) {
                v[0] += sum_of(y[k]);
                v[1] += sum_of(b[k]);
            }
            row_sum(v, reduction);
            stats.mean_y = pre_mean ? v[0] * a.inverse_n : 0.f;
            stats.mean_b = post_mean ? v[1] * a.inverse_n : 0.f;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (pre_mean) centre(y[k], stats.mean_y, k < C - 1 ? 0 : io.column(k), n);
                if (post_mean) centre(b[k], stats.mean_b, k < C - 1 ? 0 : io.column(k), n);
            }
        }
        if (a.pre.weight.p) {
#pragma unroll
            for (int k = 0; k < C; ++k) q[k] = q[k] * io.param(a.pre.weight, k);
        }
        if (pre || post) {
            float v[4] = {};  // squares of y and b, q, q y
#pragma unroll
            for (int k = 0; k < C; ++k) {
                v[0] += dot(y[k], y[k]);
                v[1] += dot(b[k], b[k]);
                v[2] += sum_of(q[k]);
                v[3] += dot(q[k], y[k]);
            }
            row_sum(v, reduction);
            if (pre) stats.ry = rsqrtf(fmaf(v[0], a.inverse_n, a.pre.eps));
            if (post) stats.rb = rsqrtf(fmaf(v[1], a.inverse_n, a.post.eps));
            stats.q_mean = pre_mean ? v[2] * a.inverse_n : 0.f;
            stats.qy = v[3] * a.inverse_n * stats.ry * stats.ry;
        }
        if (a.stats && io.tid == 0 && io.live) a.stats[io.row] = stats;
        const Param gate{a.gate.p ? a.gate.row((int)io.row / a.gate_every) : nullptr, 0, a.gate_vec};
        float u[2] = {};  // the sums for the block's norm
#pragma unroll
        for (int k = 0; k < C; ++k) {
            Eight t = values8<F16>(wt[k]);
            if (pre) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    t.v[i] = fma2(q[k].v[i] - fma2(y[k].v[i], both(stats.qy), both(stats.q_mean)), both(stats.ry), t.v[i]);
            }
            if (a.d_residual.p) io.store(a.d_residual, k, t * a.scale);
            if (!a.d_block.p) continue;
            if (a.drop.below) dropped(a.drop, offset, (uint32_t)io.row, (uint32_t)(k * io.threads + io.tid), t);
            if (k == C - 1 && io.last) centre(t, 0.f, io.column(k), n);
            if (a.gate.p) t = t * io.param(gate, k);
            if (a.post.weight.p) t = t * io.param(a.post.weight, k);
            q[k] = t;
            b[k] = b[k] * stats.rb;  // now normalised
            u[0] += sum_of(t);
            u[1] += dot(t, b[k]);
        }
        if (a.d_block.p) {
            float mean = 0.f, along = 0.f;
            if (post) {
                row_sum(u, reduction);
                mean = post_mean ? u[0] * a.inverse_n : 0.f;
                along = u[1] * a.inverse_n;
            }
#pragma unroll
            for (int k = 0; k < C; ++k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) q[k].v[i] = (q[k].v[i] - fma2(b[k].v[i], both(along), both(mean))) * both(stats.rb);
                io.store(a.d_block, k, q[k]);
            }
        }
    } while (io.next());
    io.end();
}

// ---- column sums: dw_pre, db_pre, dw_post, db_post, d_gate
enum Sum : int { kSumPreW, kSumPreB, kSumPostW, kSumPostB, kSumGate, kSums };

// Slices of rows: `parts` of a gate row's rows each, or, with parts = 1, `groups_each`
// whole gate rows.
struct Slices {
    int count, parts, groups_each;
    int rows;  // of a part
    __device__ __forceinline__ void range(int slice, int gate_every, int m, int64_t &r0, int64_t &r1) const {
        if (parts > 1) {
            const int64_t begin = (int64_t)(slice / parts) * gate_every, at = (int64_t)(slice % parts) * rows;
            const int64_t end = min(begin + gate_every, (int64_t)m);
            r0 = min(begin + at, end);
            r1 = min(begin + at + rows, end);
        } else {
            r0 = min((int64_t)slice * groups_each * gate_every, (int64_t)m);
            r1 = min(r0 + (int64_t)groups_each * gate_every, (int64_t)m);
        }
    }
};

struct SumArgs {
    SeamGradArgs g;
    Slices slices;
    float *partial[kSums];  // [slices][n] sums, or the result itself; null: not wanted
    float *gate_out;        // of whole gate rows: d_gate
    int64_t gate_ld;
};

constexpr int kSumBlocks = 3, kSumBlocksPre = 5;  // of an SM at once
constexpr int kSumThreads = 128, kSumRows = kSumThreads / 32;

// How rows lie: on the 16-byte grid; off it, but all matrices' alike; anyhow.
//   kAlike: the row 8 rows on lies as this one does, so a warp that takes every eighth row has
//   its lanes' aligned 16 bytes at the same columns in each, c .. c + 7 with c = -shift of 8,
//   and nothing is shifted into place: only the sums are, once, when they are joined.
//   (8192 x 5461, as kAny: 290 us of such a call, 340 with fewer blocks at once.)
enum Lie : int { kGrid, kAlike, kAny };
constexpr int kAlikeColumns = 31 * kPiece;  // of a block: its 32 lanes' pieces hold them at any shift

template <Lie LIE>
struct SumPiece {
    Piece16<LIE == kAny> w;
    __device__ __forceinline__ void clear() { w.clear(); }
    __device__ __forceinline__ void load(const Rows16 &a, int64_t row, int c, int m, int n) {
        if constexpr (LIE == kAlike) {
            // what lies around a row is of its neighbours, but for the first and last rows'
            if ((c >= 0 || row >= kPiece) && (c + kPiece <= n || row < m - kPiece)) {
                const uint4 x = *reinterpret_cast<const uint4 *>(a.row(row) + c);
                w.x[0] = x.x, w.x[1] = x.y, w.x[2] = x.z, w.x[3] = x.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) w.x[i] = 0u;
#pragma unroll
                for (int i = 0; i < kPiece; ++i)
                    if (c + i >= 0 && c + i < n) w.x[i / 2] |= (uint32_t)a.row(row)[c + i] << (16 * (i % 2));
            }
        } else {
            w.load(a, row, c, m, n);
        }
    }
    template <bool F16>
    __device__ __forceinline__ Eight values() const {
        return w.template values<F16>();
    }
};
template <bool F16, Lie LIE>
__device__ __forceinline__ Eight sum_param(const Param &p, int c, int n) {
    if constexpr (LIE == kAlike) {
        float v[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            v[i] = 0.f;
            if (c + i < 0 || c + i >= n) continue;
            v[i] = p.f32 ? __ldg(static_cast<const float *>(p.p) + c + i) : from16<F16>(__ldg(static_cast<const uint16_t *>(p.p) + c + i));
        }
        Eight e;
#pragma unroll
        for (int i = 0; i < 4; ++i) e.v[i] = make_float2(v[2 * i], v[2 * i + 1]);
        return e;
    } else {
        return param8<F16>(p, c, n, c + kPiece <= n);
    }
}

// The sums of the block's warps for its columns c0 .. (`columns` of them, below n), in order, to
// `to`; shift: columns before c0 that the warp's pieces begin at.
__device__ __forceinline__ void flush_sum(Eight &e, float (*shared)[33 * kPiece], float *to, int c0, int columns, int shift, int n) {
    __syncthreads();
    float *const mine = shared[threadIdx.x / 32] + threadIdx.x % 32 * kPiece + kPiece - shift;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mine[2 * i] = e.v[i].x;
        mine[2 * i + 1] = e.v[i].y;
    }
    __syncthreads();
#pragma unroll
    for (int c = threadIdx.x; c < 32 * kPiece; c += kSumThreads) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < kSumRows; ++r) sum += shared[r][kPiece + c];
        if (c < columns && c0 + c < n) to[c0 + c] = sum;
    }
    e.fill(0.f);
}

// A block takes 256 columns and a slice's rows, a warp every fourth of them (kAlike: 248 columns, a
// warp every eighth row, and two blocks share a slice), a piece to a lane.  BLOCK: sums
// over the block's output (all inputs are read); else of the norm after it alone (y and dh).
template <bool F16, Lie LIE, bool BLOCK>
__global__ void __launch_bounds__(kSumThreads, BLOCK ? kSumBlocks : kSumBlocksPre) residual_norm_sum_kernel(const __grid_constant__ SumArgs a) {
    __shared__ float shared[kSumRows][33 * kPiece];
    const SeamGradArgs &g = a.g;
    const int n = g.in.n, m = g.in.m, slice = blockIdx.y;
    constexpr int kColumns = LIE == kAlike ? kAlikeColumns : 32 * kPiece, kStep = LIE == kAlike ? 8 : kSumRows;
    const int phase = threadIdx.x / 32 + (LIE == kAlike ? kSumRows * (int)blockIdx.z : 0);  // of the warp's rows
    const int shift = LIE == kAlike ? (int)(reinterpret_cast<uintptr_t>(g.in.in[BLOCK ? kInOut : kInY].row(phase)) % 16) / 2 : 0;
    const int c0 = blockIdx.x * kColumns, c = c0 + (int)(threadIdx.x % 32) * kPiece - shift;
    const bool in = c < n && c < c0 + kColumns, pre = g.pre.kind != EMTK_NORM_NONE;
    pdl_trigger();
    pdl_wait();
    int64_t r0, r1;
    a.slices.range(slice, g.gate_every, m, r0, r1);
    Eight sum[BLOCK ? kSums : 2], weight, post_weight, post_bias;
#pragma unroll
    for (Eight &e : sum) e.fill(0.f);
    weight.fill(1.f);
    post_weight.fill(1.f);
    post_bias.fill(0.f);
    if (in && g.pre.weight.p) weight = sum_param<F16, LIE>(g.pre.weight, c, n);
    if (BLOCK && in && g.post.weight.p) post_weight = sum_param<F16, LIE>(g.post.weight, c, n);
    if (BLOCK && in && g.post.bias.p) post_bias = sum_param<F16, LIE>(g.post.bias, c, n);
    const uint64_t offset = BLOCK && g.drop.below ? drop_offset(g.drop) : 0u;
    // a gate row's rows after another's, where their sums are apart; all at once where only the
    // gate that they are multiplied with changes
    const bool one_gate = a.gate_out || a.slices.parts > 1 || a.slices.groups_each == 1;
    for (int64_t begin = r0; begin < r1;) {
        const int group = (int)begin / g.gate_every;
        const int64_t end = a.gate_out ? min((int64_t)(group + 1) * g.gate_every, r1) : r1;
        Eight gate;
        gate.fill(1.f);
        if (BLOCK && g.gate.p && in && one_gate) gate = sum_param<F16, LIE>({g.gate.row(group), 0, g.gate_vec}, c, n);
        SumPiece<LIE> wy, wd, wb, wt;
        float4 s;
        float2 s2;
        auto fetch = [&](int64_t row) {
            s = __ldg(reinterpret_cast<const float4 *>(g.stats + row));
            if (BLOCK) s2 = __ldg(reinterpret_cast<const float2 *>(g.stats + row) + 2);
            if (!in) return;
            if (pre) wy.load(g.in.in[kInY], row, c, m, n);
            if (pre) wd.load(g.in.in[kInDh], row, c, m, n);
            if (BLOCK) wb.load(g.in.in[kInOut], row, c, m, n);
            if (BLOCK && g.in.in[kInDy].p) wt.load(g.in.in[kInDy], row, c, m, n);
        };
        wy.clear();
        wd.clear();
        wb.clear();
        wt.clear();
        int64_t row = LIE == kAlike ? begin + ((phase - (int)begin) & 7) : begin + phase;
        if (row < end) fetch(row);
        for (; row < end; row += kStep) {
            Eight y = wy.template values<F16>(), d = wd.template values<F16>();
            Eight b = wb.template values<F16>(), t = wt.template values<F16>();
            const float mean_y = s.x, ry = s.y, q_mean = s.z, qy = s.w, mean_b = s2.x, rb = s2.y;
            if (row + kStep < end) fetch(row + kStep);
            if (pre) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y.v[i] = y.v[i] - both(mean_y);
                    sum[kSumPreW].v[i] = fma2(d.v[i], y.v[i] * both(ry), sum[kSumPreW].v[i]);
                    sum[kSumPreB].v[i] = sum[kSumPreB].v[i] + d.v[i];
                    if (BLOCK) t.v[i] = fma2(d.v[i] * weight.v[i] - fma2(y.v[i], both(qy), both(q_mean)), both(ry), t.v[i]);
                }
            }
            if constexpr (BLOCK) {
                if (g.drop.below) {
                    uint32_t x[8], z[4];
                    drop_numbers(g.drop, offset, (uint32_t)row, (uint32_t)(c >> 3), x);
                    if (LIE == kAlike && shift) {  // the piece is of two pieces' columns
                        drop_numbers(g.drop, offset, (uint32_t)row, (uint32_t)(c >> 3) + 1u, x + 4);
                        shift_words(x, c & 7, z);
                        dropped_by(g.drop, z, t);
                    } else {
                        dropped_by(g.drop, x, t);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    b.v[i] = (b.v[i] - both(mean_b)) * both(rb);
                    sum[kSumGate].v[i] = fma2(t.v[i], fma2(b.v[i], post_weight.v[i], post_bias.v[i]), sum[kSumGate].v[i]);
                }
                if (g.gate.p && in && !one_gate) gate = sum_param<F16, LIE>({g.gate.row((int)row / g.gate_every), 0, g.gate_vec}, c, n);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    t.v[i] = t.v[i] * gate.v[i];
                    sum[kSumPostW].v[i] = fma2(t.v[i], b.v[i], sum[kSumPostW].v[i]);
                    sum[kSumPostB].v[i] = sum[kSumPostB].v[i] + t.v[i];
                }
            }
        }
        if (BLOCK && a.gate_out) flush_sum(sum[BLOCK ? kSumGate : 0], shared, a.gate_out + group * a.gate_ld, c0, kColumns, shift, n);
        begin = end;
    }
#pragma unroll
    for (int i = 0; i < (BLOCK ? kSums : 2); ++i)
        if (a.partial[i]) flush_sum(sum[i], shared, a.partial[i] + ((int64_t)slice * gridDim.z + blockIdx.z) * n, c0, kColumns, shift, n);
}

// Adds slices' sums: a block takes 32 columns of one result, each of its warps every
// 32nd slice, and the warps' sums are added in order.
struct JoinArgs {
    const float *from[kSums];  // of each result but the gate's: [slices][n]
    float *to[kSums];
    int results;      // those; then one for each gate row
    const float *gate_from;  // [gate rows][parts][n]
    float *gate_to;
    int64_t gate_ld;
    int slices, parts, n;
};
__global__ void __launch_bounds__(32 * kMaxWarps) residual_norm_join_kernel(const __grid_constant__ JoinArgs a) {
    __shared__ float part[kMaxWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    const int which = blockIdx.y, group = which - a.results;
    const float *from = group >= 0 ? a.gate_from + (int64_t)group * a.parts * a.n : a.from[which];
    float *const to = group >= 0 ? a.gate_to + group * a.gate_ld : a.to[which];
    const int count = group >= 0 ? a.parts : a.slices;
    pdl_trigger();
    pdl_wait();
    float sum = 0.f;
    if (c < a.n) {
#pragma unroll 8
        for (int s = warp; s < count; s += kMaxWarps) sum += from[(int64_t)s * a.n + c];
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || c >= a.n) return;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kMaxWarps; ++w) sum += part[w][lane];
    to[c] = sum;
}

// ---------------------------------------------------------------- host
// How rows are had, threads of a row, rows of a block.
// Up to 128 pieces several rows go to a block (and to a warp: 200000 x 128 forward 96 us a row to a
// warp, 79 two to one), a piece to a thread; longer ones take two.  The gradients' kernel has four
// matrices to hold and gets them by bulk copies ahead, without registers (8192 x 5461 backward 711 us by
// plain loads, 494 so, packed arithmetic included).  The forward pass has two and is faster with plain
// loads (8192 x 5461: 165 us by bulk copies, 110 without).
struct Shape {
    Kind kind;
    int threads, groups;
};
Shape shape_of(int n, bool on_grid, bool bulk) {
    const int all = (n + kPiece - 1) / kPiece;
    const bool whole = on_grid && n % kPiece == 0;
    if (all <= kGroupThreads) {
        int threads = (all + 31) / 32 * 32;
        while (threads <= 32 && threads > 4 && threads / 2 >= all) threads /= 2;
        return {whole ? kSmall : kSmallAny, threads, threads < 32 ? 128 / threads : std::min(kMostGroups, 256 / threads)};
    }
    return {bulk ? (whole ? kBulk : kBulkAny) : whole ? kDirect : kDirectAny, ((all + 1) / 2 + 31) / 32 * 32, 1};
}

// The gradients' blocks of an SM at once, as far as registers and shared memory go.
int blocks_of(const Shape &h, size_t shared, int registers) {
    return (int)std::max<size_t>(1, std::min<size_t>((size_t)65536 / (registers * h.threads), (size_t)222 * 1024 / (shared + 2560)));
}

// The forward pass: a group of threads for each row.
cudaError_t run_rows(void (*kernel)(const SeamArgs), const Shape &h, const SeamArgs &a, cudaStream_t s) {
    const int64_t blocks = ((int64_t)a.in.m + h.groups - 1) / h.groups;
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3((unsigned)h.threads, (unsigned)h.groups), 0, s, a);
}
// The gradients.
cudaError_t run_rows(void (*kernel)(const SeamGradArgs, const Waits), const Shape &h, int registers, SeamGradArgs &a, const emtk_nn *nn, cudaStream_t s) {
    int64_t blocks = ((int64_t)a.in.m + h.groups - 1) / h.groups;
    size_t shared = 0;
    if (is_bulk(h.kind)) {
        const size_t row = (size_t)4 * a.in.row_bytes;
        a.in.stages = 2 * row <= 222 * 1024 ? 2 : 1;
        shared = a.in.stages * row;
        blocks = std::min<int64_t>(blocks, (int64_t)nn->sm_count * blocks_of(h, shared, registers));
    }
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3((unsigned)h.threads, (unsigned)h.groups), shared, s, a, Waits{nn->status, nn->timeout_ns});
}

template <bool F16>
cudaError_t run(SeamArgs &a, const Shape &h, const emtk_nn *, cudaStream_t s) {
    switch (h.kind) {
        case kSmall: return run_rows(residual_norm_kernel<F16, kSmall, 256>, h, a, s);
        case kSmallAny: return run_rows(residual_norm_kernel<F16, kSmallAny, 256>, h, a, s);
        case kDirect:
            return run_rows(h.threads <= 256   ? residual_norm_kernel<F16, kDirect, 256>
                            : h.threads <= 512 ? residual_norm_kernel<F16, kDirect, 512>
                                               : residual_norm_kernel<F16, kDirect, 1024>, h, a, s);
        default:
            return run_rows(h.threads <= 256   ? residual_norm_kernel<F16, kDirectAny, 256>
                            : h.threads <= 512 ? residual_norm_kernel<F16, kDirectAny, 512>
                                               : residual_norm_kernel<F16, kDirectAny, 1024>, h, a, s);
    }
}
template <bool F16, Kind KIND>
cudaError_t run_bulk(SeamGradArgs &a, const Shape &h, const emtk_nn *nn, cudaStream_t s) {
    if (h.threads <= 256) return run_rows(residual_norm_grad_kernel<F16, KIND, 256, 3>, h, 80, a, nn, s);
    if (h.threads <= 384) return run_rows(residual_norm_grad_kernel<F16, KIND, 384, 2>, h, 80, a, nn, s);
    if (h.threads <= 512) return run_rows(residual_norm_grad_kernel<F16, KIND, 512, 1>, h, 128, a, nn, s);
    return run_rows(residual_norm_grad_kernel<F16, KIND, 1024, 1>, h, 64, a, nn, s);
}
template <bool F16>
cudaError_t run(SeamGradArgs &a, const Shape &h, const emtk_nn *nn, cudaStream_t s) {
    switch (h.kind) {
        case kSmall: return run_rows(residual_norm_grad_kernel<F16, kSmall, 256, 3>, h, 80, a, nn, s);
        case kSmallAny: return run_rows(residual_norm_grad_kernel<F16, kSmallAny, 256, 3>, h, 80, a, nn, s);
        case kBulk: return run_bulk<F16, kBulk>(a, h, nn, s);
        default: return run_bulk<F16, kBulkAny>(a, h, nn, s);
    }
}
template <typename Args>
cudaError_t run(Args &a, int type, const Shape &h, const emtk_nn *nn, cudaStream_t s) {
    return type == EMTK_TYPE_F16 ? run<true>(a, h, nn, s) : run<false>(a, h, nn, s);
}

// Blocks across.
int64_t sum_columns(int n, Lie lie) {
    const int64_t each = lie == kAlike ? kAlikeColumns : 32 * kPiece;
    return (n + each - 1) / each;
}
// How the columns' kernel cuts the rows: as many blocks as run at once (a second round of
// few blocks costs as much as the first), of 16 rows at least.
Slices slices_of(int m, int n, int gate_every, bool block, Lie lie, int sms) {
    const int64_t columns = sum_columns(n, lie) * (lie == kAlike ? 2 : 1);
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>((block ? kSumBlocks : kSumBlocksPre) * (int64_t)sms / columns, ((int64_t)m + 15) / 16));
    const int64_t groups = std::max<int64_t>(1, ((int64_t)m + gate_every - 1) / gate_every);
    Slices l;
    if (groups < want) {
        const int64_t parts = want / groups, rows = std::min<int64_t>(gate_every, std::max(1, m));
        l.rows = (int)((rows + parts - 1) / parts);
        l.parts = (int)((rows + l.rows - 1) / l.rows);
        l.groups_each = 1;
        l.count = (int)(groups * l.parts);
    } else {
        l.parts = 1;
        l.groups_each = (int)((groups + want - 1) / want);
        l.rows = 0;
        l.count = (int)((groups + l.groups_each - 1) / l.groups_each);
    }
    return l;
}

}  // namespace

template <bool F16, Kind KIND>
static cudaError_t init_kernels() {
    cudaError_t e = cudaSuccess;
    for (void (*kernel)(const SeamGradArgs, const Waits) :
         {residual_norm_grad_kernel<F16, KIND, 256, 3>, residual_norm_grad_kernel<F16, KIND, 384, 2>,
          residual_norm_grad_kernel<F16, KIND, 512, 1>, residual_norm_grad_kernel<F16, KIND, 1024, 1>})
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 222 * 1024);
    return e;
}
cudaError_t init_norm_kernels() {
    for (const cudaError_t e : {init_kernels<false, kBulk>(), init_kernels<true, kBulk>(), init_kernels<false, kBulkAny>(), init_kernels<true, kBulkAny>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

cudaError_t launch_residual_norm(const emtk_residual_norm_args &p, const emtk_nn *nn, cudaStream_t s) {
    SeamArgs a{};
    a.in = {{rows16_of(p.residual), rows16_of(p.block)}, p.m, p.n, 0, 0};
    a.gate = rows16_of(p.gate);
    a.gate_vec = on_grid(p.gate, 2);
    a.y = rows16_of(p.y);
    a.h = rows16_of(p.h);
    a.post = norm_args(p.post);
    a.pre = norm_args(p.pre);
    if (p.block.d) a.drop = drop_of(p.drop);
    a.scale = p.scale;
    a.inverse_n = 1.f / (float)p.n;
    a.gate_every = p.gate_every;
    const bool whole = on_grid(p.residual, p.m) && on_grid(p.block, p.m) && on_grid(p.y, p.m) && on_grid(p.h, p.m);
    return run(a, p.type, shape_of(p.n, whole, false), nn, s);
}

// The sums that a call wants, and the workspace that they take.
static int norm_sums(const emtk_residual_norm_grad_args &p) {
    return (p.dw_pre ? 1 : 0) + (p.db_pre ? 1 : 0) + (p.dw_post ? 1 : 0) + (p.db_post ? 1 : 0) + (p.d_gate.d ? 1 : 0);
}
static bool block_sums(const emtk_residual_norm_grad_args &p) { return p.dw_post || p.db_post || p.d_gate.d; }
template <bool F16, bool BLOCK>
static void (*sum_kernel(Lie lie))(const SumArgs) {
    return lie == kGrid    ? residual_norm_sum_kernel<F16, kGrid, BLOCK>
           : lie == kAlike ? residual_norm_sum_kernel<F16, kAlike, BLOCK>
                           : residual_norm_sum_kernel<F16, kAny, BLOCK>;
}
// The columns' kernel of a call and its slices.
struct SumPlan {
    Lie lie;
    Slices slices;
    int64_t partials;  // of each slice's sums
};
static SumPlan sum_plan(const emtk_residual_norm_grad_args &p, int sms) {
    const emtk_matrix *const in[] = {&p.y, &p.dh, &p.dy, &p.block};
    bool grid = true, alike = true;
    const emtk_matrix *one = nullptr;
    for (int i = 0; i < (block_sums(p) ? 4 : 2); ++i) {
        if (!in[i]->d) continue;
        grid = grid && on_grid(*in[i], p.m);
        if (one) alike = alike && (reinterpret_cast<uintptr_t>(one->d) - reinterpret_cast<uintptr_t>(in[i]->d)) % 16 == 0 && (one->ld - in[i]->ld) % 8 == 0;
        one = in[i];
    }
    SumPlan plan;
    plan.lie = grid ? kGrid : alike ? kAlike : kAny;
    plan.slices = slices_of(p.m, p.n, p.gate_every, block_sums(p), plan.lie, sms);
    if (plan.lie == kAlike && p.d_gate.d && plan.slices.parts == 1) {  // a gate row's sum is one block's
        plan.lie = kAny;
        plan.slices = slices_of(p.m, p.n, p.gate_every, block_sums(p), plan.lie, sms);
    }
    plan.partials = plan.lie == kAlike ? 2 : 1;
    return plan;
}
size_t residual_norm_workspace(const emtk_residual_norm_grad_args &p, int sms) {
    const int sums = norm_sums(p);
    if (!sums) return 0;
    const SumPlan plan = sum_plan(p, sms);
    return (size_t)p.m * sizeof(RowStats) + (size_t)sums * plan.slices.count * plan.partials * p.n * sizeof(float);
}

cudaError_t launch_residual_norm_grad(const emtk_residual_norm_grad_args &p, void *workspace, const emtk_nn *nn, cudaStream_t s) {
    SeamGradArgs a{};
    a.in = {{rows16_of(p.y), rows16_of(p.dh), rows16_of(p.block), rows16_of(p.dy)}, p.m, p.n, bulk_row_bytes(p.n), 1};
    a.gate = rows16_of(p.gate);
    a.gate_vec = on_grid(p.gate, 2);
    a.d_residual = rows16_of(p.d_residual);
    a.d_block = rows16_of(p.d_block);
    a.post = norm_args(p.post);
    a.pre = norm_args(p.pre);
    if (p.block.d) a.drop = drop_of(p.drop);
    a.scale = p.scale;
    a.inverse_n = 1.f / (float)p.n;
    a.gate_every = p.gate_every;
    const int sums = norm_sums(p);
    if (sums) a.stats = static_cast<RowStats *>(workspace);
    const bool whole = on_grid(p.dy, p.m) && on_grid(p.dh, p.m) && on_grid(p.y, p.m) && on_grid(p.block, p.m) && on_grid(p.d_residual, p.m) && on_grid(p.d_block, p.m);
    cudaError_t e = p.m > 0 ? run(a, p.type, shape_of(p.n, whole, true), nn, s) : cudaSuccess;
    if (e != cudaSuccess || !sums) return e;

    const SumPlan plan = sum_plan(p, nn->sm_count);
    const Slices &slices = plan.slices;
    SumArgs t{};
    t.g = a;
    t.slices = slices;
    float *at = reinterpret_cast<float *>(a.stats + p.m);
    float *const out[kSums] = {p.dw_pre, p.db_pre, p.dw_post, p.db_post, static_cast<float *>(p.d_gate.d)};
    JoinArgs j{};
    for (int i = 0; i < kSums; ++i) {
        if (!out[i]) continue;
        if (i == kSumGate && slices.parts == 1 && p.m > 0) {
            t.gate_out = out[i];
            t.gate_ld = p.d_gate.ld;
            continue;
        }
        t.partial[i] = at;
        at += (size_t)slices.count * plan.partials * p.n;
        if (i == kSumGate) {
            j.gate_from = t.partial[i];
            j.gate_to = out[i];
            j.gate_ld = p.d_gate.ld;
        } else {
            j.from[j.results] = t.partial[i];
            j.to[j.results++] = out[i];
        }
    }
    j.slices = (int)(slices.count * plan.partials);
    j.parts = (int)(slices.parts * plan.partials);
    j.n = p.n;
    const bool f16 = p.type == EMTK_TYPE_F16;
    void (*const kernel)(const SumArgs) = block_sums(p) ? (f16 ? sum_kernel<true, true>(plan.lie) : sum_kernel<false, true>(plan.lie))
                                                        : (f16 ? sum_kernel<true, false>(plan.lie) : sum_kernel<false, false>(plan.lie));
    e = launch_pdl(kernel, dim3((unsigned)sum_columns(p.n, plan.lie), (unsigned)slices.count, (unsigned)plan.partials), dim3(kSumThreads), 0, s, t);
    const int gates = j.gate_to ? std::max(1, slices.count / slices.parts) : 0;
    if (e == cudaSuccess && j.results + gates > 0)
        e = launch_pdl(residual_norm_join_kernel, dim3((unsigned)((p.n + 31) / 32), (unsigned)(j.results + gates)),
                       dim3(32 * kMaxWarps), 0, s, j);
    return e;
}

}  // namespace emtk
