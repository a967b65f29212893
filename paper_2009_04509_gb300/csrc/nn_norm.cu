// Residual norms: the seam between two blocks, and its gradients.
//
//   v = D post(b);  y = s r + g v;  h = pre(y)
//   post(b) = (b - mean) / sqrt(mean((b - mean)^2) + eps) w + c   (mean 0 for RMS)
//
// A row is held in the registers of one block of threads, eight neighbouring columns to a
// piece, so each matrix is read once and every output written once; variances are of the
// centred values.  HBM bounds the forward pass (8 bytes a value in 16 bits) and the
// backward pass (12), the call a single row.
//
// Gradients.  With x^ = (x - mean) / std and q = w d of an output's gradient d, a norm's
// input has the gradient (q - mean(q) - x^ mean(q x^)) / std (mean(q) not for RMS).  A block
// of threads takes a slice of the rows, one after another, which bulk copies bring to shared
// memory ahead, and adds the columns' sums (the parameters' and the gate's gradients) in shared
// memory too, where each column is one thread's; a second kernel adds the slices in order, so results do not depend on timing.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_pieces.cuh"
#include "nn_ptx.cuh"

namespace emtk {
namespace {

constexpr int kMaxWarps = 32;

struct NormArgs {
    int kind;
    float eps;
    Param weight, bias;
};
NormArgs norm_args(const emtk_norm &n) {
    const int f32 = n.param_type == EMTK_TYPE_F32;
    return {n.kind, n.eps, {n.weight, f32}, {n.bias, f32}};
}

struct SeamArgs {
    Rows16 residual, block, gate, y, h;
    NormArgs post, pre;
    Drop drop;
    float scale, inverse_n;
    int m, n, gate_every;
};

// The sums of K (1, 2 or 4) values over the block's threads, in every thread.  In a warp
// each exchange halves the values that a lane still holds, and then the lanes; the warps'
// sums are read back with one value to a lane and added the same way: a sum costs a third
// of the shuffles that one tree for each value would.  `turn` alternates between two
// buffers, so that one barrier a call is enough.
struct Reduction {
    float (*buffer)[4 * kMaxWarps];  // [2]
    int warps, turn;
};
template <int K>
__device__ __forceinline__ void block_sum(float (&v)[K], Reduction &b) {
    const int lane = threadIdx.x & 31;
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
    for (int d = K; d < 32; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
    if (b.warps > 1) {
        float *const buffer = b.buffer[b.turn];
        if (lane < K) buffer[threadIdx.x / 32 * K + lane] = x;
        __syncthreads();
        x = 0.f;
        for (int i = lane; i < b.warps * K; i += 32) x += buffer[i];
#pragma unroll
        for (int d = K; d < 32; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
        b.turn ^= 1;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = K == 1 ? x : __shfl_sync(0xffffffffu, x, k);
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

// x becomes norm(x) weight + bias.
template <bool F16, int C>
__device__ __forceinline__ void normalise(const NormArgs &a, Eight (&x)[C], int n, float inverse_n, Reduction &b) {
    if (a.kind == EMTK_NORM_LAYER) {
        float sum[1] = {0.f};
#pragma unroll
        for (int k = 0; k < C; ++k) sum[0] += sum_of(x[k]);
        block_sum(sum, b);
#pragma unroll
        for (int k = 0; k < C; ++k) centre(x[k], sum[0] * inverse_n, (k * blockDim.x + threadIdx.x) * kPiece, n);
    }
    float square[1] = {0.f};
#pragma unroll
    for (int k = 0; k < C; ++k) square[0] += dot(x[k], x[k]);
    block_sum(square, b);
    const float r = rsqrtf(fmaf(square[0], inverse_n, a.eps));
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const int c = (k * blockDim.x + threadIdx.x) * kPiece;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[k].v[i] = x[k].v[i] * both(r);
        if (a.weight.p && c < n) {
            const Eight w = param8<F16>(a.weight, c, n);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[k].v[i] = x[k].v[i] * w.v[i];
        }
        if (a.bias.p && c < n) {
            const Eight w = param8<F16>(a.bias, c, n);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[k].v[i] = x[k].v[i] + w.v[i];
        }
    }
}

// The run of a row that a warp stores together: from column `run` on.
template <bool F16, bool ANY>
__device__ __forceinline__ void store_piece(const Rows16 &to, int64_t row, int n, const Eight &e, int k) {
    uint32_t w[4];
    words8<F16>(e, w);
    const int run = (k * blockDim.x + (threadIdx.x & ~31)) * kPiece;
    store_run<ANY>(to.row(row) + run, max(0, min(n - run, 32 * kPiece)), w, 32, threadIdx.x & 31);
}

// A row to a block of threads, C pieces to a thread.
template <bool F16, bool ANY, int C, int THREADS>
__global__ void __launch_bounds__(THREADS) residual_norm_kernel(const __grid_constant__ SeamArgs a) {
    __shared__ float buffer[2][4 * kMaxWarps];
    Reduction reduction{buffer, (int)blockDim.x / 32, 0};
    const int64_t row = blockIdx.x;
    Piece16<ANY> residual[C], block[C];
    pdl_trigger();
    pdl_wait();
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const int c = (k * blockDim.x + threadIdx.x) * kPiece;
        residual[k].clear();
        block[k].clear();
        if (a.block.p && c < a.n) block[k].load(a.block, row, c, a.m, a.n);
        if (a.residual.p && c < a.n) residual[k].load(a.residual, row, c, a.m, a.n);
    }
    Eight v[C];
#pragma unroll
    for (int k = 0; k < C; ++k) v[k] = block[k].template values<F16>();
    if (a.post.kind != EMTK_NORM_NONE) normalise<F16>(a.post, v, a.n, a.inverse_n, reduction);
    const uint64_t offset = a.drop.below ? drop_offset(a.drop) : 0u;
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const int first = k * blockDim.x + threadIdx.x, c = first * kPiece;
        if (a.drop.below) dropped(a.drop, offset, (uint32_t)row, (uint32_t)first, v[k]);
        if (a.gate.p && c < a.n) {
            const Eight g = param8<F16>({a.gate.row(row / a.gate_every), 0}, c, a.n);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k].v[i] = v[k].v[i] * g.v[i];
        }
        const Eight r = residual[k].template values<F16>();
#pragma unroll
        for (int i = 0; i < 4; ++i) v[k].v[i] = fma2(r.v[i], both(a.scale), v[k].v[i]);
        if (a.y.p) store_piece<F16, ANY>(a.y, row, a.n, v[k], k);
    }
    if (a.pre.kind == EMTK_NORM_NONE) return;
    normalise<F16>(a.pre, v, a.n, a.inverse_n, reduction);
#pragma unroll
    for (int k = 0; k < C; ++k) store_piece<F16, ANY>(a.h, row, a.n, v[k], k);
}

// ---------------------------------------------------------------- gradients
// Column sums of a slice: dw_pre, db_pre, dw_post, db_post, d_gate.
enum Sum : int { kSumPreW, kSumPreB, kSumPostW, kSumPostB, kSumGate, kSums };

// Slices of rows: `parts` of a gate row's rows each, or, with parts = 1, `groups_each`
// whole gate rows.
struct Slices {
    int count, parts, groups_each;
    int rows;  // of a part
};

enum Input : int { kInY, kInDh, kInBlock, kInDy, kInputs };

struct SeamGradArgs {
    Rows16 in[kInputs];  // y, dh, block, dy
    Rows16 gate, d_residual, d_block;
    NormArgs post, pre;
    Drop drop;
    float scale, inverse_n;
    int m, n, gate_every;
    Slices slices;
    float *partial[kSums];  // [slices][n] sums, or the result itself; null: not wanted
    float *gate_out;        // of whole gate rows: d_gate
    int64_t gate_ld;
    float *spill;           // not null: the running sums, in place of shared memory, [slices][sums][columns]
    int sums;               // wanted
    int at[kSums];          // place of each among them
    int stages, row_bytes;  // rows in shared memory, and the room for one of a matrix
};

template <int C>
struct Columns {  // a thread's running sums: [sum][piece][half][thread] of four
    float4 *base;
    __device__ __forceinline__ float4 *of(int sum, int k, int half) const {
        return base + ((sum * C + k) * 2 + half) * (int)blockDim.x + threadIdx.x;
    }
    __device__ __forceinline__ void add(int sum, int k, const Eight &e) const {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float4 *const p = of(sum, k, half);
            const float4 s = *p;
            const float2 a = make_float2(s.x, s.y) + e.v[2 * half], b = make_float2(s.z, s.w) + e.v[2 * half + 1];
            *p = make_float4(a.x, a.y, b.x, b.y);
        }
    }
    // Writes columns c .. of a sum to `to` and starts it again.
    __device__ __forceinline__ void flush(int sum, int k, float *to, int c, int n) const {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float4 *const p = of(sum, k, half);
            const float v[4] = {p->x, p->y, p->z, p->w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + 4 * half + i < n) to[c + 4 * half + i] = v[i];
            *p = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
};

// Rows on their way into shared memory: a stage has room for one row of each matrix, as it
// lies in its aligned 16-byte pieces, copied a row or two ahead by one thread.  Rows whose
// outer pieces would reach beyond the matrix are copied by elements when their turn comes.
struct RowPipe {
    uint8_t *stages;
    uint64_t *full;
    Guard guard;
    uint32_t phases = 0;  // of each stage
    bool ok = true;

    __device__ __forceinline__ uint8_t *place(const SeamGradArgs &a, int s, int input) const {
        return stages + (s * kInputs + input) * a.row_bytes;
    }
    static __device__ __forceinline__ int head_of(const Rows16 &x, int64_t row) {
        return (int)(reinterpret_cast<uintptr_t>(x.row(row)) % 16);
    }
    static __device__ __forceinline__ int bytes_of(const SeamGradArgs &a, int input, int64_t row) {  // of its aligned pieces
        return (head_of(a.in[input], row) + 2 * a.n + 15) / 16 * 16;
    }
    static __device__ __forceinline__ bool by_hand(const SeamGradArgs &a, int64_t row) {
        if (row >= kPiece && row < a.m - kPiece) return false;  // the 14 bytes around are of rows between
#pragma unroll
        for (int i = 0; i < kInputs; ++i) {
            if (!a.in[i].p) continue;
            const int64_t first = row * a.in[i].row_bytes - head_of(a.in[i], row), last = (a.m - 1) * a.in[i].row_bytes + 2 * a.n;
            if (first < 0 || first + bytes_of(a, i, row) > last) return true;
        }
        return false;
    }
    // One thread starts the copies of a row.
    __device__ __forceinline__ void fetch(const SeamGradArgs &a, int64_t row, int s) const {
        if (by_hand(a, row)) return;
        const uint32_t bar = smem_u32(full + s);
        int bytes[kInputs], all = 0;
#pragma unroll
        for (int i = 0; i < kInputs; ++i) {
            bytes[i] = a.in[i].p ? bytes_of(a, i, row) : 0;
            all += bytes[i];
        }
        mbar_expect_tx(bar, (uint32_t)all);
#pragma unroll
        for (int i = 0; i < kInputs; ++i)
            if (bytes[i])
                bulk_load(smem_u32(place(a, s, i)), reinterpret_cast<const uint8_t *>(a.in[i].row(row)) - head_of(a.in[i], row), bytes[i], bar);
    }
    // All threads: the row is in stage s.
    __device__ __forceinline__ void wait(const SeamGradArgs &a, int64_t row, int s) {
        if (by_hand(a, row)) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kInputs; ++i) {
                if (!a.in[i].p) continue;
                uint16_t *const to = reinterpret_cast<uint16_t *>(place(a, s, i) + head_of(a.in[i], row));
                for (int c = threadIdx.x; c < a.n; c += blockDim.x) to[c] = a.in[i].row(row)[c];
            }
            bulk_fence();
            __syncthreads();
            return;
        }
        if (ok) ok = wait_bounded(smem_u32(full + s), (phases >> s) & 1u, guard);
        phases ^= 1u << s;
    }
    // A piece of the row, columns from n on 0.
    __device__ __forceinline__ void piece(const SeamGradArgs &a, int64_t row, int s, int input, int c, uint32_t (&w)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = 0u;
        if (!a.in[input].p || c >= a.n) return;
        const uint4 *const p = reinterpret_cast<const uint4 *>(place(a, s, input)) + c / kPiece;
        const int halves = head_of(a.in[input], row) / 2;
        const uint4 lo = p[0];
        if (halves) {
            const uint4 hi = p[1];
            const uint32_t x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            shift_words(x, halves, w);
        } else {
            w[0] = lo.x, w[1] = lo.y, w[2] = lo.z, w[3] = lo.w;
        }
        if (c + kPiece > a.n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] &= (c + 2 * i < a.n ? 0xffffu : 0u) | (c + 2 * i + 1 < a.n ? 0xffff0000u : 0u);
        }
    }
};

template <bool F16, int C>
__global__ void __launch_bounds__(1024) residual_norm_grad_kernel(const __grid_constant__ SeamGradArgs a, int *status, int64_t timeout_ns) {
    extern __shared__ __align__(128) uint8_t shared[];
    __shared__ float buffer[2][4 * kMaxWarps];
    __shared__ uint64_t full[2];
    __shared__ uint32_t abort_flag;
    Reduction reduction{buffer, (int)blockDim.x / 32, 0};
    const int slice = blockIdx.x;
    RowPipe pipe{shared, full, {&abort_flag, status, timeout_ns}};
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(full), 1);
        mbar_init(smem_u32(full + 1), 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    Columns<C> sums{reinterpret_cast<float4 *>(shared + a.stages * kInputs * a.row_bytes)};
    pdl_trigger();
    pdl_wait();
    if (a.spill) sums.base = reinterpret_cast<float4 *>(a.spill) + (int64_t)slice * a.sums * C * 2 * blockDim.x;
    for (int i = 0; i < a.sums * C * 2; ++i) sums.base[i * blockDim.x + threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
    int64_t r0, r1;  // the slice's rows
    if (a.slices.parts > 1) {
        const int64_t begin = (int64_t)(slice / a.slices.parts) * a.gate_every, at = (int64_t)(slice % a.slices.parts) * a.slices.rows;
        const int64_t end = min(begin + a.gate_every, (int64_t)a.m);
        r0 = min(begin + at, end);
        r1 = min(begin + at + a.slices.rows, end);
    } else {
        r0 = min((int64_t)slice * a.slices.groups_each * a.gate_every, (int64_t)a.m);
        r1 = min(r0 + (int64_t)a.slices.groups_each * a.gate_every, (int64_t)a.m);
    }
    const bool pre = a.pre.kind != EMTK_NORM_NONE, post = a.post.kind != EMTK_NORM_NONE, has_block = a.in[kInBlock].p != nullptr;
    const bool pre_mean = a.pre.kind == EMTK_NORM_LAYER, post_mean = a.post.kind == EMTK_NORM_LAYER;
    const bool gate_sum = a.partial[kSumGate] || a.gate_out;
    const uint64_t offset = a.drop.below ? drop_offset(a.drop) : 0u;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 0; i < a.stages && r0 + i < r1; ++i) pipe.fetch(a, r0 + i, i);
    int s = 0;
    int64_t group = r0 / a.gate_every, group_end = (group + 1) * a.gate_every;
    for (int64_t row = r0; row < r1; ++row) {
        pipe.wait(a, row, s);
        Eight y[C], d[C], b[C], t[C];  // y, b: centred; d: dh, then q; t: of dy on
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int c = (k * blockDim.x + threadIdx.x) * kPiece;
            uint32_t w[4];
            pipe.piece(a, row, s, kInY, c, w);
            y[k] = values8<F16>(w);
            pipe.piece(a, row, s, kInDh, c, w);
            d[k] = values8<F16>(w);
            pipe.piece(a, row, s, kInBlock, c, w);
            b[k] = values8<F16>(w);
            pipe.piece(a, row, s, kInDy, c, w);
            t[k] = values8<F16>(w);
        }
        if (pre_mean || post_mean) {
            float v[2] = {};
#pragma unroll
            for (int k = 0; k < C; ++k) {
                v[0] += sum_of(y[k]);
                v[1] += sum_of(b[k]);
            }
            block_sum(v, reduction);
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int c = (k * blockDim.x + threadIdx.x) * kPiece;
                if (pre_mean) centre(y[k], v[0] * a.inverse_n, c, a.n);
                if (post_mean) centre(b[k], v[1] * a.inverse_n, c, a.n);
            }
        }
        if (a.partial[kSumPreB]) {
#pragma unroll
            for (int k = 0; k < C; ++k) sums.add(a.at[kSumPreB], k, d[k]);
        }
        float ry = 0.f, rb = 1.f;
        if (pre || post) {
            float v[4] = {};  // squares of y and b, q, q y
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int c = (k * blockDim.x + threadIdx.x) * kPiece;
                v[0] += dot(y[k], y[k]);
                v[1] += dot(b[k], b[k]);
                Eight q = d[k];
                if (a.pre.weight.p && c < a.n) {
                    const Eight w = param8<F16>(a.pre.weight, c, a.n);
#pragma unroll
                    for (int i = 0; i < 4; ++i) q.v[i] = q.v[i] * w.v[i];
                }
                v[2] += sum_of(q);
                v[3] += dot(q, y[k]);
            }
            block_sum(v, reduction);
            if (pre) ry = rsqrtf(fmaf(v[0], a.inverse_n, a.pre.eps));
            if (post) rb = rsqrtf(fmaf(v[1], a.inverse_n, a.post.eps));
            if (pre) {
                const float q_mean = pre_mean ? v[2] * a.inverse_n : 0.f, qy = v[3] * a.inverse_n * ry * ry;
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    const int c = (k * blockDim.x + threadIdx.x) * kPiece;
                    if (a.partial[kSumPreW]) {
                        Eight x;
#pragma unroll
                        for (int i = 0; i < 4; ++i) x.v[i] = d[k].v[i] * (y[k].v[i] * both(ry));
                        sums.add(a.at[kSumPreW], k, x);
                    }
                    if (a.pre.weight.p && c < a.n) {
                        const Eight w = param8<F16>(a.pre.weight, c, a.n);
#pragma unroll
                        for (int i = 0; i < 4; ++i) d[k].v[i] = d[k].v[i] * w.v[i];
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        t[k].v[i] = fma2(d[k].v[i] - fma2(y[k].v[i], both(qy), both(q_mean)), both(ry), t[k].v[i]);
                }
            }
        }
        // every thread has taken the row from its stage: the sums' barrier, or where there was none, one more
        if (!(reduction.warps > 1 && (pre || post))) __syncthreads();
        if (threadIdx.x == 0 && row + a.stages < r1) pipe.fetch(a, row + a.stages, s);
        if (++s == a.stages) s = 0;
        if (row >= group_end) {
            ++group;
            group_end += a.gate_every;
        }
        float u[2] = {};  // the sums for the block's norm
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int first = k * blockDim.x + threadIdx.x, c = first * kPiece;
            if (a.d_residual.p) {
                Eight x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[i] = t[k].v[i] * both(a.scale);
                store_piece<F16, true>(a.d_residual, row, a.n, x, k);
            }
            if (!has_block) continue;
            if (a.drop.below) dropped(a.drop, offset, (uint32_t)row, (uint32_t)first, t[k]);
            if (c + kPiece > a.n) centre(t[k], 0.f, c, a.n);
#pragma unroll
            for (int i = 0; i < 4; ++i) b[k].v[i] = b[k].v[i] * both(rb);  // now normalised
            Eight w;
            w.fill(1.f);
            if (a.post.weight.p && c < a.n) w = param8<F16>(a.post.weight, c, a.n);
            if (gate_sum) {
                Eight x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[i] = b[k].v[i] * w.v[i];
                if (a.post.bias.p && c < a.n) {
                    const Eight bias = param8<F16>(a.post.bias, c, a.n);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.v[i] = x.v[i] + bias.v[i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[i] = x.v[i] * t[k].v[i];
                sums.add(a.at[kSumGate], k, x);
            }
            if (a.gate.p && c < a.n) {
                const Eight g = param8<F16>({a.gate.row(group), 0}, c, a.n);
#pragma unroll
                for (int i = 0; i < 4; ++i) t[k].v[i] = t[k].v[i] * g.v[i];
            }
            if (a.partial[kSumPostW]) {
                Eight x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[i] = t[k].v[i] * b[k].v[i];
                sums.add(a.at[kSumPostW], k, x);
            }
            if (a.partial[kSumPostB]) sums.add(a.at[kSumPostB], k, t[k]);
#pragma unroll
            for (int i = 0; i < 4; ++i) t[k].v[i] = t[k].v[i] * w.v[i];
            u[0] += sum_of(t[k]);
            u[1] += dot(t[k], b[k]);
        }
        if (a.d_block.p) {
            float mean = 0.f, along = 0.f;
            if (post) {
                block_sum(u, reduction);
                mean = post_mean ? u[0] * a.inverse_n : 0.f;
                along = u[1] * a.inverse_n;
            }
#pragma unroll
            for (int k = 0; k < C; ++k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) t[k].v[i] = (t[k].v[i] - fma2(b[k].v[i], both(along), both(mean))) * both(rb);
                store_piece<F16, true>(a.d_block, row, a.n, t[k], k);
            }
        }
        if (a.gate_out && (row + 1 == group_end || row + 1 == r1)) {
#pragma unroll
            for (int k = 0; k < C; ++k)
                sums.flush(a.at[kSumGate], k, a.gate_out + group * a.gate_ld, (k * blockDim.x + threadIdx.x) * kPiece, a.n);
        }
    }
#pragma unroll
    for (int k = 0; k < C; ++k)
        for (int i = 0; i < kSums; ++i)
            if (a.partial[i])
                sums.flush(a.at[i], k, a.partial[i] + (int64_t)slice * a.n, (k * blockDim.x + threadIdx.x) * kPiece, a.n);
    if (!pipe.ok) {  // copies in flight land within microseconds: leave them a millisecond
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 1000000u) {
        }
    }
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
// Pieces of a thread and threads of a block.
struct Shape {
    int pieces, threads;
};
Shape shape_of(int n, int most_threads) {
    const int all = (n + kPiece - 1) / kPiece, c = all > most_threads ? 2 : 1;
    return {c, std::max(1, ((all + c - 1) / c + 31) / 32) * 32};
}

template <bool F16, bool ANY>
cudaError_t run(const SeamArgs &a, cudaStream_t s) {
    const Shape h = shape_of(a.n, 256);
    void (*kernel)(const SeamArgs) = h.pieces == 1      ? residual_norm_kernel<F16, ANY, 1, 256>
                                     : h.threads <= 256 ? residual_norm_kernel<F16, ANY, 2, 256>
                                                        : residual_norm_kernel<F16, ANY, 2, 1024>;
    return launch_pdl(kernel, dim3((unsigned)a.m), dim3((unsigned)h.threads), 0, s, a);
}

constexpr int kMostShared = 222 * 1024;  // of a block, beside what it has fixed

struct GradPlan {
    Shape shape;
    Slices slices;
    size_t columns;  // bytes of a slice's running sums
    size_t shared;   // of a block: rows, and the sums if there is room
    bool spilled;
    int sums, stages, row_bytes;
};
GradPlan grad_plan(int m, int n, int gate_every, int sums, int sms) {
    GradPlan p;
    p.shape = shape_of(n, 1024);
    p.sums = sums;
    p.columns = (size_t)sums * p.shape.pieces * p.shape.threads * kPiece * 4;
    // a row as it lies: up to 14 bytes before it, whole pieces, and the one after the last
    p.row_bytes = (2 * n + 14 + 15) / 16 * 16 + 16;
    const size_t stage = (size_t)kInputs * p.row_bytes;
    p.spilled = stage + p.columns > kMostShared;
    const size_t sums_bytes = p.spilled ? 0 : p.columns;
    p.stages = 2 * stage + sums_bytes <= kMostShared ? 2 : 1;
    p.shared = p.stages * stage + sums_bytes;
    const int warps = p.shape.threads / 32;
    const int each = std::max(1, std::min(32 / warps, (int)(kMostShared / (p.shared + 2048))));  // blocks of an SM
    // two rows at least to a slice, and no more slices than are resident at once
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>((int64_t)sms * each, ((int64_t)m + 1) / 2));
    const int64_t groups = std::max<int64_t>(1, ((int64_t)m + gate_every - 1) / gate_every);
    Slices &l = p.slices;
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
    return p;
}

template <bool F16>
cudaError_t run_grad(const SeamGradArgs &a, const GradPlan &p, const emtk_nn *nn, cudaStream_t s) {
    return launch_pdl(p.shape.pieces == 1 ? residual_norm_grad_kernel<F16, 1> : residual_norm_grad_kernel<F16, 2>,
                      dim3((unsigned)p.slices.count), dim3((unsigned)p.shape.threads), p.shared, s, a, nn->status, nn->timeout_ns);
}

}  // namespace

cudaError_t init_norm_kernels() {
    cudaError_t e = cudaSuccess;
    for (void (*kernel)(const SeamGradArgs, int *, int64_t) : {residual_norm_grad_kernel<false, 1>, residual_norm_grad_kernel<false, 2>,
                                                               residual_norm_grad_kernel<true, 1>, residual_norm_grad_kernel<true, 2>})
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    return e;
}

cudaError_t launch_residual_norm(const emtk_residual_norm_args &p, cudaStream_t s) {
    SeamArgs a{};
    a.residual = rows16_of(p.residual);
    a.block = rows16_of(p.block);
    a.gate = rows16_of(p.gate);
    a.y = rows16_of(p.y);
    a.h = rows16_of(p.h);
    a.post = norm_args(p.post);
    a.pre = norm_args(p.pre);
    if (p.block.d) a.drop = drop_of(p.drop);
    a.scale = p.scale;
    a.inverse_n = 1.f / (float)p.n;
    a.m = p.m;
    a.n = p.n;
    a.gate_every = p.gate_every;
    const bool any = !(on_grid(p.residual, p.m) && on_grid(p.block, p.m) && on_grid(p.y, p.m) && on_grid(p.h, p.m));
    if (p.type == EMTK_TYPE_F16) return any ? run<true, true>(a, s) : run<true, false>(a, s);
    return any ? run<false, true>(a, s) : run<false, false>(a, s);
}

// The sums that a call wants, and the workspace that they take.
static int norm_sums(const emtk_residual_norm_grad_args &p) {
    return (p.dw_pre ? 1 : 0) + (p.db_pre ? 1 : 0) + (p.dw_post ? 1 : 0) + (p.db_post ? 1 : 0) + (p.d_gate.d ? 1 : 0);
}
size_t residual_norm_workspace(const emtk_residual_norm_grad_args &p, int sms) {
    const GradPlan g = grad_plan(p.m, p.n, p.gate_every, norm_sums(p), sms);
    return (g.spilled ? g.columns * g.slices.count : 0) + (size_t)g.sums * g.slices.count * p.n * 4;
}

cudaError_t launch_residual_norm_grad(const emtk_residual_norm_grad_args &p, void *workspace, const emtk_nn *nn, cudaStream_t s) {
    const GradPlan g = grad_plan(p.m, p.n, p.gate_every, norm_sums(p), nn->sm_count);
    SeamGradArgs a{};
    a.in[kInY] = rows16_of(p.y);
    a.in[kInDh] = rows16_of(p.dh);
    a.in[kInBlock] = rows16_of(p.block);
    a.in[kInDy] = rows16_of(p.dy);
    a.gate = rows16_of(p.gate);
    a.d_residual = rows16_of(p.d_residual);
    a.d_block = rows16_of(p.d_block);
    a.post = norm_args(p.post);
    a.pre = norm_args(p.pre);
    if (p.block.d) a.drop = drop_of(p.drop);
    a.scale = p.scale;
    a.inverse_n = 1.f / (float)p.n;
    a.m = p.m;
    a.n = p.n;
    a.gate_every = p.gate_every;
    a.slices = g.slices;
    a.sums = g.sums;
    float *at = static_cast<float *>(workspace);
    a.stages = g.stages;
    a.row_bytes = g.row_bytes;
    if (g.spilled) {
        a.spill = at;
        at += g.columns / 4 * g.slices.count;
    }
    float *const out[kSums] = {p.dw_pre, p.db_pre, p.dw_post, p.db_post, static_cast<float *>(p.d_gate.d)};
    JoinArgs j{};
    int place = 0;
    for (int i = 0; i < kSums; ++i) {
        if (!out[i]) continue;
        a.at[i] = place++;
        if (i == kSumGate && g.slices.parts == 1 && p.m > 0) {
            a.gate_out = out[i];
            a.gate_ld = p.d_gate.ld;
            continue;
        }
        a.partial[i] = at;
        at += (size_t)g.slices.count * p.n;
        if (i == kSumGate) {
            j.gate_from = a.partial[i];
            j.gate_to = out[i];
            j.gate_ld = p.d_gate.ld;
        } else {
            j.from[j.results] = a.partial[i];
            j.to[j.results++] = out[i];
        }
    }
    j.slices = g.slices.count;
    j.parts = g.slices.parts;
    j.n = p.n;
    cudaError_t e = p.type == EMTK_TYPE_F16 ? run_grad<true>(a, g, nn, s) : run_grad<false>(a, g, nn, s);
    const int gates = j.gate_to ? std::max(1, g.slices.count / g.slices.parts) : 0;
    if (e == cudaSuccess && j.results + gates > 0)
        e = launch_pdl(residual_norm_join_kernel, dim3((unsigned)((p.n + 31) / 32), (unsigned)(j.results + gates)),
                       dim3(32 * kMaxWarps), 0, s, j);
    return e;
}

}  // namespace emtk
