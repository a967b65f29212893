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
// of threads takes a slice of the rows, one after another, and adds the columns' sums (the
// parameters' and the gate's gradients) in shared memory, where each column is one
// thread's; a second kernel adds the slices in order, so results do not depend on timing.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_pieces.cuh"

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

// The sums of K values over the block's threads, in every thread.  `turn` alternates
// between two buffers, so that one barrier a call is enough.
template <int K>
__device__ __forceinline__ void block_sum(float (&v)[K], float (*buffer)[4][kMaxWarps], int &turn, int warps) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], d);
    if (warps == 1) return;
    const int lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) buffer[turn][k][threadIdx.x / 32] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lane < warps ? buffer[turn][k][lane] : 0.f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], d);
    turn ^= 1;
}

// x becomes norm(x) w + c; columns from n on stay out of the sums.
template <bool F16, int C>
__device__ __forceinline__ void normalise(const NormArgs &a, float (&x)[C][kPiece], int n, float inverse_n,
                                          float (*buffer)[4][kMaxWarps], int &turn, int warps) {
    float mean = 0.f;
    if (a.kind == EMTK_NORM_LAYER) {
        float sum[1] = {0.f};
#pragma unroll
        for (int k = 0; k < C; ++k)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) sum[0] += x[k][i];
        block_sum(sum, buffer, turn, warps);
        mean = sum[0] * inverse_n;
    }
    float square[1] = {0.f};
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const int c = (k * blockDim.x + threadIdx.x) * kPiece;
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            x[k][i] = c + i < n ? x[k][i] - mean : 0.f;
            square[0] = fmaf(x[k][i], x[k][i], square[0]);
        }
    }
    block_sum(square, buffer, turn, warps);
    const float r = rsqrtf(fmaf(square[0], inverse_n, a.eps));
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const int c = (k * blockDim.x + threadIdx.x) * kPiece;
        if (c >= n) continue;
        float w[kPiece], b[kPiece];
        param8<F16>(a.weight, c, n, 1.f, w);
        param8<F16>(a.bias, c, n, 0.f, b);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) x[k][i] = fmaf(x[k][i] * r, w[i], b[i]);
    }
}

// A row to a block of threads, C pieces to a thread.
template <bool F16, bool ANY, int C, int THREADS>
__global__ void __launch_bounds__(THREADS) residual_norm_kernel(const __grid_constant__ SeamArgs a) {
    __shared__ float buffer[2][4][kMaxWarps];
    int turn = 0;
    const int64_t row = blockIdx.x;
    const int warps = blockDim.x / 32, lane = threadIdx.x & 31;
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
    float v[C][kPiece];
#pragma unroll
    for (int k = 0; k < C; ++k) block[k].template values<F16>(v[k]);
    if (a.post.kind != EMTK_NORM_NONE) normalise<F16>(a.post, v, a.n, a.inverse_n, buffer, turn, warps);
    const uint64_t offset = a.drop.below ? drop_offset(a.drop) : 0u;
    const Param gate{a.gate.p ? a.gate.row(row / a.gate_every) : nullptr, 0};
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const int first = k * blockDim.x + threadIdx.x, c = first * kPiece;
        if (a.drop.below) dropped(a.drop, offset, (uint32_t)row, (uint32_t)first, v[k]);
        float g[kPiece], r[kPiece];
        if (c < a.n) {
            param8<F16>(gate, c, a.n, 1.f, g);
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) g[i] = 0.f;
        }
        residual[k].template values<F16>(r);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[k][i] = fmaf(v[k][i], g[i], a.scale * r[i]);
        if (a.y.p) {
            uint32_t w[4];
            words8<F16>(v[k], w);
            const int run = c - kPiece * lane;
            store_run<ANY>(a.y.row(row) + run, max(0, min(a.n - run, 32 * kPiece)), w, 32, lane);
        }
    }
    if (a.pre.kind == EMTK_NORM_NONE) return;
    normalise<F16>(a.pre, v, a.n, a.inverse_n, buffer, turn, warps);
#pragma unroll
    for (int k = 0; k < C; ++k) {
        uint32_t w[4];
        words8<F16>(v[k], w);
        const int run = (k * blockDim.x + (threadIdx.x & ~31)) * kPiece;
        store_run<ANY>(a.h.row(row) + run, max(0, min(a.n - run, 32 * kPiece)), w, 32, lane);
    }
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

struct SeamGradArgs {
    Rows16 dy, dh, y, block, gate, d_residual, d_block;
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
};

template <int C>
struct Columns {  // a thread's running sums: [sum][piece][half][thread] of four
    float4 *base;
    __device__ __forceinline__ float4 *of(int sum, int k, int half) const {
        return base + ((sum * C + k) * 2 + half) * (int)blockDim.x + threadIdx.x;
    }
    __device__ __forceinline__ void add(int sum, int k, const float (&v)[kPiece]) const {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float4 *const p = of(sum, k, half);
            float4 s = *p;
            s.x += v[4 * half], s.y += v[4 * half + 1], s.z += v[4 * half + 2], s.w += v[4 * half + 3];
            *p = s;
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

template <bool F16, bool ANY, int C, int THREADS>
__global__ void __launch_bounds__(THREADS) residual_norm_grad_kernel(const __grid_constant__ SeamGradArgs a) {
    extern __shared__ float4 columns_smem[];
    __shared__ float buffer[2][4][kMaxWarps];
    int turn = 0;
    const int warps = blockDim.x / 32, lane = threadIdx.x & 31;
    const int slice = blockIdx.x;
    Columns<C> sums{columns_smem};
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
    const bool pre = a.pre.kind != EMTK_NORM_NONE, has_block = a.block.p != nullptr;
    const bool pre_mean = a.pre.kind == EMTK_NORM_LAYER, post_mean = a.post.kind == EMTK_NORM_LAYER;
    const uint64_t offset = a.drop.below ? drop_offset(a.drop) : 0u;
    Piece16<ANY> py[C], ph[C], pb[C], pd[C];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int c = (k * blockDim.x + threadIdx.x) * kPiece;
            py[k].clear();
            ph[k].clear();
            pb[k].clear();
            pd[k].clear();
            if (c >= a.n) continue;
            if (pre) py[k].load(a.y, row, c, a.m, a.n);
            if (pre) ph[k].load(a.dh, row, c, a.m, a.n);
            if (has_block) pb[k].load(a.block, row, c, a.m, a.n);
            if (a.dy.p) pd[k].load(a.dy, row, c, a.m, a.n);
        }
    };
    if (r0 < r1) fetch(r0);
    for (int64_t row = r0; row < r1; ++row) {
        float y[C][kPiece], d[C][kPiece], b[C][kPiece], t[C][kPiece];  // y, b: centred; d: dh
#pragma unroll
        for (int k = 0; k < C; ++k) {
            py[k].template values<F16>(y[k]);
            ph[k].template values<F16>(d[k]);
            pb[k].template values<F16>(b[k]);
            pd[k].template values<F16>(t[k]);
        }
        if (C == 1 && row + 1 < r1) fetch(row + 1);
        float mean_y = 0.f, mean_b = 0.f;
        if (pre_mean || post_mean) {
            float s[2] = {};
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int i = 0; i < kPiece; ++i) s[0] += y[k][i], s[1] += b[k][i];
            block_sum(s, buffer, turn, warps);
            if (pre_mean) mean_y = s[0] * a.inverse_n;
            if (post_mean) mean_b = s[1] * a.inverse_n;
        }
        float s[4] = {};  // squares of y and b, q, q y
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int c = (k * blockDim.x + threadIdx.x) * kPiece;
            float w[kPiece];
            if (c < a.n) {
                param8<F16>(a.pre.weight, c, a.n, 1.f, w);
            } else {
#pragma unroll
                for (int i = 0; i < kPiece; ++i) w[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                y[k][i] = c + i < a.n ? y[k][i] - mean_y : 0.f;
                b[k][i] = c + i < a.n ? b[k][i] - mean_b : 0.f;
                const float q = d[k][i] * w[i];
                s[0] = fmaf(y[k][i], y[k][i], s[0]);
                s[1] = fmaf(b[k][i], b[k][i], s[1]);
                s[2] += q;
                s[3] = fmaf(q, y[k][i], s[3]);
            }
        }
        block_sum(s, buffer, turn, warps);
        const float ry = pre ? rsqrtf(fmaf(s[0], a.inverse_n, a.pre.eps)) : 0.f;
        const float rb = a.post.kind != EMTK_NORM_NONE ? rsqrtf(fmaf(s[1], a.inverse_n, a.post.eps)) : 1.f;
        const float q_mean = pre_mean ? s[2] * a.inverse_n : 0.f, qy = s[3] * a.inverse_n * ry * ry;
        const Param gate{a.gate.p ? a.gate.row(row / a.gate_every) : nullptr, 0};
        float u[2] = {};  // the sums for the block's norm
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int first = k * blockDim.x + threadIdx.x, c = first * kPiece;
            const bool in = c < a.n;
            float w[kPiece], x[kPiece];
            if (pre && in) {
                param8<F16>(a.pre.weight, c, a.n, 1.f, w);
#pragma unroll
                for (int i = 0; i < kPiece; ++i) {
                    t[k][i] = fmaf(ry, d[k][i] * w[i] - q_mean - y[k][i] * qy, t[k][i]);
                    x[i] = d[k][i] * y[k][i] * ry;
                }
                if (a.partial[kSumPreW]) sums.add(a.at[kSumPreW], k, x);
                if (a.partial[kSumPreB]) sums.add(a.at[kSumPreB], k, d[k]);
            }
            if (a.d_residual.p) {
                uint32_t q[4];
#pragma unroll
                for (int i = 0; i < kPiece; ++i) x[i] = t[k][i] * a.scale;
                words8<F16>(x, q);
                const int run = c - kPiece * lane;
                store_run<ANY>(a.d_residual.row(row) + run, max(0, min(a.n - run, 32 * kPiece)), q, 32, lane);
            }
            if (!has_block || !in) continue;
            if (a.drop.below) dropped(a.drop, offset, (uint32_t)row, (uint32_t)first, t[k]);
            float g[kPiece];
            param8<F16>(a.post.weight, c, a.n, 1.f, w);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) b[k][i] *= rb;  // now normalised
            if (a.partial[kSumGate] || a.gate_out) {
                param8<F16>(a.post.bias, c, a.n, 0.f, g);
#pragma unroll
                for (int i = 0; i < kPiece; ++i) x[i] = t[k][i] * fmaf(b[k][i], w[i], g[i]);
                sums.add(a.at[kSumGate], k, x);
            }
            param8<F16>(gate, c, a.n, 1.f, g);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) t[k][i] *= g[i];
            if (a.partial[kSumPostW]) {
#pragma unroll
                for (int i = 0; i < kPiece; ++i) x[i] = t[k][i] * b[k][i];
                sums.add(a.at[kSumPostW], k, x);
            }
            if (a.partial[kSumPostB]) sums.add(a.at[kSumPostB], k, t[k]);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                t[k][i] *= w[i];
                u[0] += c + i < a.n ? t[k][i] : 0.f;
                u[1] = fmaf(c + i < a.n ? t[k][i] : 0.f, b[k][i], u[1]);
            }
        }
        if (a.d_block.p) {
            if (a.post.kind != EMTK_NORM_NONE) block_sum(u, buffer, turn, warps);
            const float t_mean = post_mean ? u[0] * a.inverse_n : 0.f;
            const float tb = a.post.kind != EMTK_NORM_NONE ? u[1] * a.inverse_n : 0.f;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                float x[kPiece];
                uint32_t q[4];
#pragma unroll
                for (int i = 0; i < kPiece; ++i) x[i] = rb * (t[k][i] - t_mean - b[k][i] * tb);
                words8<F16>(x, q);
                const int run = (k * blockDim.x + (threadIdx.x & ~31)) * kPiece;
                store_run<ANY>(a.d_block.row(row) + run, max(0, min(a.n - run, 32 * kPiece)), q, 32, lane);
            }
        }
        if (a.gate_out && ((row + 1) % a.gate_every == 0 || row + 1 == r1)) {
#pragma unroll
            for (int k = 0; k < C; ++k)
                sums.flush(a.at[kSumGate], k, a.gate_out + row / a.gate_every * a.gate_ld, (k * blockDim.x + threadIdx.x) * kPiece, a.n);
        }
        if (C > 1 && row + 1 < r1) fetch(row + 1);
    }
#pragma unroll
    for (int k = 0; k < C; ++k)
        for (int i = 0; i < kSums; ++i)
            if (a.partial[i])
                sums.flush(a.at[i], k, a.partial[i] + (int64_t)slice * a.n, (k * blockDim.x + threadIdx.x) * kPiece, a.n);
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

constexpr int kMostShared = 220 * 1024;  // of running sums in shared memory

struct GradPlan {
    Shape shape;
    Slices slices;
    size_t columns;   // bytes of a slice's running sums
    size_t shared;    // of them in shared memory, else 0
    int sums;
};
GradPlan grad_plan(int m, int n, int gate_every, int sums, int sms) {
    GradPlan p;
    p.shape = shape_of(n, 1024);
    p.sums = sums;
    p.columns = (size_t)sums * p.shape.pieces * p.shape.threads * kPiece * 4;
    p.shared = p.columns <= kMostShared ? p.columns : 0;
    const int warps = p.shape.threads / 32;
    int each = std::max(1, 32 / warps);  // blocks of an SM
    if (p.shared) each = std::max(1, std::min(each, (int)(kMostShared / p.shared)));
    // two rows at least to a slice, and no more slices than are resident at once
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>((int64_t)sms * each, ((int64_t)m + 1) / 2));
    const int64_t groups = std::max<int64_t>(1, ((int64_t)m + gate_every - 1) / gate_every);
    Slices &l = p.slices;
    if (groups < want) {
        const int64_t parts = want / groups;
        l.rows = (int)((std::min<int64_t>(gate_every, std::max(1, m)) + parts - 1) / parts);
        l.parts = (int)((std::min<int64_t>(gate_every, std::max(1, m)) + l.rows - 1) / l.rows);
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

template <bool F16, bool ANY, int C, int THREADS>
cudaError_t run_grad(const SeamGradArgs &a, const GradPlan &p, cudaStream_t s) {
    return launch_pdl(residual_norm_grad_kernel<F16, ANY, C, THREADS>, dim3((unsigned)p.slices.count),
                      dim3((unsigned)p.shape.threads), p.shared, s, a);
}
template <bool F16, bool ANY>
cudaError_t run_grad(const SeamGradArgs &a, const GradPlan &p, cudaStream_t s) {
    if (p.shape.pieces == 2) return run_grad<F16, ANY, 2, 1024>(a, p, s);
    return p.shape.threads <= 256   ? run_grad<F16, ANY, 1, 256>(a, p, s)
           : p.shape.threads <= 512 ? run_grad<F16, ANY, 1, 512>(a, p, s)
                                    : run_grad<F16, ANY, 1, 1024>(a, p, s);
}

}  // namespace

cudaError_t init_norm_kernels() {
    cudaError_t e = cudaSuccess;
#define EMTK_NORM_ATTR(F16, ANY, C, THREADS)                                             \
    if (e == cudaSuccess)                                                                \
        e = cudaFuncSetAttribute(residual_norm_grad_kernel<F16, ANY, C, THREADS>,        \
                                 cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
#define EMTK_NORM_ATTRS(F16, ANY)      \
    EMTK_NORM_ATTR(F16, ANY, 1, 256)   \
    EMTK_NORM_ATTR(F16, ANY, 1, 512)   \
    EMTK_NORM_ATTR(F16, ANY, 1, 1024)  \
    EMTK_NORM_ATTR(F16, ANY, 2, 1024)
    EMTK_NORM_ATTRS(false, false)
    EMTK_NORM_ATTRS(false, true)
    EMTK_NORM_ATTRS(true, false)
    EMTK_NORM_ATTRS(true, true)
#undef EMTK_NORM_ATTRS
#undef EMTK_NORM_ATTR
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
    const size_t spill = g.shared == g.columns ? 0 : g.columns * g.slices.count;
    return spill + (size_t)g.sums * g.slices.count * p.n * 4;
}

cudaError_t launch_residual_norm_grad(const emtk_residual_norm_grad_args &p, void *workspace, int sms, cudaStream_t s) {
    const GradPlan g = grad_plan(p.m, p.n, p.gate_every, norm_sums(p), sms);
    SeamGradArgs a{};
    a.dy = rows16_of(p.dy);
    a.dh = rows16_of(p.dh);
    a.y = rows16_of(p.y);
    a.block = rows16_of(p.block);
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
    if (g.shared != g.columns) {
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
    const bool any = !(on_grid(p.dy, p.m) && on_grid(p.dh, p.m) && on_grid(p.y, p.m) && on_grid(p.block, p.m) &&
                       on_grid(p.d_residual, p.m) && on_grid(p.d_block, p.m));
    cudaError_t e;
    if (p.type == EMTK_TYPE_F16)
        e = any ? run_grad<true, true>(a, g, s) : run_grad<true, false>(a, g, s);
    else
        e = any ? run_grad<false, true>(a, g, s) : run_grad<false, false>(a, g, s);
    const int gates = j.gate_to ? std::max(1, g.slices.count / g.slices.parts) : 0;
    if (e == cudaSuccess && j.results + gates > 0)
        e = launch_pdl(residual_norm_join_kernel, dim3((unsigned)((p.n + 31) / 32), (unsigned)(j.results + gates)),
                       dim3(32 * kMaxWarps), 0, s, j);
    return e;
}

}  // namespace emtk
