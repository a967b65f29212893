// Pointwise passes of the dense and gated layers' gradients, and the 8-bit
// checkpoints.  All of them stream: every element is read once with 16-byte
// loads (8 columns a thread) where address and row distance allow it, one
// element at a time where they do not, and what bounds them is HBM.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_math.cuh"

namespace emtk {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;  // columns of a thread

enum Access : int { kAbsent = 0, kWide16, kNarrow16, kWideQ8, kNarrowQ8 };

struct Source {
    const void *p;
    const uint8_t *scale;
    int64_t ld, ld_scale;
    int access;
};

bool aligned(const void *p, int64_t row_bytes, int bytes) {
    return (reinterpret_cast<uintptr_t>(p) % bytes) == 0 && row_bytes % bytes == 0;
}

Source source_of(const emtk_matrix &m) {
    Source s{m.d, m.d_scale, m.ld, m.ld_scale, kAbsent};
    if (m.d == nullptr) return s;
    if (m.d_scale)
        s.access = aligned(m.d, m.ld, kVec) ? kWideQ8 : kNarrowQ8;
    else
        s.access = aligned(m.d, 2 * m.ld, 16) ? kWide16 : kNarrow16;
    return s;
}

// Columns c .. c + 7 of row r as fp32; columns from n on read as 0.
template <bool F16>
__device__ __forceinline__ void load8(const Source &s, int64_t r, int c, int n, float (&v)[kVec]) {
    const bool full = c + kVec <= n;
    if (s.access == kWide16 && full) {
        const uint4 w = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(s.p) + r * s.ld + c));
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = from16<F16>(x[i] & 0xffffu);
            v[2 * i + 1] = from16<F16>(x[i] >> 16);
        }
    } else if (s.access == kWide16 || s.access == kNarrow16) {
        const uint16_t *p = static_cast<const uint16_t *>(s.p) + r * s.ld + c;
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = c + i < n ? from16<F16>(__ldg(p + i)) : 0.f;
    } else {
        const uint8_t *p = static_cast<const uint8_t *>(s.p) + r * s.ld + c;
        const float step = c < n ? q8_step(__ldg(s.scale + r * s.ld_scale + c / kQ8Block)) : 0.f;
        uint32_t w[2] = {0u, 0u};
        if (s.access == kWideQ8 && full) {
            const uint2 q = __ldg(reinterpret_cast<const uint2 *>(p));
            w[0] = q.x;
            w[1] = q.y;
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (c + i < n) w[i / 4] |= (uint32_t)__ldg(p + i) << (8 * (i % 4));
        }
        q8_values4(w[0], step, v);
        q8_values4(w[1], step, v + 4);
    }
}

template <bool F16>
__device__ __forceinline__ void store8(uint16_t *row, int c, int n, bool wide, const float (&v)[kVec]) {
    if (wide && c + kVec <= n) {
        *reinterpret_cast<uint4 *>(row + c) = make_uint4(pack16<F16>(v[0], v[1]), pack16<F16>(v[2], v[3]),
                                                         pack16<F16>(v[4], v[5]), pack16<F16>(v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (c + i < n) row[c + i] = (uint16_t)to16<F16>(v[i]);
    }
}

// ------------------------------------------------------------- slopes
// A block takes 8 * lanes columns (lanes = 32 .. 4, the fewest that cover
// narrow matrices) and one slice of the rows, kThreads / lanes rows at a time;
// a thread adds its rows in order, the block its threads' sums and the second
// kernel the slices' in fixed orders, so the column sums do not depend on
// timing.
struct SlopeShape {
    int lanes_log2;  // threads across
    int col_blocks, slices;
    int rows;  // of a slice
};

// Blocks for every SM: with sums few enough that the slices' partial sums stay
// small against the rows, without them enough to even out the end.
SlopeShape slope_shape(int m, int n, int sms, bool sums) {
    SlopeShape h;
    h.lanes_log2 = 5;
    while (h.lanes_log2 > 2 && (kVec << (h.lanes_log2 - 1)) >= n) --h.lanes_log2;
    const int cols = kVec << h.lanes_log2;
    const int at_once = kThreads >> h.lanes_log2;
    h.col_blocks = (int)(((int64_t)n + cols - 1) / cols);
    int64_t slices = std::max<int64_t>(1, (int64_t)(sums ? 8 : 24) * sms / std::max(1, h.col_blocks));
    slices = std::min<int64_t>(slices, std::max<int64_t>(1, ((int64_t)m + 2 * at_once - 1) / (2 * at_once)));
    slices = std::min<int64_t>(slices, 65535);
    int64_t rows = ((int64_t)m + slices - 1) / slices;
    rows = (rows + at_once - 1) / at_once * at_once;
    rows = std::max<int64_t>(rows, at_once);
    h.rows = (int)std::min<int64_t>(rows, INT32_MAX / 2);
    h.slices = (int)std::max<int64_t>(1, ((int64_t)m + h.rows - 1) / h.rows);
    return h;
}

struct SlopeArgs {
    Source dy, gate, up;  // gate: the activation's input (pre of a dense layer); up: gated only
    uint16_t *dg, *du;    // 16-byte aligned rows of d_ld elements; dg: dz of a dense layer
    int64_t d_ld;
    uint16_t *h;
    int64_t h_ld;
    int h_wide;
    float *partial;  // [slices][n], gated: [2][slices][n]; null: no sums
    int m, n, rows, lanes_log2;
};

template <bool F16, bool GATED, int ACT, bool SUMS>
__global__ void __launch_bounds__(kThreads) slope_kernel(const __grid_constant__ SlopeArgs a) {
    const int lanes = 1 << a.lanes_log2;
    const int at_once = kThreads >> a.lanes_log2;
    const int c = (int)blockIdx.x * (kVec << a.lanes_log2) + (threadIdx.x & (lanes - 1)) * kVec;
    const int sub = threadIdx.x >> a.lanes_log2;
    const int64_t r0 = (int64_t)blockIdx.y * a.rows;
    const int64_t r1 = min(r0 + a.rows, (int64_t)a.m);
    float sg[kVec] = {}, su[kVec] = {};
    pdl_trigger();
    pdl_wait();
    if (c < a.n) {
#pragma unroll 2
        for (int64_t r = r0 + sub; r < r1; r += at_once) {
            float d[kVec], g[kVec], dg[kVec];
            load8<F16>(a.dy, r, c, a.n, d);
            if (GATED || ACT != EMTK_ACT_NONE) load8<F16>(a.gate, r, c, a.n, g);
            if (GATED) {
                float u[kVec], du[kVec], h[kVec];
                load8<F16>(a.up, r, c, a.n, u);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    float f, s;
                    act_slope<ACT>(g[i], f, s);
                    dg[i] = d[i] * u[i] * s;
                    du[i] = d[i] * f;
                    h[i] = f * u[i];
                    if (SUMS) su[i] += du[i];
                }
                if (a.du) store8<F16>(a.du + r * a.d_ld, c, a.n, true, du);
                if (a.h) store8<F16>(a.h + r * a.h_ld, c, a.n, a.h_wide != 0, h);
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    float f, s = 1.f;
                    if (ACT != EMTK_ACT_NONE) act_slope<ACT>(g[i], f, s);
                    dg[i] = d[i] * s;
                }
            }
            if (SUMS) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) sg[i] += dg[i];
            }
            if (a.dg) store8<F16>(a.dg + r * a.d_ld, c, a.n, true, dg);
        }
    }
    if constexpr (SUMS) {
        __shared__ float part[kThreads * kVec];
        const int cols = kVec << a.lanes_log2;
        const int col = (int)blockIdx.x * cols + (int)threadIdx.x;
#pragma unroll
        for (int half = 0; half < (GATED ? 2 : 1); ++half) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kVec; ++i) part[threadIdx.x * kVec + i] = half ? su[i] : sg[i];
            __syncthreads();
            if ((int)threadIdx.x < cols && col < a.n) {
                float sum = 0.f;
                for (int g = 0; g < at_once; ++g) sum += part[g * cols + threadIdx.x];
                a.partial[((int64_t)half * gridDim.y + blockIdx.y) * a.n + col] = sum;
            }
        }
    }
}

// Column sums from the slices' partial sums: a block takes 32 columns, each of
// its 16 warps every 16th slice, and the warps' sums are added in order.
constexpr int kSumWarps = 16;
__global__ void __launch_bounds__(32 * kSumWarps) slice_sum_kernel(const float *partial, int slices, int n, float *db0,
                                                                   float *db1) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    __shared__ float part[kSumWarps][32];
    pdl_trigger();
    pdl_wait();
    float sum = 0.f;
    if (c < n) {
        const float *p = partial + (int64_t)blockIdx.y * slices * n + c;
#pragma unroll 8
        for (int s = warp; s < slices; s += kSumWarps) sum += p[(int64_t)s * n];
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || c >= n) return;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kSumWarps; ++w) sum += part[w][lane];
    (blockIdx.y ? db1 : db0)[c] = sum;
}

template <bool F16, bool GATED, bool SUMS>
cudaError_t start_slope(const SlopeArgs &a, int act, dim3 grid, cudaStream_t s) {
    auto kernel = slope_kernel<F16, GATED, EMTK_ACT_NONE, SUMS>;
    if (act == EMTK_ACT_RELU) kernel = slope_kernel<F16, GATED, EMTK_ACT_RELU, SUMS>;
    if (act == EMTK_ACT_GELU) kernel = slope_kernel<F16, GATED, EMTK_ACT_GELU, SUMS>;
    if (act == EMTK_ACT_SILU) kernel = slope_kernel<F16, GATED, EMTK_ACT_SILU, SUMS>;
    if (act == EMTK_ACT_SIGMOID) kernel = slope_kernel<F16, GATED, EMTK_ACT_SIGMOID, SUMS>;
    return launch_pdl(kernel, grid, dim3(kThreads), 0, s, a);
}

template <bool GATED>
cudaError_t run_slope(emtk_type type, int act, SlopeArgs &a, float *db0, float *db1, int sms, cudaStream_t s) {
    if (a.n == 0) return cudaSuccess;
    const SlopeShape h = slope_shape(a.m, a.n, sms, a.partial != nullptr);
    a.rows = h.rows;
    a.lanes_log2 = h.lanes_log2;
    const dim3 grid((unsigned)h.col_blocks, (unsigned)h.slices);
    const bool f16 = type == EMTK_TYPE_F16;
    cudaError_t e = a.partial ? (f16 ? start_slope<true, GATED, true>(a, act, grid, s)
                                     : start_slope<false, GATED, true>(a, act, grid, s))
                              : (f16 ? start_slope<true, GATED, false>(a, act, grid, s)
                                     : start_slope<false, GATED, false>(a, act, grid, s));
    if (e == cudaSuccess && a.partial)
        e = launch_pdl(slice_sum_kernel, dim3((unsigned)((a.n - 1) / 32 + 1), GATED ? 2u : 1u), dim3(32 * kSumWarps), 0,
                       s, static_cast<const float *>(a.partial), h.slices, a.n, db0, db1);
    return e;
}

// -------------------------------------------------------- checkpoints
// A warp takes rows, 256 columns of a row at a time (four threads hold a block
// of 32), up to four such pieces in flight; blocks along y share a row where
// there are few.
constexpr int kWarpCols = 32 * kVec;
constexpr int kPieces = 4;

template <bool F16>
__global__ void __launch_bounds__(kThreads) pack8_kernel(const Source x, uint8_t *q, int64_t q_ld, uint8_t *scale,
                                                         int64_t ld_scale, int m, int k, int wide) {
    const int lane = threadIdx.x & 31;
    const int step = (int)gridDim.y * kWarpCols;
    pdl_trigger();
    pdl_wait();
    for (int64_t r = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32; r < m;
         r += (int64_t)gridDim.x * (kThreads / 32)) {
        for (int64_t c0 = (int64_t)blockIdx.y * kWarpCols; c0 < k; c0 += (int64_t)kPieces * step) {
            float v[kPieces][kVec] = {};
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int64_t c = c0 + (int64_t)i * step + lane * kVec;
                if (c < k) load8<F16>(x, r, (int)c, k, v[i]);
            }
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                if (c0 + (int64_t)i * step >= k) break;  // the whole warp
                const int64_t c = c0 + (int64_t)i * step + lane * kVec;
                bool all_finite;
                float top = finite_top(v[i], all_finite);
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                if (c >= k) continue;
                const uint32_t b = q8_scale(top);
                const float inverse = q8_inverse(b);
                if ((lane & 3) == 0) scale[r * ld_scale + c / kQ8Block] = (uint8_t)b;
                uint8_t *p = q + r * q_ld + c;
                const uint2 w = make_uint2(q8_codes4(v[i], inverse, all_finite), q8_codes4(v[i] + 4, inverse, all_finite));
                if (wide && c + kVec <= k) {
                    *reinterpret_cast<uint2 *>(p) = w;
                } else {
#pragma unroll
                    for (int j = 0; j < kVec; ++j)
                        if (c + j < k) p[j] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j % 4)));
                }
            }
        }
    }
}

struct CopyArgs {
    struct One {
        Source from;
        uint16_t *to;
        int64_t to_ld;
        int rows, cols, wide;
    } job[kMaxCopies];
};

template <bool F16>
__global__ void __launch_bounds__(kThreads) copy16_kernel(const __grid_constant__ CopyArgs a) {
    const CopyArgs::One &j = a.job[blockIdx.z];
    const int lane = threadIdx.x & 31;
    const int step = (int)gridDim.y * kWarpCols;
    pdl_trigger();
    pdl_wait();
    for (int64_t r = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32; r < j.rows;
         r += (int64_t)gridDim.x * (kThreads / 32)) {
        for (int64_t c0 = (int64_t)blockIdx.y * kWarpCols + lane * kVec; c0 < j.cols; c0 += (int64_t)kPieces * step) {
            float v[kPieces][kVec];
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (c0 + (int64_t)i * step < j.cols) load8<F16>(j.from, r, (int)(c0 + (int64_t)i * step), j.cols, v[i]);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                if (c0 + (int64_t)i * step >= j.cols) break;
                if (j.from.scale) {
#pragma unroll
                    for (int t = 0; t < kVec; ++t) v[i][t] = q8_operand<F16>(v[i][t]);
                }
                store8<F16>(j.to + r * j.to_ld, (int)(c0 + (int64_t)i * step), j.cols, j.wide != 0, v[i]);
            }
        }
    }
}

// Rows over x, eight blocks an SM at most; columns over y where rows alone
// would leave the SMs short of warps.
dim3 row_grid(int m, int k, int sms, int jobs) {
    const int64_t most = (int64_t)8 * sms;
    const int64_t x = std::min<int64_t>(most, ((int64_t)m + kThreads / 32 - 1) / (kThreads / 32));
    const int64_t pieces = ((int64_t)k + kWarpCols - 1) / kWarpCols;
    const int64_t y = std::max<int64_t>(1, std::min<int64_t>(pieces, most / (2 * x)));
    return dim3((unsigned)x, (unsigned)y, (unsigned)jobs);
}

}  // namespace

int slope_slices(int m, int n, int sms) { return n > 0 ? slope_shape(m, n, sms, true).slices : 1; }

cudaError_t launch_slope(emtk_type type, int act, int m, int n, const emtk_matrix &dy, const emtk_matrix &pre,
                         void *dz, int64_t dz_ld, float *db, float *partial, int sms, cudaStream_t s) {
    SlopeArgs a{};
    a.dy = source_of(dy);
    if (act != EMTK_ACT_NONE) a.gate = source_of(pre);
    a.dg = static_cast<uint16_t *>(dz);
    a.d_ld = dz_ld;
    a.partial = db ? partial : nullptr;
    a.m = m;
    a.n = n;
    return run_slope<false>(type, act, a, db, nullptr, sms, s);
}

cudaError_t launch_gated_slope(emtk_type type, int act, int m, int f, const emtk_matrix &dh, const emtk_matrix &gate,
                               const emtk_matrix &up, void *dg, void *du, int64_t d_ld, const emtk_matrix &h,
                               float *db_gate, float *db_up, float *partial, int sms, cudaStream_t s) {
    SlopeArgs a{};
    a.dy = source_of(dh);
    a.gate = source_of(gate);
    a.up = source_of(up);
    a.dg = static_cast<uint16_t *>(dg);
    a.du = static_cast<uint16_t *>(du);
    a.d_ld = d_ld;
    a.h = static_cast<uint16_t *>(h.d);
    a.h_ld = h.ld;
    a.h_wide = h.d && aligned(h.d, 2 * h.ld, 16);
    a.partial = db_gate ? partial : nullptr;
    a.m = m;
    a.n = f;
    return run_slope<true>(type, act, a, db_gate, db_up, sms, s);
}

cudaError_t launch_pack8(emtk_type type, int m, int k, const emtk_matrix &x, const emtk_matrix &q, int sms,
                         cudaStream_t s) {
    if (m == 0 || k == 0) return cudaSuccess;
    const dim3 grid = row_grid(m, k, sms, 1);
    const int wide = aligned(q.d, q.ld, kVec);
    return launch_pdl(type == EMTK_TYPE_F16 ? pack8_kernel<true> : pack8_kernel<false>, grid, dim3(kThreads), 0, s,
                      source_of(x), static_cast<uint8_t *>(q.d), q.ld, q.d_scale, q.ld_scale, m, k, wide);
}

cudaError_t launch_copy16(emtk_type type, const Copy16 *copies, int n, int sms, cudaStream_t s) {
    CopyArgs a{};
    int rows = 0, cols = 0, jobs = 0;
    for (int i = 0; i < n; ++i) {
        const Copy16 &c = copies[i];
        if (c.rows == 0 || c.cols == 0) continue;
        a.job[jobs++] = {source_of(c.from), static_cast<uint16_t *>(c.to.d), c.to.ld, c.rows, c.cols,
                         aligned(c.to.d, 2 * c.to.ld, 16)};
        rows = std::max(rows, c.rows);
        cols = std::max(cols, c.cols);
    }
    if (jobs == 0) return cudaSuccess;
    return launch_pdl(type == EMTK_TYPE_F16 ? copy16_kernel<true> : copy16_kernel<false>,
                      row_grid(rows, cols, sms, jobs), dim3(kThreads), 0, s, a);
}

}  // namespace emtk
