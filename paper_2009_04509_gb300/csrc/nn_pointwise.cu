// Pointwise passes of the dense and gated layers' gradients, and the 8-bit
// checkpoints.  All of them stream: every element is read once with 16-byte
// loads (8 columns a thread) where address and row distance allow it, one
// element at a time where they do not, and what bounds them is HBM.
#include <algorithm>

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
        if (s.access == kWideQ8 && full) {
            const uint2 w = __ldg(reinterpret_cast<const uint2 *>(p));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = q8_value((w.x >> (8 * i)) & 0xffu, step);
                v[i + 4] = q8_value((w.y >> (8 * i)) & 0xffu, step);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = c + i < n ? q8_value(__ldg(p + i), step) : 0.f;
        }
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
// a thread adds its rows in order and the block adds its threads' sums in
// order, so the column sums do not depend on timing.
struct SlopeShape {
    int lanes_log2;  // threads across
    int col_blocks, slices;
    int rows;  // of a slice
};

SlopeShape slope_shape(int m, int n, int sms) {
    SlopeShape h;
    h.lanes_log2 = 5;
    while (h.lanes_log2 > 2 && (kVec << (h.lanes_log2 - 1)) >= n) --h.lanes_log2;
    const int cols = kVec << h.lanes_log2;
    const int at_once = kThreads >> h.lanes_log2;
    h.col_blocks = (int)(((int64_t)n + cols - 1) / cols);
    // about four blocks an SM, each of at least two passes over its rows
    int64_t slices = std::max<int64_t>(1, (int64_t)4 * sms / std::max(1, h.col_blocks));
    slices = std::min<int64_t>(slices, std::max<int64_t>(1, ((int64_t)m + 2 * at_once - 1) / (2 * at_once)));
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
    int m, n, act, rows, lanes_log2;
};

template <bool F16, bool GATED>
__global__ void __launch_bounds__(kThreads) slope_kernel(const SlopeArgs a) {
    const int lanes = 1 << a.lanes_log2;
    const int at_once = kThreads >> a.lanes_log2;
    const int c = (int)blockIdx.x * (kVec << a.lanes_log2) + (threadIdx.x & (lanes - 1)) * kVec;
    const int sub = threadIdx.x >> a.lanes_log2;
    const int64_t r0 = (int64_t)blockIdx.y * a.rows;
    const int64_t r1 = min(r0 + a.rows, (int64_t)a.m);
    float sg[kVec] = {}, su[kVec] = {};
    if (c < a.n) {
        for (int64_t r = r0 + sub; r < r1; r += at_once) {
            float d[kVec], g[kVec], dg[kVec];
            load8<F16>(a.dy, r, c, a.n, d);
            if (a.gate.access != kAbsent) load8<F16>(a.gate, r, c, a.n, g);
            if (GATED) {
                float u[kVec], du[kVec], h[kVec];
                load8<F16>(a.up, r, c, a.n, u);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    float f, s;
                    act_slope(a.act, g[i], f, s);
                    dg[i] = d[i] * u[i] * s;
                    du[i] = d[i] * f;
                    h[i] = f * u[i];
                    su[i] += du[i];
                }
                if (a.du) store8<F16>(a.du + r * a.d_ld, c, a.n, true, du);
                if (a.h) store8<F16>(a.h + r * a.h_ld, c, a.n, a.h_wide != 0, h);
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    float f, s = 1.f;
                    if (a.gate.access != kAbsent) act_slope(a.act, g[i], f, s);
                    dg[i] = d[i] * s;
                }
            }
#pragma unroll
            for (int i = 0; i < kVec; ++i) sg[i] += dg[i];
            if (a.dg) store8<F16>(a.dg + r * a.d_ld, c, a.n, true, dg);
        }
    }
    if (!a.partial) return;
    __shared__ float part[kThreads * kVec];
#pragma unroll
    for (int half = 0; half < (GATED ? 2 : 1); ++half) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kVec; ++i) part[threadIdx.x * kVec + i] = half ? su[i] : sg[i];
        __syncthreads();
        const int cols = kVec << a.lanes_log2;
        const int col = (int)blockIdx.x * cols + (int)threadIdx.x;
        if ((int)threadIdx.x < cols && col < a.n) {
            float sum = 0.f;
            for (int g = 0; g < at_once; ++g) sum += part[g * cols + threadIdx.x];
            a.partial[((int64_t)half * gridDim.y + blockIdx.y) * a.n + col] = sum;
        }
    }
}

// Column sums from the slices' partial sums, in slice order.
__global__ void __launch_bounds__(kThreads) slice_sum_kernel(const float *partial, int slices, int n, float *db0,
                                                             float *db1) {
    const int c = (int)blockIdx.x * kThreads + (int)threadIdx.x;
    if (c >= n) return;
    const float *p = partial + (int64_t)blockIdx.y * slices * n + c;
    float sum = 0.f;
#pragma unroll 8
    for (int s = 0; s < slices; ++s) sum += p[(int64_t)s * n];
    (blockIdx.y ? db1 : db0)[c] = sum;
}

template <bool GATED>
cudaError_t run_slope(emtk_type type, SlopeArgs &a, float *db0, float *db1, int sms, cudaStream_t s) {
    if (a.n == 0) return cudaSuccess;
    const SlopeShape h = slope_shape(a.m, a.n, sms);
    a.rows = h.rows;
    a.lanes_log2 = h.lanes_log2;
    const dim3 grid((unsigned)h.col_blocks, (unsigned)h.slices);
    if (type == EMTK_TYPE_F16)
        slope_kernel<true, GATED><<<grid, kThreads, 0, s>>>(a);
    else
        slope_kernel<false, GATED><<<grid, kThreads, 0, s>>>(a);
    if (a.partial)
        slice_sum_kernel<<<dim3((unsigned)((a.n - 1) / kThreads + 1), GATED ? 2u : 1u), kThreads, 0, s>>>(
            a.partial, h.slices, a.n, db0, db1);
    return cudaGetLastError();
}

// -------------------------------------------------------- checkpoints
// A warp takes 256 columns of a row: four threads hold a block of 32.
constexpr int kWarpCols = 32 * kVec;

template <bool F16>
__global__ void __launch_bounds__(kThreads) pack8_kernel(Source x, uint8_t *q, int64_t q_ld, uint8_t *scale,
                                                         int64_t ld_scale, int64_t items, int per_row, int k,
                                                         int wide) {
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (kThreads / 32);
    for (int64_t it = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32; it < items; it += warps) {
        const int64_t r = it / per_row;
        const int c = (int)(it - r * per_row) * kWarpCols + lane * kVec;
        float v[kVec] = {};
        if (c < k) load8<F16>(x, r, c, k, v);
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) top = fmaxf(top, finite_abs(v[i]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        if (c >= k) continue;
        const uint32_t b = q8_scale(top);
        const float inverse = q8_inverse(b);
        if ((lane & 3) == 0) scale[r * ld_scale + c / kQ8Block] = (uint8_t)b;
        uint8_t *p = q + r * q_ld + c;
        if (wide && c + kVec <= k) {
            uint32_t w[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < kVec; ++i) w[i / 4] |= q8_code(v[i], inverse) << (8 * (i % 4));
            *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (c + i < k) p[i] = (uint8_t)q8_code(v[i], inverse);
        }
    }
}

template <bool F16>
__global__ void __launch_bounds__(kThreads) copy16_kernel(Source src, uint16_t *x, int64_t x_ld, int64_t items,
                                                           int per_row, int k, int wide) {
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (kThreads / 32);
    for (int64_t it = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32; it < items; it += warps) {
        const int64_t r = it / per_row;
        const int c = (int)(it - r * per_row) * kWarpCols + lane * kVec;
        if (c >= k) continue;
        float v[kVec];
        load8<F16>(src, r, c, k, v);
        if (src.scale) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = q8_operand<F16>(v[i]);
        }
        store8<F16>(x + r * x_ld, c, k, wide != 0, v);
    }
}

struct WarpGrid {
    int64_t items;
    int per_row;
    unsigned blocks;
};
WarpGrid warp_grid(int m, int k, int sms) {
    WarpGrid g;
    g.per_row = (int)(((int64_t)k + kWarpCols - 1) / kWarpCols);
    g.items = (int64_t)m * g.per_row;
    const int64_t blocks = (g.items + kThreads / 32 - 1) / (kThreads / 32);
    g.blocks = (unsigned)std::min<int64_t>(blocks, (int64_t)16 * sms);
    return g;
}

}  // namespace

int slope_slices(int m, int n, int sms) { return n > 0 ? slope_shape(m, n, sms).slices : 1; }

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
    a.act = act;
    return run_slope<false>(type, a, db, nullptr, sms, s);
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
    a.act = act;
    return run_slope<true>(type, a, db_gate, db_up, sms, s);
}

cudaError_t launch_pack8(emtk_type type, int m, int k, const emtk_matrix &x, const emtk_matrix &q, int sms,
                         cudaStream_t s) {
    if (m == 0 || k == 0) return cudaSuccess;
    const WarpGrid g = warp_grid(m, k, sms);
    const int wide = aligned(q.d, q.ld, kVec);
    uint8_t *d = static_cast<uint8_t *>(q.d);
    if (type == EMTK_TYPE_F16)
        pack8_kernel<true><<<g.blocks, kThreads, 0, s>>>(source_of(x), d, q.ld, q.d_scale, q.ld_scale, g.items,
                                                         g.per_row, k, wide);
    else
        pack8_kernel<false><<<g.blocks, kThreads, 0, s>>>(source_of(x), d, q.ld, q.d_scale, q.ld_scale, g.items,
                                                          g.per_row, k, wide);
    return cudaGetLastError();
}

cudaError_t launch_copy16(emtk_type type, int m, int k, const emtk_matrix &src, const emtk_matrix &x, int sms,
                          cudaStream_t s) {
    if (m == 0 || k == 0) return cudaSuccess;
    const WarpGrid g = warp_grid(m, k, sms);
    const int wide = aligned(x.d, 2 * x.ld, 16);
    uint16_t *d = static_cast<uint16_t *>(x.d);
    if (type == EMTK_TYPE_F16)
        copy16_kernel<true><<<g.blocks, kThreads, 0, s>>>(source_of(src), d, x.ld, g.items, g.per_row, k, wide);
    else
        copy16_kernel<false><<<g.blocks, kThreads, 0, s>>>(source_of(src), d, x.ld, g.items, g.per_row, k, wide);
    return cudaGetLastError();
}

}  // namespace emtk
