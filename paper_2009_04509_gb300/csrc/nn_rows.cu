// The layers' forward pass for a few rows (single tokens or hits), on CUDA cores.
//
// With 1 to 4 rows every weight is used a handful of times, so the time is that
// of reading the weights once: a warp holds four weight rows (of the gated
// block: two of each projection) and one piece of the contraction, 16 bytes a
// lane and row at a time, and multiplies them with the rows of x, which come
// from L1.  The warps of a group hold different pieces and add their sums in
// shared memory, in order.  A tile of the tensor-core kernel would be 97% zero
// rows and needs a second kernel to join its split contraction.  Four rows a warp
// and no unrolling measured best (4096 -> 2 x 10240 gated, one row, bf16: 25.4 us, 6.6
// TB/s, with blocks of 8 warps 26.0; two or eight weight rows a warp 31.6, unrolled
// twice 27.5).  HBM bounds it from 50 MB of weights on; 4096 -> 4096 takes 7.4 us with
// the weights from HBM, of which 5 are their bytes (5.8 from L2).
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_math.cuh"

namespace emtk {
namespace {

constexpr int kMostWarps = 8;  // of a block
constexpr int kHeld = 4;  // weight rows of a warp

struct RowsParams {
    const uint16_t *x, *w[2];
    int64_t x_ld, w_ld[2];
    MmEpilogue epi;
    int N, K;
    int split_log2;  // warps of a group
};

__device__ __forceinline__ uint4 load_once(const uint16_t *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

template <bool F16>
__device__ __forceinline__ void unpack(const uint4 &q, float (&v)[8]) {
    const uint32_t x[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = F16 ? from16<F16>(x[i] & 0xffffu) : __uint_as_float(x[i] << 16);
        v[2 * i + 1] = F16 ? from16<F16>(x[i] >> 16) : __uint_as_float(x[i] & 0xffff0000u);
    }
}

// ROWS: rows of x.  WIDE: every row of x and w starts on 16 bytes.
template <bool F16, bool GATED, int ROWS, bool WIDE>
__global__ void __launch_bounds__(32 * kMostWarps) rows_kernel(const __grid_constant__ RowsParams p) {
    constexpr int kOut = GATED ? kHeld / 2 : kHeld;  // output columns of a group
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const int split = 1 << p.split_log2, part = warp & (split - 1);
    const int64_t n0 = ((int64_t)blockIdx.x * (blockDim.x >> (5 + p.split_log2)) + (warp >> p.split_log2)) * kOut;
    const uint16_t *w[kHeld];
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
        const int which = GATED ? r / kOut : 0;
        w[r] = p.w[which] + min(n0 + r % kOut, (int64_t)p.N - 1) * p.w_ld[which];  // past the end: read, not stored
    }
    float acc[kHeld][ROWS] = {};
    pdl_trigger();
    pdl_wait();
    int done = 0;
    if (WIDE) {
        done = p.K / 8 * 8;
#pragma unroll 1
        for (int k = (part * 32 + lane) * 8; k < done; k += split * 256) {
            uint4 q[kHeld], xq[ROWS];
#pragma unroll
            for (int r = 0; r < kHeld; ++r) q[r] = load_once(w[r] + k);
#pragma unroll
            for (int i = 0; i < ROWS; ++i) xq[i] = __ldg(reinterpret_cast<const uint4 *>(p.x + i * p.x_ld + k));
            float xv[ROWS][8];
#pragma unroll
            for (int i = 0; i < ROWS; ++i) unpack<F16>(xq[i], xv[i]);
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
                float wv[8];
                unpack<F16>(q[r], wv);
#pragma unroll
                for (int i = 0; i < ROWS; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[r][i] = fmaf(wv[j], xv[i][j], acc[r][i]);
            }
        }
    }
    // one element a lane: all of the contraction, or what 16-byte pieces leave
#pragma unroll 4
    for (int k = done + part * 32 + lane; k < p.K; k += split * 32) {
        float wv[kHeld];
#pragma unroll
        for (int r = 0; r < kHeld; ++r) wv[r] = from16<F16>(__ldg(w[r] + k));
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const float xv = from16<F16>(__ldg(p.x + i * p.x_ld + k));
#pragma unroll
            for (int r = 0; r < kHeld; ++r) acc[r][i] = fmaf(wv[r], xv, acc[r][i]);
        }
    }
#pragma unroll
    for (int r = 0; r < kHeld; ++r)
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) acc[r][i] += __shfl_xor_sync(0xffffffffu, acc[r][i], d);
    __shared__ float sums[kMostWarps][kHeld * ROWS];
    if (lane == 0) {
#pragma unroll
        for (int r = 0; r < kHeld; ++r)
#pragma unroll
            for (int i = 0; i < ROWS; ++i) sums[warp][r * ROWS + i] = acc[r][i];
    }
    __syncthreads();
    // lane (column c, row i) of each group's first warp finishes one output
    const int c = lane / ROWS, i = lane % ROWS;
    if (part != 0 || c >= kOut || n0 + c >= p.N) return;
    const MmEpilogue &e = p.epi;
    const int64_t n = n0 + c;
    float z[GATED ? 2 : 1];
#pragma unroll
    for (int h = 0; h < (GATED ? 2 : 1); ++h) {
        z[h] = 0.f;
        for (int s = 0; s < split; ++s) z[h] += sums[warp + s][(h * kOut + c) * ROWS + i];
        if (e.bias[h])
            z[h] += e.bias_f32 ? __ldg(static_cast<const float *>(e.bias[h]) + n)
                               : from16<F16>(__ldg(static_cast<const uint16_t *>(e.bias[h]) + n));
        const emtk_matrix &m = e.saved[h];
        if (m.d) static_cast<uint16_t *>(m.d)[i * m.ld + n] = (uint16_t)to16<F16>(z[h]);
    }
    float a[1] = {z[0]};
    apply_act(e.act, a);
    float y = a[0];
    if (GATED) y *= z[GATED ? 1 : 0];
    if (e.residual.d) y += from16<F16>(static_cast<const uint16_t *>(e.residual.d)[i * e.residual.ld + n]);
    static_cast<uint16_t *>(e.out.d)[i * e.out.ld + n] = (uint16_t)to16<F16>(y);
}

template <bool F16, bool GATED, int ROWS>
cudaError_t run(const RowsParams &p, unsigned warps, unsigned blocks, bool wide, cudaStream_t s) {
    if (wide) return launch_pdl(rows_kernel<F16, GATED, ROWS, true>, dim3(blocks), dim3(32 * warps), 0, s, p);
    return launch_pdl(rows_kernel<F16, GATED, ROWS, false>, dim3(blocks), dim3(32 * warps), 0, s, p);
}

template <bool F16, bool GATED>
cudaError_t run(const RowsParams &p, int rows, unsigned warps, unsigned blocks, bool wide, cudaStream_t s) {
    switch (rows) {
        case 1: return run<F16, GATED, 1>(p, warps, blocks, wide, s);
        case 2: return run<F16, GATED, 2>(p, warps, blocks, wide, s);
        case 3: return run<F16, GATED, 3>(p, warps, blocks, wide, s);
        default: return run<F16, GATED, 4>(p, warps, blocks, wide, s);
    }
}

}  // namespace

namespace {
// Every row of the operands starts on 16 bytes.
bool wide_operands(const MmJob &j) {
    bool wide = mm_operand_ok(j.a[0].p, j.a[0].ld, j.M);
    for (int i = 0; i < (j.kind == kMmGated ? 2 : 1); ++i) wide = wide && mm_operand_ok(j.b[i].p, j.b[i].ld, j.N);
    return wide;
}
}  // namespace

// Up to 2 rows; of 3 and 4 only where TMA cannot read the weights as they lie and
// nn_skinny.cu would have to copy them first.  bf16, weights from HBM, 1, 2, 3, 4 rows:
//                                  here                nn_skinny.cu
//   4096 -> 2 x 10240 gated, wide  25.3 28.7 31.9 34.9 29.9 31.2 30.6 30.2
//     rows of 4097 elements        70   88   64   97   88 for each
//   4096 -> 4096 dense, wide       7.4  7.4  9.9  11.6 9.5 for each
//     rows of 4097 elements        25   32   18   21   17.6 for each: the copy stays in L2
// Checkpoints are left to the kernels that hold 32 columns of a row together.
bool few_rows(const MmJob &j) {
    return j.M <= 4 && (j.M <= 2 || !wide_operands(j)) && !j.epi.saved[0].d_scale && !j.epi.saved[1].d_scale;
}

cudaError_t launch_rows(const MmJob &j, int sms, cudaStream_t s) {
    const bool gated = j.kind == kMmGated;
    RowsParams p{};
    p.x = static_cast<const uint16_t *>(j.a[0].p);
    p.x_ld = j.a[0].ld;
    const bool wide = wide_operands(j);
    for (int i = 0; i < (gated ? 2 : 1); ++i) {
        p.w[i] = static_cast<const uint16_t *>(j.b[i].p);
        p.w_ld[i] = j.b[i].ld;
    }
    p.epi = j.epi;
    p.N = j.N;
    p.K = j.K;
    // Warps of a group: one for every four steps of 256 (a longer way leaves the end of
    // the launch uneven), and more down to a step each while an SM has fewer than 16.
    // One row, bf16, the same weights each time: 8192 -> 2 x 8192 with 8 warps 39.6 us, 4
    // 40.6, 2 44.7; 4096 -> 4096 with 4 warps 7.3 us in a row, 8 7.6, 2 8.8; 1024 -> 2 x 4096 with 2 4.7 us, 4 5.0.
    const int out = gated ? kHeld / 2 : kHeld;
    const int64_t groups = ((int64_t)j.N + out - 1) / out;
    while (p.split_log2 < 3 && (1024 << (p.split_log2 + 1)) <= j.K) ++p.split_log2;
    while ((1 << p.split_log2) < kMostWarps && (256 << (p.split_log2 + 1)) <= j.K && (groups << p.split_log2) < (int64_t)16 * sms)
        ++p.split_log2;
    const unsigned warps = std::max(4u, 1u << p.split_log2);
    const int64_t per_block = (int64_t)(warps >> p.split_log2) * out;
    const unsigned blocks = (unsigned)((j.N + per_block - 1) / per_block);
    if (j.type == EMTK_TYPE_F16)
        return gated ? run<true, true>(p, j.M, warps, blocks, wide, s) : run<true, false>(p, j.M, warps, blocks, wide, s);
    return gated ? run<false, true>(p, j.M, warps, blocks, wide, s) : run<false, false>(p, j.M, warps, blocks, wide, s);
}

}  // namespace emtk
