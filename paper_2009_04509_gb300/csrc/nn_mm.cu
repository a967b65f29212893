// The layers' matrix products, on CUDA cores: a block computes a 64 x 64 tile
// of the output, 16 steps of the contraction at a time from shared memory, a
// thread 4 x 4 sums (two sets for the gated block).  Any row distance and
// alignment.
#include "nn_internal.h"
#include "nn_math.cuh"

namespace emtk {
namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256;

template <bool F16>
__device__ __forceinline__ float element(const MmOperand &o, int64_t i, int64_t t) {
    const uint16_t *p = static_cast<const uint16_t *>(o.p);
    return from16<F16>(o.across ? p[t * o.ld + i] : p[i * o.ld + t]);
}

template <bool F16>
__device__ __forceinline__ float load_bias(const MmEpilogue &e, int which, int n) {
    if (!e.bias[which]) return 0.f;
    return e.bias_f32 ? static_cast<const float *>(e.bias[which])[n]
                      : from16<F16>(static_cast<const uint16_t *>(e.bias[which])[n]);
}

template <bool F16, bool GATED>
__global__ void __launch_bounds__(kThreads) mm_kernel(const MmJob job) {
    __shared__ float sa[kStep][kTile + 1], sb[GATED ? 2 : 1][kStep][kTile + 1];
    __shared__ float sz[GATED ? 2 : 1][kTile][kTile + 1];
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int64_t i0 = (int64_t)blockIdx.y * kTile, j0 = (int64_t)blockIdx.x * kTile;
    float acc[GATED ? 2 : 1][4][4] = {};
    for (int term = 0; term < job.terms; ++term) {
        for (int t0 = 0; t0 < job.K; t0 += kStep) {
            __syncthreads();
            for (int e = threadIdx.x; e < kTile * kStep; e += kThreads) {
                const int i = e / kStep, t = e % kStep;
                const bool in = t0 + t < job.K;
                sa[t][i] = in && i0 + i < job.M ? element<F16>(job.a[term], i0 + i, t0 + t) : 0.f;
                for (int w = 0; w < (GATED ? 2 : 1); ++w)
                    sb[w][t][i] = in && j0 + i < job.N ? element<F16>(job.b[GATED ? w : term], j0 + i, t0 + t) : 0.f;
            }
            __syncthreads();
            for (int t = 0; t < kStep; ++t)
#pragma unroll
                for (int w = 0; w < (GATED ? 2 : 1); ++w)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            acc[w][i][j] = fmaf(sa[t][ty + 16 * i], sb[w][t][tx + 16 * j], acc[w][i][j]);
        }
    }
    const MmEpilogue &e = job.epi;
#pragma unroll
    for (int w = 0; w < (GATED ? 2 : 1); ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t n = j0 + tx + 16 * j;
                sz[w][ty + 16 * i][tx + 16 * j] =
                    n < job.N ? acc[w][i][j] + load_bias<F16>(e, w, (int)n) : 0.f;
            }
    __syncthreads();
    // a thread takes 16 columns of a row, half a checkpoint block
    const int r = threadIdx.x / 4, c0 = (threadIdx.x % 4) * 16;
    const int64_t i = i0 + r;
    const bool row_in = i < job.M;
#pragma unroll
    for (int w = 0; w < (GATED ? 2 : 1); ++w) {
        const emtk_matrix &m = e.saved[w];
        if (!m.d) continue;
        float inverse = 0.f;
        if (m.d_scale) {
            float top = 0.f;
            for (int c = 0; c < 16; ++c) top = fmaxf(top, finite_abs(sz[w][r][c0 + c]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            const uint32_t b = q8_scale(top);
            inverse = q8_inverse(b);
            if (row_in && (threadIdx.x & 1) == 0 && j0 + c0 < job.N)
                m.d_scale[i * m.ld_scale + (j0 + c0) / kQ8Block] = (uint8_t)b;
        }
        for (int c = 0; c < 16; ++c) {
            const int64_t j = j0 + c0 + c;
            if (!row_in || j >= job.N) continue;
            if (m.d_scale)
                static_cast<uint8_t *>(m.d)[i * m.ld + j] = (uint8_t)q8_code(sz[w][r][c0 + c], inverse);
            else
                static_cast<uint16_t *>(m.d)[i * m.ld + j] = (uint16_t)to16<F16>(sz[w][r][c0 + c]);
        }
    }
    for (int c = 0; c < 16; ++c) {
        const int64_t j = j0 + c0 + c;
        if (!row_in || j >= job.N) continue;
        float v = act_f(e.act, sz[0][r][c0 + c]);
        if (GATED) v *= sz[GATED ? 1 : 0][r][c0 + c];
        if (e.residual.d) v += from16<F16>(static_cast<const uint16_t *>(e.residual.d)[i * e.residual.ld + j]);
        if (e.out_f32)
            static_cast<float *>(e.out.d)[i * e.out.ld + j] = v;
        else
            static_cast<uint16_t *>(e.out.d)[i * e.out.ld + j] = (uint16_t)to16<F16>(v);
    }
}

}  // namespace

cudaError_t launch_mm(const MmJob &job, const emtk_nn *, cudaStream_t s) {
    if (job.M == 0 || job.N == 0) return cudaSuccess;
    const dim3 grid((job.N - 1) / kTile + 1, (job.M - 1) / kTile + 1);
    const bool f16 = job.type == EMTK_TYPE_F16;
    if (job.kind == kMmGated)
        f16 ? mm_kernel<true, true><<<grid, kThreads, 0, s>>>(job) : mm_kernel<false, true><<<grid, kThreads, 0, s>>>(job);
    else
        f16 ? mm_kernel<true, false><<<grid, kThreads, 0, s>>>(job)
            : mm_kernel<false, false><<<grid, kThreads, 0, s>>>(job);
    return cudaGetLastError();
}

}  // namespace emtk
