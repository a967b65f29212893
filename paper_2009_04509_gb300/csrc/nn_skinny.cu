// The layers' forward pass for up to 64 rows, on the tcgen05 tensor cores.
//
// The time is that of reading the weights once.  So the weights take the MMA's
// 128 rows (of the gated block 64 rows of each projection) and the rows of x its
// 16, 32 or 64 columns: every byte staged by TMA but x's is a weight, where a
// tile of nn_mm.cu would stage 256 mostly empty rows of x.  Two CTAs of about
// 105 KB share an SM, so that one's set-up and epilogue run beside the other's
// stream.  Where the output tiles are fewer than the CTAs that fit, a cluster of
// up to 8 CTAs splits the contraction: each leaves its fp32 sums in shared
// memory, and every CTA adds the cluster's sums for its share of the rows, in
// rank order, over distributed shared memory; no second kernel, no workspace.
//
// HBM bounds it.  4096 -> 2 x 10240 gated, bf16 (168 MB of weights): 31 us for 8 rows,
// 32 for 16, 38 for 64 (5.4, 5.2 and 4.5 TB/s); 4096 -> 10240 dense: 18 us for 8 rows.
// With all CTAs starting at the same chunk 16 rows took 56 us.  What is left to the
// copy's 6.8 TB/s is the ramp and, from 32 rows on, the epilogue.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_math.cuh"
#include "nn_ptx.cuh"

namespace emtk {
namespace {

constexpr int kThreads = 128;
constexpr int kStep = 64;                    // contraction steps of a chunk: 128 bytes
constexpr int kWeightRows = 128;
constexpr int kWBytes = kWeightRows * kStep * 2;
constexpr int kMostParts = 8;                // portable cluster size

template <int NT>  // columns of the MMA: rows of x
struct Shape {
    static constexpr int kChunk = kWBytes + NT * kStep * 2;
    static constexpr int kSlots = NT == 16 ? 6 : NT == 32 ? 5 : 4;
    static constexpr int kTmemCols = NT < 32 ? 32 : NT;
    static constexpr int kSmem = 1024 + kSlots * kChunk + 256;
};
static_assert(Shape<16>::kSmem <= 113 * 1024 && Shape<32>::kSmem <= 113 * 1024 && Shape<64>::kSmem <= 113 * 1024,
              "two CTAs an SM");
static_assert(64 * kWeightRows * 4 <= 4 * Shape<64>::kChunk, "the sums take the slots' place");

struct SkinnyParams {
    CUtensorMap w[2], x;
    MmEpilogue epi;
    int M, N, K, parts, chunks_per_part, chunks;
    int *status;
    int64_t timeout_ns;
    int debug_stall;
};

__device__ __forceinline__ float load_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(
            dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}

enum Bar : int { kBarFull = 0, kBarEmpty = 6, kBarAcc = 12, kBarDrain = 13, kBarStall = 14, kBars = 15 };

template <bool F16, bool GATED, int NT>
__global__ void __launch_bounds__(kThreads) skinny_kernel(const __grid_constant__ SkinnyParams p) {
    using S = Shape<NT>;
    constexpr int kOut = GATED ? kWeightRows / 2 : kWeightRows;  // output columns of a tile
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    uint8_t *const base = smem_raw + ((1024u - (raw & 1023u)) & 1023u);
    const uint32_t slots = smem_u32(base);
    uint64_t *const bars = reinterpret_cast<uint64_t *>(base + S::kSlots * S::kChunk);
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(bars + kBars);
    volatile uint32_t *const abort_flag = tmem_slot + 1;
    auto bar = [&](int i) { return smem_u32(bars + i); };

    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank();
    const int n0 = (int)(blockIdx.x / p.parts) * kOut;
    const int c0 = rank * p.chunks_per_part, c1 = min(c0 + p.chunks_per_part, p.chunks);
    const Guard guard{abort_flag, p.status, p.timeout_ns};

    pdl_trigger();
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kSlots; ++s) {
            mbar_init(bar(kBarFull + s), 1);
            mbar_init(bar(kBarEmpty + s), 1);
        }
        for (int b : {kBarAcc, kBarDrain, kBarStall}) mbar_init(bar(b), 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(S::kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();

    if (warp == 0) {
        // ---------------------------------------------------- TMA producer
        bool ok = !(p.debug_stall && !warp_wait(bar(kBarStall), 0u, guard, lane));
        // Each tile starts at another chunk of its part and wraps around: in step, all
        // CTAs would read the same few address bits of their rows at a time.
        int at = c0 + (int)(blockIdx.x / p.parts * 5u) % max(1, c1 - c0);
        int s = 0;
        uint32_t phase = 1;  // a fresh barrier's previous phase counts as complete
        for (int c = c0; ok && c < c1; ++c) {
            if (!warp_wait_all(bar(kBarEmpty + s), phase, guard, lane)) {
                ok = false;
                break;
            }
            if (elect_one()) {
                const uint32_t sw = slots + s * S::kChunk;
                mbar_expect_tx_relaxed(bar(kBarFull + s), S::kChunk);
                tma_load_2d(sw, &p.w[0], bar(kBarFull + s), at * kStep, n0);
                if (GATED) tma_load_2d(sw + kWBytes / 2, &p.w[1], bar(kBarFull + s), at * kStep, n0);
                tma_load_2d(sw + kWBytes, &p.x, bar(kBarFull + s), at * kStep, 0);
            }
            __syncwarp();
            if (++at == c1) at = c0;
            if (++s == S::kSlots) {
                s = 0;
                phase ^= 1;
            }
        }
        if (!ok) {  // copies in flight land within microseconds: leave them a millisecond
            const uint64_t t0 = global_timer_ns();
            while (global_timer_ns() - t0 < 1000000u) {
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------ MMA issuer
        constexpr uint32_t idesc = make_idesc(kWeightRows, NT, F16);
        int s = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int c = c0; c < c1; ++c) {
            if (!warp_wait_all(bar(kBarFull + s), phase, guard, lane)) {
                ok = false;
                break;
            }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t dw = sw128_desc(slots + s * S::kChunk), dx = sw128_desc(slots + s * S::kChunk + kWBytes);
#pragma unroll
                for (int i = 0; i < kStep / 16; ++i)
                    mma_ss(tmem, dw + 2 * i, dx + 2 * i, idesc, (i > 0 || c > c0) ? 1u : 0u);
                mma_commit(bar(kBarEmpty + s));
            }
            __syncwarp();
            if (++s == S::kSlots) {
                s = 0;
                phase ^= 1;
            }
        }
        if (elect_one()) {
            if (ok) mma_commit(bar(kBarAcc));
            mma_commit(bar(kBarDrain));  // every MMA issued completes before TMEM is released
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait(bar(kBarDrain), 0u) && (int64_t)(global_timer_ns() - t0) < p.timeout_ns) {
            }
        }
        __syncwarp();
    }
    __syncwarp();

    // ------------------------------------------------------------ epilogue
    // Sums out of TMEM (lane = weight row, column = row of x) into the slots, which
    // nothing reads or writes any more: [row of x][weight row].
    float *const sums = reinterpret_cast<float *>(base);
    const bool ok = warp_wait(bar(kBarAcc), 0u, guard, lane);
    tc_fence_after();
    if (ok) {
        const uint32_t acc = tmem + ((uint32_t)(32 * warp) << 16);
        float *const mine = sums + 32 * warp + lane;
#pragma unroll
        for (int t = 0; t < NT; t += 16) {
            uint32_t r[16];
            tmem_ld16<0>(acc + t, r);
            tmem_ld_wait();
            reg_fence(r);
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[(t + i) * kWeightRows] = c0 < c1 ? __uint_as_float(r[i]) : 0.f;
        }
    }
    tc_fence_before();
    cluster_sync();
    // Rows rank, rank + parts, ..: a thread's output column stays its own.
    const MmEpilogue &e = p.epi;
    const int col = threadIdx.x % kOut, first = rank + p.parts * (threadIdx.x / kOut);
    const int n = n0 + col;
    const bool in = n < p.N;
    float bias[GATED ? 2 : 1] = {};
#pragma unroll
    for (int h = 0; h < (GATED ? 2 : 1); ++h)
        if (e.bias[h] && in)
            bias[h] = e.bias_f32 ? __ldg(static_cast<const float *>(e.bias[h]) + n)
                                 : from16<F16>(__ldg(static_cast<const uint16_t *>(e.bias[h]) + n));
    // four rows at a time: their remote loads and stores are independent
    constexpr int kRows = 4, kSums = GATED ? 2 : 1;
    const int step = p.parts * (kThreads / kOut);
    for (int t0 = first; t0 < p.M; t0 += kRows * step) {
        float z[kRows][kSums], y[kRows];
        uint16_t res[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int t = min(t0 + i * step, p.M - 1);
            res[i] = !GATED && e.residual.d && in
                         ? static_cast<const uint16_t *>(e.residual.d)[t * e.residual.ld + n] : (uint16_t)0;
        }
        for (int r = 0; r < p.parts; ++r) {
            const uint32_t from = cluster_addr(smem_u32(sums + col), r);
#pragma unroll
            for (int i = 0; i < kRows; ++i)
#pragma unroll
                for (int h = 0; h < kSums; ++h) {
                    const float v = load_cluster(from + 4 * ((t0 + i * step) % NT * kWeightRows + h * kOut));
                    z[i][h] = r == 0 ? v : z[i][h] + v;
                }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int t = t0 + i * step;
            if (t >= p.M) break;  // the whole warp
#pragma unroll
            for (int h = 0; h < kSums; ++h) {
                const float v = z[i][h] += bias[h];
                const emtk_matrix &m = e.saved[h];
                if (m.d == nullptr) continue;
                if (m.d_scale) {  // a warp's lanes are one block of 32 columns
                    const bool finite = fabsf(v) < __int_as_float(0x7f800000);
                    const uint32_t top = __reduce_max_sync(0xffffffffu, in && finite ? __float_as_uint(fabsf(v)) : 0u);
                    const uint32_t b = q8_scale(__uint_as_float(top));
                    if (in && lane == 0) m.d_scale[t * m.ld_scale + n / kQ8Block] = (uint8_t)b;
                    if (in)
                        static_cast<uint8_t *>(m.d)[t * m.ld + n] =
                            (uint8_t)(finite ? __float_as_uint(fmaf(v, q8_inverse(b), 12582912.f)) : 0x80u);
                } else if (in) {
                    static_cast<uint16_t *>(m.d)[t * m.ld + n] = (uint16_t)to16<F16>(v);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) y[i] = z[i][0];
        apply_act(e.act, y);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int t = t0 + i * step;
            if (GATED) y[i] *= z[i][kSums - 1];
            if (!GATED && e.residual.d) y[i] += from16<F16>(res[i]);
            if (in && t < p.M) static_cast<uint16_t *>(e.out.d)[t * e.out.ld + n] = (uint16_t)to16<F16>(y[i]);
        }
    }
    cluster_sync();  // the cluster's sums have been read
    tc_fence_after();
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols));
}

template <bool F16, bool GATED, int NT>
cudaError_t run(const SkinnyParams &p, unsigned ctas, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Shape<NT>::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.parts;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, skinny_kernel<F16, GATED, NT>, p);
}

template <bool F16, bool GATED>
cudaError_t run(const SkinnyParams &p, int nt, unsigned ctas, cudaStream_t s) {
    if (nt == 16) return run<F16, GATED, 16>(p, ctas, s);
    if (nt == 32) return run<F16, GATED, 32>(p, ctas, s);
    return run<F16, GATED, 64>(p, ctas, s);
}

int tiles_of(const MmJob &j) {
    const int out = j.kind == kMmGated ? kWeightRows / 2 : kWeightRows;
    return (int)(((int64_t)j.N + out - 1) / out);
}
int chunks_of(const MmJob &j) { return (int)(((int64_t)j.K + kStep - 1) / kStep); }

}  // namespace

// A cluster splits the contraction 8 ways at most, so a few columns with a very
// long contraction are left to nn_mm.cu, which splits it over all SMs.
bool skinny(const MmJob &j) {
    return j.M <= 64 && j.K > 0 && (tiles_of(j) * kMostParts >= 76 || chunks_of(j) <= 512);
}

cudaError_t init_skinny_kernels() {
    cudaError_t e = cudaSuccess;
#define EMTK_SKINNY_ATTR(F16, GATED, NT)                                                                       \
    if (e == cudaSuccess)                                                                                      \
        e = cudaFuncSetAttribute(skinny_kernel<F16, GATED, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,   \
                                 Shape<NT>::kSmem);
#define EMTK_SKINNY_ATTRS(NT)         \
    EMTK_SKINNY_ATTR(false, false, NT) \
    EMTK_SKINNY_ATTR(false, true, NT)  \
    EMTK_SKINNY_ATTR(true, false, NT)  \
    EMTK_SKINNY_ATTR(true, true, NT)
    EMTK_SKINNY_ATTRS(16)
    EMTK_SKINNY_ATTRS(32)
    EMTK_SKINNY_ATTRS(64)
#undef EMTK_SKINNY_ATTRS
#undef EMTK_SKINNY_ATTR
    return e;
}

cudaError_t launch_skinny(const MmJob &j, const emtk_nn *nn, cudaStream_t s) {
    const bool gated = j.kind == kMmGated;
    const int nt = j.M <= 16 ? 16 : j.M <= 32 ? 32 : 64, tiles = tiles_of(j);
    SkinnyParams p;
    for (int i = 0; i < (gated ? 2 : 1); ++i)
        if (!encode_operand(nn, &p.w[i], j.b[i], j.N, j.K, gated ? 64 : 128)) return cudaErrorInvalidValue;
    if (!encode_operand(nn, &p.x, j.a[0], j.M, j.K, nt)) return cudaErrorInvalidValue;
    p.epi = j.epi;
    p.M = j.M;
    p.N = j.N;
    p.K = j.K;
    p.chunks = chunks_of(j);
    // two CTAs an SM, each with at least 4 chunks
    p.parts = std::max(1, std::min({kMostParts, 2 * nn->sm_count / tiles, p.chunks / 4}));
    p.chunks_per_part = (p.chunks + p.parts - 1) / p.parts;
    p.parts = (p.chunks + p.chunks_per_part - 1) / p.chunks_per_part;
    p.status = nn->status;
    p.timeout_ns = nn->timeout_ns;
    p.debug_stall = nn->debug_stall;
    const unsigned ctas = (unsigned)tiles * (unsigned)p.parts;
    if (j.type == EMTK_TYPE_F16) return gated ? run<true, true>(p, nt, ctas, s) : run<true, false>(p, nt, ctas, s);
    return gated ? run<false, true>(p, nt, ctas, s) : run<false, false>(p, nt, ctas, s);
}

}  // namespace emtk
