// The layers' forward pass for up to 128 rows, on the tcgen05 tensor cores.
//
// The time is that of reading the weights once.  So the weights take the MMA's
// 128 rows (of the gated block 64 rows of each projection) and the rows of x its
// 16 to 128 columns: every byte staged by TMA but x's is a weight, where a
// tile of nn_mm.cu would stage 256 mostly empty rows of x.  Two CTAs of about
// 105 KB share an SM, so that one's set-up and epilogue run beside the other's
// stream.  Where the output tiles are fewer than the CTAs that fit, a cluster of
// up to 8 CTAs splits the contraction: each leaves its fp32 sums in shared
// memory, and every CTA adds the cluster's sums for its share of the rows, in
// rank order, over distributed shared memory; no second kernel, no workspace.
//
// HBM bounds it.  4096 -> 2 x 10240 gated, bf16 (168 MB of weights, none of them in L2):
// 30.4 us for 3 rows, 31.3 for 8, 32.5 for 16, 33.8 for 64, 38.7 for 128 (5.5, 5.4, 5.2,
// 5.0 and 4.3 TB/s); 4096 -> 4096 dense: 9.8 us for 8 rows.  With all CTAs starting at the same chunk 16 rows took 56
// us, and with a thread finishing one column, its cluster's sums one after another, 64
// rows took 38.  What is left to the copy's 6.8 TB/s is the ramp and, from 32 rows on,
// the epilogue and x's tiles.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_math.cuh"
#include "nn_ptx.cuh"

namespace emtk {
namespace {

constexpr int kThreads = 256;
constexpr int kStep = 64;                    // contraction steps of a chunk: 128 bytes
constexpr int kWeightRows = 128;
constexpr int kWBytes = kWeightRows * kStep * 2;
constexpr int kMostParts = 8;                // portable cluster size

template <int NT>  // columns of the MMA: rows of x
struct Shape {
    static constexpr int kChunk = kWBytes + NT * kStep * 2;
    static constexpr int kSlots = NT == 16 ? 6 : NT == 32 ? 5 : NT == 64 ? 4 : 3;
    static constexpr int kTmemCols = NT < 32 ? 32 : NT;
    static constexpr int kSmem = 1024 + kSlots * kChunk + 256;
    static_assert(kSmem <= 113 * 1024, "two CTAs an SM");
    static_assert(NT * kWeightRows * 4 <= kSlots * kChunk, "the sums take the slots' place");
};

struct SkinnyParams {
    CUtensorMap w[2], x;
    MmEpilogue epi;
    int M, N, parts, chunks_per_part, chunks;
    int *status;
    int64_t timeout_ns;
    int debug_stall;
};

__device__ __forceinline__ float4 load_cluster(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
// Up to four neighbouring 16-bit elements, one access where the matrix allows.
__device__ __forceinline__ void store4(void *base, int64_t at, int n, bool wide, uint32_t lo, uint32_t hi) {
    uint16_t *p = static_cast<uint16_t *>(base) + at;
    if (wide && n >= 4) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(lo, hi);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (uint16_t)((i < 2 ? lo : hi) >> (16 * (i % 2)));
    }
}
__device__ __forceinline__ uint2 load4(const void *base, int64_t at, int n, bool wide) {
    const uint16_t *p = static_cast<const uint16_t *>(base) + at;
    if (wide && n >= 4) return *reinterpret_cast<const uint2 *>(p);
    uint32_t x[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) x[i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
    return make_uint2(x[0], x[1]);
}
__device__ __forceinline__ bool wide4(const void *p, int64_t row_bytes, unsigned bytes) {
    return ((reinterpret_cast<uintptr_t>(p) | (uint64_t)row_bytes) & (bytes - 1)) == 0;
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
    if (ok && warp < 4) {
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
    // This CTA's rows of x are rank, rank + parts, ..; a thread keeps four columns, and
    // has the whole cluster's sums of them in flight at once.
    constexpr int kLanes = kOut / 4, kSums = GATED ? 2 : 1;
    const MmEpilogue &e = p.epi;
    const int col = threadIdx.x % kLanes * 4, n = n0 + col, valid = min(4, p.N - n);
    const bool out_wide = wide4(e.out.d, 2 * e.out.ld, 8), res_wide = wide4(e.residual.d, 2 * e.residual.ld, 8);
    float bias[kSums][4] = {};
#pragma unroll
    for (int h = 0; h < kSums; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e.bias[h] && i < valid)
                bias[h][i] = e.bias_f32 ? __ldg(static_cast<const float *>(e.bias[h]) + n + i)
                                        : from16<F16>(__ldg(static_cast<const uint16_t *>(e.bias[h]) + n + i));
    const uint32_t from = smem_u32(sums + col);
    for (int t = rank + p.parts * (threadIdx.x / kLanes); t < p.M; t += p.parts * (kThreads / kLanes)) {
        uint2 res = make_uint2(0u, 0u);
        if (!GATED && e.residual.d) res = load4(e.residual.d, t * e.residual.ld + n, valid, res_wide);
        float z[kSums][4];
#pragma unroll
        for (int h = 0; h < kSums; ++h) {
            float4 part[kMostParts];
#pragma unroll
            for (int r = 0; r < kMostParts; ++r)
                if (r < p.parts) part[r] = load_cluster(cluster_addr(from + 4 * (t * kWeightRows + h * kOut), r));
            z[h][0] = part[0].x, z[h][1] = part[0].y, z[h][2] = part[0].z, z[h][3] = part[0].w;
#pragma unroll
            for (int r = 1; r < kMostParts; ++r)
                if (r < p.parts) z[h][0] += part[r].x, z[h][1] += part[r].y, z[h][2] += part[r].z, z[h][3] += part[r].w;
        }
#pragma unroll
        for (int h = 0; h < kSums; ++h) {
#pragma unroll
            for (int i = 0; i < 4; ++i) z[h][i] = i < valid ? z[h][i] + bias[h][i] : 0.f;
            const emtk_matrix &m = e.saved[h];
            if (m.d == nullptr) continue;
            if (m.d_scale) {  // eight neighbouring threads are a block of 32 columns
                const uint32_t group = 0xffu << (lane & 24);
                bool all_finite;
                float top = finite_top(z[h], all_finite);
#pragma unroll
                for (int d = 1; d < 8; d <<= 1) top = fmaxf(top, __shfl_xor_sync(group, top, d));
                const uint32_t b = q8_scale(top);
                if (valid > 0 && (lane & 7) == 0) m.d_scale[t * m.ld_scale + n / kQ8Block] = (uint8_t)b;
                const uint32_t codes = q8_codes4(z[h], q8_inverse(b), all_finite);
                uint8_t *const to = static_cast<uint8_t *>(m.d) + t * m.ld + n;
                if (valid == 4 && wide4(m.d, m.ld, 4)) {
                    *reinterpret_cast<uint32_t *>(to) = codes;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < valid) to[i] = (uint8_t)(codes >> (8 * i));
                }
            } else {
                store4(m.d, t * m.ld + n, valid, wide4(m.d, 2 * m.ld, 8), pack16<F16>(z[h][0], z[h][1]),
                       pack16<F16>(z[h][2], z[h][3]));
            }
        }
        apply_act(e.act, z[0]);
        const uint32_t x[2] = {res.x, res.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (GATED) z[0][i] *= z[kSums - 1][i];
            if (!GATED && e.residual.d) z[0][i] += from16<F16>((x[i / 2] >> (16 * (i % 2))) & 0xffffu);
        }
        store4(e.out.d, t * e.out.ld + n, valid, out_wide, pack16<F16>(z[0][0], z[0][1]), pack16<F16>(z[0][2], z[0][3]));
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
    if (nt == 64) return run<F16, GATED, 64>(p, ctas, s);
    return run<F16, GATED, 128>(p, ctas, s);
}

int tiles_of(const MmJob &j) {
    const int out = j.kind == kMmGated ? kWeightRows / 2 : kWeightRows;
    return (int)(((int64_t)j.N + out - 1) / out);
}
int chunks_of(const MmJob &j) { return (int)(((int64_t)j.K + kStep - 1) / kStep); }
// Two CTAs an SM, each with at least 4 chunks.
int parts_of(const MmJob &j, int sms) {
    return std::max(1, std::min({kMostParts, 2 * sms / std::max(1, tiles_of(j)), chunks_of(j) / 4}));
}

}  // namespace

// Up to 128 rows, where this is the faster kernel.  A cluster splits the contraction 8
// ways at most, so a few columns with a long contraction are left to nn_mm.cu, which
// splits it over all SMs (16384 -> 128, 8 rows, bf16: 9.1 us here, 7.5 there; -> 1024: 11.0
// and 14.1).  From 25 rows on the epilogue counts against a short contraction (256 ->
// 8192, 48 rows: 6.1 and 5.4; 1024 -> 4096: 6.5 and 7.8) and a second round of CTAs
// shows (1024 -> 40960, 48 rows: 26.0 and 23.0); beyond 64 it takes a longer one still
// (1024 -> 4096, 96 rows: 8.2 and 7.5; 4096 -> 4096: 12.8 and 15.0).
bool skinny(const MmJob &j, int sms) {
    if (j.M > 128 || j.K == 0) return false;
    const int tiles = tiles_of(j), chunks = chunks_of(j), parts = parts_of(j, sms);
    const bool short_way = (chunks + parts - 1) / parts <= 16, one_round = tiles <= 2 * sms;
    const int64_t ctas = (int64_t)tiles * parts;
    if (j.M <= 24) return short_way || 4 * ctas >= sms;
    if (j.M <= 64) return chunks >= 8 && one_round && (short_way || 4 * ctas >= sms);
    return chunks >= 32 && one_round && (short_way || 2 * ctas >= sms);
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
    EMTK_SKINNY_ATTRS(128)
#undef EMTK_SKINNY_ATTRS
#undef EMTK_SKINNY_ATTR
    return e;
}

cudaError_t launch_skinny(const MmJob &j, const emtk_nn *nn, cudaStream_t s) {
    const bool gated = j.kind == kMmGated;
    const int nt = j.M <= 16 ? 16 : j.M <= 32 ? 32 : j.M <= 64 ? 64 : 128, tiles = tiles_of(j);
    SkinnyParams p;
    for (int i = 0; i < (gated ? 2 : 1); ++i)
        if (!encode_operand(nn, &p.w[i], j.b[i], j.N, j.K, gated ? 64 : 128)) return cudaErrorInvalidValue;
    if (!encode_operand(nn, &p.x, j.a[0], j.M, j.K, nt)) return cudaErrorInvalidValue;
    p.epi = j.epi;
    p.M = j.M;
    p.N = j.N;
    p.chunks = chunks_of(j);
    p.parts = parts_of(j, nn->sm_count);
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
