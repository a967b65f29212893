// Pointwise passes of the dense and gated layers' gradients, and the 8-bit
// checkpoints.  All of them stream, every element read once, and HBM bounds
// them.  A thread takes 8 neighbouring columns.  Where every operand's rows start
// on 16 bytes (8 for codes) and hold a multiple of 8 columns, that is one load,
// with the next ones in flight; elsewhere it is the two aligned words around
// them, shifted into place, or single elements at the ends of rows and matrices.
// Measured, bf16: the gated slopes of 8192 x 10240 from 8-bit g and u, 104 us (6.5 TB/s
// of the bytes they need); a dense layer's of 20000 x 512 with column sums, 15 us;
// pack8 of 20000 x 2304, 21 us (6.7 TB/s); unpack8 of the same, 22 us (6.3 TB/s).  At
// odd alignment the gated slopes of 2048 x 5461 take 25 us (4.5 TB/s; 80 registers, three
// blocks an SM), pack8 and unpack8 of 8192 x 4095 44 and 31 us against 14 and 15 of 8192 x
// 4096: there instructions bound them, the shifting of words and the rows' ends.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_math.cuh"

namespace emtk {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;  // columns of a thread

struct Source {  // a 16-bit matrix or a checkpoint
    const uint8_t *p;
    const uint8_t *scale;  // not null: checkpoint
    int64_t row_bytes, ld_scale;
};

Source source_of(const emtk_matrix &m) {
    return {static_cast<const uint8_t *>(m.d), m.d_scale, m.d_scale ? m.ld : 2 * m.ld, m.ld_scale};
}
// Every piece of 8 columns is one aligned load.
bool wide_source(const Source &s, int cols) {
    const unsigned bytes = s.scale ? kVec : 2 * kVec;
    return cols % kVec == 0 && (reinterpret_cast<uintptr_t>(s.p) | (uintptr_t)s.row_bytes) % bytes == 0;
}
bool wide_matrix(const void *p, int64_t row_bytes, unsigned bytes) {
    return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)row_bytes) % bytes == 0;
}

// Eight neighbouring columns as they lie in memory.
template <bool Q8>
struct Piece {
    uint4 w;
    __device__ __forceinline__ void load(const uint8_t *p, const uint8_t *) { w = __ldg(reinterpret_cast<const uint4 *>(p)); }
    template <bool F16>
    __device__ __forceinline__ void values(float *v) const {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = F16 ? from16<F16>(x[i] & 0xffffu) : __uint_as_float(x[i] << 16);
            v[2 * i + 1] = F16 ? from16<F16>(x[i] >> 16) : __uint_as_float(x[i] & 0xffff0000u);
        }
    }
};
template <>
struct Piece<true> {
    uint2 w;
    uint32_t scale;
    __device__ __forceinline__ void load(const uint8_t *p, const uint8_t *s) {
        w = __ldg(reinterpret_cast<const uint2 *>(p));
        scale = __ldg(s);
    }
    template <bool F16>
    __device__ __forceinline__ void values(float *v) const {
        q8_values4(w.x, q8_step(scale), v);
        q8_values4(w.y, q8_step(scale), v + 4);
    }
};

// Columns c .. c + 7 of a row at any alignment; those from n on are 0.  A full piece
// of any row but the first and the last lies in two aligned words of the matrix
// (between its rows, at worst), which are read whole; others go by elements.
template <bool Q8>
struct AnyPiece {
    static constexpr int kBytes = Q8 ? 1 : 2, kWord = kVec * kBytes, kWords = kWord / 4;
    uint32_t x[2 * kWords];
    uint32_t scale;
    int shift;  // bytes to drop
    // p: the first element; valid: columns up to n, at least 1
    __device__ __forceinline__ void load(const uint8_t *p, const uint8_t *s, bool inside, int valid) {
        if (Q8) scale = __ldg(s);
        shift = 0;
        if (inside) {
            shift = (int)(reinterpret_cast<uintptr_t>(p) % kWord);
            fetch(p - shift, x);
            fetch(p - shift + kWord, x + kWords);
        } else {
#pragma unroll
            for (int i = 0; i < 2 * kWords; ++i) x[i] = 0u;
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i < valid)
                    x[i * kBytes / 4] |= (Q8 ? (uint32_t)__ldg(p + i) : (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(p) + i))
                                         << (8 * kBytes * i % 32);
        }
    }
    __device__ __forceinline__ void load(const Source &s, int64_t r, int64_t c, int rows, int n) {
        load(s.p + r * s.row_bytes + kBytes * c, Q8 ? s.scale + r * s.ld_scale + c / kQ8Block : nullptr,
             inside_of(r, c, rows, n), (int)min((int64_t)kVec, n - c));
    }
    static __device__ __forceinline__ bool inside_of(int64_t r, int64_t c, int rows, int n) {
        return r > 0 && r < rows - 1 && c + kVec <= n;
    }
    template <bool F16>
    __device__ __forceinline__ void values(float *v) const {
        if constexpr (Q8) {
            const uint64_t lo = x[0] | (uint64_t)x[1] << 32, hi = x[2] | (uint64_t)x[3] << 32;
            const uint64_t w = shift ? (lo >> (8 * shift)) | (hi << (64 - 8 * shift)) : lo;
            q8_values4((uint32_t)w, q8_step(scale), v);
            q8_values4((uint32_t)(w >> 32), q8_step(scale), v + 4);
        } else {
            uint32_t y[4];
            const int half = 8 * (shift & 3);
            switch (shift >> 2) {  // one case to a row
                case 0: words<0>(y, half); break;
                case 1: words<1>(y, half); break;
                case 2: words<2>(y, half); break;
                default: words<3>(y, half);
            }
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = from16<F16>((y[i / 2] >> (16 * (i % 2))) & 0xffffu);
        }
    }

private:
    template <int FIRST>
    __device__ __forceinline__ void words(uint32_t (&y)[4], int bits) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __funnelshift_r(x[FIRST + i], x[FIRST + i + 1], bits);
    }
    static __device__ __forceinline__ void fetch(const uint8_t *p, uint32_t *to) {
        if constexpr (Q8) {
            const uint2 w = __ldg(reinterpret_cast<const uint2 *>(p));
            to[0] = w.x, to[1] = w.y;
        } else {
            const uint4 w = __ldg(reinterpret_cast<const uint4 *>(p));
            to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
        }
    }
};

template <bool F16>
__device__ __forceinline__ uint4 pack8x16(const float *v) {
    return make_uint4(pack16<F16>(v[0], v[1]), pack16<F16>(v[2], v[3]), pack16<F16>(v[4], v[5]), pack16<F16>(v[6], v[7]));
}

// Columns c .. c + 7 (below n) of a row, in one store where it may be.
template <bool F16>
__device__ __forceinline__ void store_any(uint16_t *row, int64_t c, int n, bool wide, const float *v) {
    if (wide && c + kVec <= n) {
        *reinterpret_cast<uint4 *>(row + c) = pack8x16<F16>(v);
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
// timing.  Up to 512 rows are one slice of 2 lanes' columns, whose sums are the
// result.
struct SlopeShape {
    int lanes_log2;  // threads across
    int col_blocks, slices;
    int rows;  // of a slice
};

// Blocks for every SM: with sums few enough that the slices' partial sums stay
// small against the rows (the any-alignment kernel, three blocks an SM at a time:
// two rounds of them), without them enough to even out the end.
SlopeShape slope_shape(int m, int n, int sms, bool sums, bool wide) {
    SlopeShape h;
    h.lanes_log2 = 5;
    const bool one_slice = sums && m <= 512;
    while (h.lanes_log2 > (one_slice ? 1 : 2) && ((kVec << (h.lanes_log2 - 1)) >= n || one_slice)) --h.lanes_log2;
    const int cols = kVec << h.lanes_log2;
    const int at_once = kThreads >> h.lanes_log2;
    h.col_blocks = (int)(((int64_t)n + cols - 1) / cols);
    int64_t slices = std::max<int64_t>(1, (int64_t)(!wide ? 6 : sums ? 8 : 24) * sms / std::max(1, h.col_blocks));
    slices = std::min<int64_t>(slices, std::max<int64_t>(1, ((int64_t)m + 2 * at_once - 1) / (2 * at_once)));
    slices = std::min<int64_t>(slices, 65535);
    if (one_slice) slices = 1;
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
    float *sums[2];  // of dg and du: [slices][n] each; null: none
    SlopeRange *range;  // fp16: null if dg and du are not stored
    int again;          // the pass that stores what the first could not hold
    int m, n, rows, lanes_log2, h_wide;
};

template <bool GATED, int ACT>
__device__ __forceinline__ void slope_of(float d, float g, float u, float &dg, float &du, float &h) {
    float f = g, s = 1.f;
    act_slope<ACT>(g, f, s);
    dg = GATED ? d * u * s : d * s;
    du = d * f;
    h = f * u;
}

// The block's sums of each column, from its threads': kThreads / cols threads take
// a column, each 8 threads' sums, and the first adds theirs.
template <bool GATED>
__device__ __forceinline__ void block_sums(const SlopeArgs &a, const float (&sg)[kVec], const float (&su)[kVec]) {
    __shared__ float part[kThreads * kVec];
    const int cols = kVec << a.lanes_log2, share = threadIdx.x / cols, in = threadIdx.x % cols;
    const int64_t col = (int64_t)blockIdx.x * cols + in;
#pragma unroll
    for (int half = 0; half < (GATED ? 2 : 1); ++half) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kVec; ++i) part[threadIdx.x * kVec + i] = half ? su[i] : sg[i];
        __syncthreads();
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < kVec; ++g) sum += part[(share * kVec + g) * cols + in];
        __syncthreads();
        part[threadIdx.x] = sum;
        __syncthreads();
        if (share == 0 && col < a.n) {
            for (int g = 1; g < kThreads / cols; ++g) sum += part[g * cols + in];
            a.sums[half][(int64_t)blockIdx.y * a.n + col] = sum;
        }
    }
}

// Slopes in fp16.  The first pass stores them as they are and finds the largest; where
// that left fp16's range, above or below, a second pass of the same kernel stores them
// all by a power of two, else it returns at once (gradients of 20000 x 2304 -> 512: 84 us
// without it, 86 where it returns, 95 where it has work; its launch is 2.5 us of a small
// call).  bf16 has fp32's range, and a dense layer's ReLU leaves dy or 0.
template <bool F16>
struct Ranged {
    float scale = 1.f;
    float peak[2] = {0.f, 0.f};
    // false: there is nothing to do again
    __device__ __forceinline__ bool start(const SlopeArgs &a) {
        if (!F16 || !a.again) return true;
        scale = slope_scale(__ldcg(a.range->peak), __ldcg(a.range->peak + 1));
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.range->unscale = slope_unscale(scale);
        return scale != 1.f;
    }
    // dy or dh, which every slope is a multiple of
    __device__ __forceinline__ void scaled(const SlopeArgs &a, float (&d)[kVec]) const {
        if (!F16 || !a.again) return;
#pragma unroll
        for (int i = 0; i < kVec; ++i) d[i] *= scale;
    }
    __device__ __forceinline__ uint4 stored(const float (&v)[kVec], int which) {
        if (F16) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < kVec; ++i) top = fmaxf(top, fabsf(v[i]));
            if (top == __int_as_float(0x7f800000)) {  // rare
                top = 0.f;
                for (int i = 0; i < kVec; ++i)
                    if (fabsf(v[i]) < __int_as_float(0x7f800000)) top = fmaxf(top, fabsf(v[i]));
            }
            peak[which] = fmaxf(peak[which], top);
        }
        return pack8x16<F16>(v);
    }
    __device__ __forceinline__ void finish(const SlopeArgs &a) {
        if (!F16 || a.range == nullptr || a.again) return;
        __shared__ uint32_t top[2];
        if (threadIdx.x < 2) top[threadIdx.x] = 0u;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(peak[w]));
            if ((threadIdx.x & 31) == 0) atomicMax(top + w, m);
        }
        __syncthreads();
        // the order of maxima changes nothing; most blocks find a larger one there
        if (threadIdx.x < 2 && top[threadIdx.x] > *static_cast<volatile uint32_t *>(a.range->peak + threadIdx.x))
            atomicMax(a.range->peak + threadIdx.x, top[threadIdx.x]);
    }
};

// Q8: gate (and up) are checkpoints.  The next row's loads are issued before
// this row's arithmetic.
template <bool F16, bool GATED, int ACT, bool Q8, bool SUMS>
__global__ void __launch_bounds__(kThreads) slope_kernel(const __grid_constant__ SlopeArgs a) {
    constexpr bool kGate = GATED || ACT != EMTK_ACT_NONE;
    const int at_once = kThreads >> a.lanes_log2;
    const int64_t c = (int64_t)blockIdx.x * (kVec << a.lanes_log2) + (threadIdx.x & ((1 << a.lanes_log2) - 1)) * kVec;
    const int64_t r0 = (int64_t)blockIdx.y * a.rows + (threadIdx.x >> a.lanes_log2);
    const int64_t r1 = min((int64_t)(blockIdx.y + 1) * a.rows, (int64_t)a.m);
    float sg[kVec] = {}, su[kVec] = {};
    Ranged<F16> ranged;
    pdl_trigger();
    pdl_wait();
    if (!ranged.start(a)) return;
    if (c < a.n && r0 < r1) {
        constexpr int kBytes = Q8 ? 1 : 2;
        const uint8_t *pd = a.dy.p + r0 * a.dy.row_bytes + 2 * c;
        const uint8_t *pg = kGate ? a.gate.p + r0 * a.gate.row_bytes + kBytes * c : nullptr;
        const uint8_t *pu = GATED ? a.up.p + r0 * a.up.row_bytes + kBytes * c : nullptr;
        const uint8_t *gs = kGate && Q8 ? a.gate.scale + r0 * a.gate.ld_scale + c / kQ8Block : nullptr;
        const uint8_t *us = GATED && Q8 ? a.up.scale + r0 * a.up.ld_scale + c / kQ8Block : nullptr;
        uint16_t *dg = a.dg + r0 * a.d_ld + c, *du = a.du + r0 * a.d_ld + c, *h = a.h + r0 * a.h_ld + c;
        const bool has_dg = a.dg != nullptr, has_du = GATED && a.du != nullptr, has_h = GATED && a.h != nullptr;
        Piece<false> d;
        Piece<Q8> g, u;
        auto fetch = [&] {
            d.load(pd, nullptr);
            if (kGate) g.load(pg, gs);
            if (GATED) u.load(pu, us);
            pd += at_once * a.dy.row_bytes;
            if (kGate) pg += at_once * a.gate.row_bytes;
            if (GATED) pu += at_once * a.up.row_bytes;
            if (kGate && Q8) gs += at_once * a.gate.ld_scale;
            if (GATED && Q8) us += at_once * a.up.ld_scale;
        };
        fetch();
        for (int64_t r = r0; r < r1; r += at_once) {
            float dv[kVec], gv[kVec], uv[kVec], x[kVec], y[kVec], z[kVec];
            const Piece<false> dn = d;
            const Piece<Q8> gn = g, un = u;
            if (r + at_once < r1) fetch();
            dn.template values<F16>(dv);
            ranged.scaled(a, dv);
            if (kGate) gn.template values<F16>(gv);
            if (GATED) un.template values<F16>(uv);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                slope_of<GATED, ACT>(dv[i], kGate ? gv[i] : 0.f, GATED ? uv[i] : 0.f, x[i], y[i], z[i]);
                if (SUMS) {
                    sg[i] = __fadd_rn(sg[i], x[i]);  // not fused with the product: the sums are of
                    if (GATED) su[i] = __fadd_rn(su[i], y[i]);  // the same values, stored or not
                }
            }
            if (has_dg) *reinterpret_cast<uint4 *>(dg) = ranged.stored(x, 0);
            if (has_du) *reinterpret_cast<uint4 *>(du) = ranged.stored(y, 1);
            if (has_h) *reinterpret_cast<uint4 *>(h) = pack8x16<F16>(z);
            dg += at_once * a.d_ld;
            du += at_once * a.d_ld;
            h += at_once * a.h_ld;
        }
    }
    if constexpr (SUMS) block_sums<GATED>(a, sg, su);
    ranged.finish(a);
}

// Any alignment and width; three blocks an SM (two or four were slower at most of
// 2048 x 5461, 8192 x 2731 and 20000 x 515).
constexpr int kAnyBlocks = 3;
template <bool F16, bool GATED, int ACT, bool Q8>
__global__ void __launch_bounds__(kThreads, kAnyBlocks) slope_any_kernel(const __grid_constant__ SlopeArgs a) {
    constexpr bool kGate = GATED || ACT != EMTK_ACT_NONE;
    const int at_once = kThreads >> a.lanes_log2;
    const int64_t c = (int64_t)blockIdx.x * (kVec << a.lanes_log2) + (threadIdx.x & ((1 << a.lanes_log2) - 1)) * kVec;
    const int64_t r1 = min((int64_t)(blockIdx.y + 1) * a.rows, (int64_t)a.m);
    float sg[kVec] = {}, su[kVec] = {};
    Ranged<F16> ranged;
    pdl_trigger();
    pdl_wait();
    if (!ranged.start(a)) return;
    if (c < a.n) {
        constexpr int kBytes = Q8 ? 1 : 2;
        const int64_t r0 = (int64_t)blockIdx.y * a.rows + (threadIdx.x >> a.lanes_log2);
        const int valid = (int)min((int64_t)kVec, a.n - c);
        const uint8_t *dp = a.dy.p + r0 * a.dy.row_bytes + 2 * c;
        const uint8_t *gp = kGate ? a.gate.p + r0 * a.gate.row_bytes + kBytes * c : nullptr;
        const uint8_t *up = GATED ? a.up.p + r0 * a.up.row_bytes + kBytes * c : nullptr;
        const uint8_t *gs = kGate && Q8 ? a.gate.scale + r0 * a.gate.ld_scale + c / kQ8Block : nullptr;
        const uint8_t *us = GATED && Q8 ? a.up.scale + r0 * a.up.ld_scale + c / kQ8Block : nullptr;
        for (int64_t r = r0; r < r1; r += at_once) {
            float d[kVec], g[kVec] = {}, u[kVec] = {}, x[kVec], y[kVec], z[kVec];
            AnyPiece<false> pd;
            AnyPiece<Q8> pg, pu;
            const bool inside = AnyPiece<false>::inside_of(r, c, a.m, a.n);
            pd.load(dp, nullptr, inside, valid);
            if (kGate) pg.load(gp, gs, inside, valid);
            if (GATED) pu.load(up, us, inside, valid);
            dp += at_once * a.dy.row_bytes;
            if (kGate) gp += at_once * a.gate.row_bytes;
            if (GATED) up += at_once * a.up.row_bytes;
            if (kGate && Q8) gs += at_once * a.gate.ld_scale;
            if (GATED && Q8) us += at_once * a.up.ld_scale;
            pd.template values<F16>(d);
            ranged.scaled(a, d);
            if (kGate) pg.template values<F16>(g);
            if (GATED) pu.template values<F16>(u);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                slope_of<GATED, ACT>(d[i], g[i], u[i], x[i], y[i], z[i]);
                sg[i] = __fadd_rn(sg[i], x[i]);
                if (GATED) su[i] = __fadd_rn(su[i], y[i]);
            }
            // dg and du lie in the workspace, whose rows have room for a last full piece
            if (a.dg) *reinterpret_cast<uint4 *>(a.dg + r * a.d_ld + c) = ranged.stored(x, 0);
            if (GATED && a.du) *reinterpret_cast<uint4 *>(a.du + r * a.d_ld + c) = ranged.stored(y, 1);
            if (GATED && a.h) store_any<F16>(a.h + r * a.h_ld, c, a.n, a.h_wide != 0, z);
        }
    }
    if (a.sums[0]) block_sums<GATED>(a, sg, su);
    ranged.finish(a);
}

// Column sums from the slices' partial sums: a block takes 32 columns, each of
// its 32 warps every 32nd slice, and the warps' sums are added in order.
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(32 * kSumWarps) slice_sum_kernel(const float *s0, const float *s1, int slices, int n,
                                                                   float *db0, float *db1) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    __shared__ float part[kSumWarps][32];
    pdl_trigger();
    pdl_wait();
    float sum = 0.f;
    if (c < n) {
        const float *p = (blockIdx.y ? s1 : s0) + c;
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

typedef void (*SlopeKernel)(const SlopeArgs);

template <bool F16, bool GATED, int ACT>
SlopeKernel slope_for(bool wide, bool q8, bool sums) {
    if (!wide) return q8 ? slope_any_kernel<F16, GATED, ACT, true> : slope_any_kernel<F16, GATED, ACT, false>;
    if (q8) return sums ? slope_kernel<F16, GATED, ACT, true, true> : slope_kernel<F16, GATED, ACT, true, false>;
    return sums ? slope_kernel<F16, GATED, ACT, false, true> : slope_kernel<F16, GATED, ACT, false, false>;
}
template <bool F16, bool GATED>
SlopeKernel slope_for(int act, bool wide, bool q8, bool sums) {
    switch (act) {
        case EMTK_ACT_RELU: return slope_for<F16, GATED, EMTK_ACT_RELU>(wide, q8, sums);
        case EMTK_ACT_GELU: return slope_for<F16, GATED, EMTK_ACT_GELU>(wide, q8, sums);
        case EMTK_ACT_SILU: return slope_for<F16, GATED, EMTK_ACT_SILU>(wide, q8, sums);
        case EMTK_ACT_SIGMOID: return slope_for<F16, GATED, EMTK_ACT_SIGMOID>(wide, q8, sums);
        default: return slope_for<F16, GATED, EMTK_ACT_NONE>(wide, q8, sums);
    }
}

template <bool GATED>
cudaError_t run_slope(emtk_type type, int act, SlopeArgs &a, float *partial, float *db0, float *db1, int sms,
                      cudaStream_t s) {
    if (a.n == 0) return cudaSuccess;
    const bool gate = GATED || act != EMTK_ACT_NONE, sums = db0 != nullptr;
    a.h_wide = a.h && wide_matrix(a.h, 2 * a.h_ld, 16);
    const bool wide = wide_source(a.dy, a.n) && (!gate || wide_source(a.gate, a.n)) &&
                      (!GATED || wide_source(a.up, a.n)) && (!a.h || a.h_wide);
    const SlopeShape h = slope_shape(a.m, a.n, sms, sums, wide);
    a.rows = h.rows;
    a.lanes_log2 = h.lanes_log2;
    a.sums[0] = h.slices == 1 ? db0 : partial;
    a.sums[1] = h.slices == 1 ? db1 : partial + (int64_t)h.slices * a.n;
    if (!sums) a.sums[0] = a.sums[1] = nullptr;
    const bool q8 = gate && a.gate.scale != nullptr;
    const SlopeKernel kernel = type == EMTK_TYPE_F16 ? slope_for<true, GATED>(act, wide, q8, sums)
                                                     : slope_for<false, GATED>(act, wide, q8, sums);
    cudaError_t e = launch_pdl(kernel, dim3((unsigned)h.col_blocks, (unsigned)h.slices), dim3(kThreads), 0, s, a);
    if (e == cudaSuccess && sums && h.slices > 1)
        e = launch_pdl(slice_sum_kernel, dim3((unsigned)((a.n - 1) / 32 + 1), GATED ? 2u : 1u), dim3(32 * kSumWarps), 0,
                       s, static_cast<const float *>(a.sums[0]), static_cast<const float *>(a.sums[1]), h.slices, a.n,
                       db0, db1);
    if (e != cudaSuccess || !a.range) return e;
    const SlopeShape g = slope_shape(a.m, a.n, sms, true, wide);  // few blocks: most often they only look
    a.again = 1;
    a.rows = g.rows;
    a.lanes_log2 = g.lanes_log2;
    a.sums[0] = a.sums[1] = nullptr;
    a.h = nullptr;
    return launch_pdl(slope_for<true, GATED>(act, wide, q8, false), dim3((unsigned)g.col_blocks, (unsigned)g.slices),
                      dim3(kThreads), 0, s, a);
}

// -------------------------------------------------------- checkpoints
// Work is dealt out in pieces of a row, every so-manieth one to a thread (or to a
// group of lanes); the step from one to the next is added to row and piece,
// without a division.
struct Walk {
    int per_row;
    int64_t step_rows;
    int step_pieces;
};

struct Item {
    int64_t r;
    int piece;
    __device__ __forceinline__ Item(const Walk &w, int64_t first) : r(first / w.per_row), piece((int)(first - r * w.per_row)) {}
    __device__ __forceinline__ void next(const Walk &w) {
        r += w.step_rows;
        piece += w.step_pieces;
        if (piece >= w.per_row) {
            piece -= w.per_row;
            ++r;
        }
    }
};

constexpr int kPackCols = 16;  // of a thread: two hold a checkpoint block
constexpr int kBlocks = 5;  // an SM, resident at once

struct PackArgs {
    Source x;
    uint8_t *q, *scale;
    int64_t q_ld, ld_scale;
    int m, k;
    Walk walk;
    int whole;       // of pack8_kernel: codes on 16 bytes, k a multiple of 16
    int lanes_log2;  // of pack8_any_kernel
};

// The largest magnitude is found among the 16-bit patterns, whose order is the
// values' with the sign off, two at a time; one at or above infinity's pattern
// sends the block to the arithmetic of finite_top.
template <bool F16>
__global__ void __launch_bounds__(kThreads, kBlocks) pack8_kernel(const __grid_constant__ PackArgs a) {
    constexpr uint32_t kInfinity = F16 ? 0x7c00u : 0x7f80u;
    constexpr int kFlight = 2;
    Item it(a.walk, (int64_t)blockIdx.x * kThreads + threadIdx.x);
    pdl_trigger();
    pdl_wait();
    while (__any_sync(0xffffffffu, it.r < a.m)) {
        Piece<false> w[kFlight][2];
        int64_t r[kFlight];
        int c[kFlight];
        bool in[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i, it.next(a.walk)) {
            r[i] = it.r;
            c[i] = it.piece * kPackCols;
            in[i] = r[i] < a.m && c[i] < a.k;
            w[i][0].w = w[i][1].w = make_uint4(0u, 0u, 0u, 0u);
            if (in[i]) {
                const uint8_t *p = a.x.p + r[i] * a.x.row_bytes + 2 * (int64_t)c[i];
                w[i][0].load(p, nullptr);
                if (c[i] + kVec < a.k) w[i][1].load(p + 16, nullptr);
            }
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            uint32_t m = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                for (const uint32_t x : {w[i][h].w.x, w[i][h].w.y, w[i][h].w.z, w[i][h].w.w})
                    m = __vmaxu2(m, x & 0x7fff7fffu);
            m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = max(m & 0xffffu, m >> 16);
            float v[kPackCols];
            w[i][0].template values<F16>(v);
            w[i][1].template values<F16>(v + 8);
            float top = from16<F16>(m);
            const bool all_finite = m < kInfinity;  // of both threads
            if (!all_finite) {
                bool mine;
                top = finite_top(v, mine);
                top = fmaxf(top, __shfl_xor_sync(3u << (threadIdx.x & 30), top, 1));
            }
            if (!in[i]) continue;
            const uint32_t b = q8_scale(top);
            const float inverse = q8_inverse(b);
            if (c[i] % kQ8Block == 0) a.scale[r[i] * a.ld_scale + c[i] / kQ8Block] = (uint8_t)b;
            uint8_t *const to = a.q + r[i] * a.q_ld + c[i];
            const uint2 lo = make_uint2(q8_codes4(v, inverse, all_finite), q8_codes4(v + 4, inverse, all_finite));
            const uint2 hi = make_uint2(q8_codes4(v + 8, inverse, all_finite), q8_codes4(v + 12, inverse, all_finite));
            if (a.whole) {
                *reinterpret_cast<uint4 *>(to) = make_uint4(lo.x, lo.y, hi.x, hi.y);
            } else {
                *reinterpret_cast<uint2 *>(to) = lo;
                if (c[i] + kVec < a.k) *reinterpret_cast<uint2 *>(to + kVec) = hi;
            }
        }
    }
}

// Eight bytes a lane, neighbours in a row of n bytes at p, whatever its alignment: each
// lane stores the 8 aligned bytes that start in its own, the row's ends go by bytes.
// Groups of `lanes` lanes hold a row each and call this together.
__device__ __forceinline__ void store_codes(uint8_t *p, int n, const uint32_t (&w)[2], int lanes, int lane) {
    const int head = (int)(-reinterpret_cast<uintptr_t>(p) & 7u);
    const uint64_t own = w[0] | (uint64_t)w[1] << 32;
    const uint64_t next = __shfl_down_sync(0xffffffffu, own, 1, lanes);
    if (8 * lane + head + 8 <= n) {
        const uint64_t x = head ? (own >> (8 * head)) | (next << (64 - 8 * head)) : own;
        *reinterpret_cast<uint2 *>(p + 8 * lane + head) = make_uint2((uint32_t)x, (uint32_t)(x >> 32));
    }
    const int tail = head + max(n - head, 0) / 8 * 8;
    for (int e0 = 0; e0 < 16; e0 += lanes) {  // every lane of the warp goes around as often: they exchange
        const int e = e0 + lane;
        const int c = e < 8 ? e : tail + e - 8;
        const uint64_t x = __shfl_sync(0xffffffffu, own, (c >> 3) & (lanes - 1), lanes);
        if (e < 16 && c < (e < 8 ? min(head, n) : n)) p[c] = (uint8_t)(x >> (8 * (c & 7)));
    }
}

// Any alignment: 2^lanes_log2 lanes (4 .. 32, the fewest that cover narrow rows) take a
// piece of a row.
template <bool F16>
__global__ void __launch_bounds__(kThreads, kBlocks) pack8_any_kernel(const __grid_constant__ PackArgs a) {
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    Item it(a.walk, ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> a.lanes_log2);
    pdl_trigger();
    pdl_wait();
    while (__any_sync(0xffffffffu, it.r < a.m)) {
        constexpr int kFlight = 2;
        AnyPiece<false> piece[kFlight];
        int64_t r[kFlight], first[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i, it.next(a.walk)) {
            r[i] = it.r;
            first[i] = (int64_t)it.piece * (kVec * lanes);
            if (r[i] < a.m && first[i] + lane * kVec < a.k) piece[i].load(a.x, r[i], first[i] + lane * kVec, a.m, a.k);
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int64_t c = first[i] + lane * kVec;
            const bool in = r[i] < a.m && c < a.k;
            float v[kVec] = {};
            if (in) piece[i].template values<F16>(v);
            bool all_finite;
            float top = finite_top(v, all_finite);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t b = q8_scale(top);
            if (in && (lane & 3) == 0) a.scale[r[i] * a.ld_scale + c / kQ8Block] = (uint8_t)b;
            const uint32_t w[2] = {q8_codes4(v, q8_inverse(b), all_finite), q8_codes4(v + 4, q8_inverse(b), all_finite)};
            store_codes(a.q + r[i] * a.q_ld + first[i], r[i] < a.m ? (int)min(a.k - first[i], (int64_t)kVec * lanes) : 0, w,
                        lanes, lane);
        }
    }
}

struct CopyArgs {
    struct One {
        Source from;
        uint16_t *to;
        int64_t to_ld;
        int rows, cols, wide, odd;  // odd: the target's rows are not on 16 bytes
        Walk walk;
    } job[kMaxCopies];
};

// A checkpoint's values, rows of codes on 8 bytes and of values on 16: 8 columns a
// thread, so that neighbours' stores meet in whole sectors (16 columns a thread in
// two stores took 35 us where this takes 22; 20000 x 2304).
template <bool F16>
__device__ __forceinline__ void unpack_wide(const CopyArgs::One &j, Item it) {
    constexpr int kFlight = 4;
    while (it.r < j.rows) {
        Piece<true> w[kFlight];
        int64_t r[kFlight];
        int c[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i, it.next(j.walk)) {
            r[i] = it.r;
            c[i] = it.piece * kVec;
            if (r[i] < j.rows)
                w[i].load(j.from.p + r[i] * j.from.row_bytes + c[i],
                          j.from.scale + r[i] * j.from.ld_scale + c[i] / kQ8Block);
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (r[i] >= j.rows) continue;
            float v[kVec];
            w[i].template values<F16>(v);
#pragma unroll
            for (int t = 0; t < kVec; ++t) v[t] = q8_operand<F16>(v[t]);
            *reinterpret_cast<uint4 *>(j.to + r[i] * j.to_ld + c[i]) = pack8x16<F16>(v);
        }
    }
}

template <bool F16, bool Q8>
__device__ __forceinline__ void copy_any(const CopyArgs::One &j, Item it) {
    while (it.r < j.rows) {
        constexpr int kFlight = 2;
        AnyPiece<Q8> w[kFlight];
        int64_t r[kFlight], c[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i, it.next(j.walk)) {
            r[i] = it.r;
            c[i] = (int64_t)it.piece * kVec;
            if (r[i] < j.rows) w[i].load(j.from, r[i], c[i], j.rows, j.cols);
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (r[i] >= j.rows) continue;
            float v[kVec];
            w[i].template values<F16>(v);
#pragma unroll
            for (int t = 0; t < kVec; ++t) v[t] = Q8 ? q8_operand<F16>(v[t]) : v[t];
            store_any<F16>(j.to + r[i] * j.to_ld, c[i], j.cols, true, v);
        }
    }
}

// A checkpoint's values into rows on any element: a thread takes the 8 columns whose
// values lie on 16 bytes there (8 piece - offset of the row ..), so that its store is one
// and only the rows' ends go by elements.  Two blocks of 32 columns may meet in them.
template <bool F16>
__device__ __forceinline__ void unpack_odd(const CopyArgs::One &j, Item it) {
    for (; it.r < j.rows; it.next(j.walk)) {
        uint16_t *const to = j.to + it.r * j.to_ld;
        const int64_t c = (int64_t)it.piece * kVec - (int64_t)((reinterpret_cast<uintptr_t>(to) >> 1) & 7u);
        const int lo = (int)max((int64_t)0, -c), hi = (int)min((int64_t)kVec, j.cols - c);
        if (lo >= hi) continue;
        const uint8_t *const p = j.from.p + it.r * j.from.row_bytes + c, *const s = j.from.scale + it.r * j.from.ld_scale;
        const bool whole = lo == 0 && hi == kVec;
        const int left = kQ8Block - (int)((c + lo) % kQ8Block) + lo;  // columns before the second block
        const float step0 = q8_step(__ldg(s + (c + lo) / kQ8Block)), step1 = q8_step(__ldg(s + (c + hi - 1) / kQ8Block));
        uint64_t w = 0;
        if (whole && it.r > 0 && it.r < j.rows - 1) {  // two aligned words, both within the matrix
            const int shift = 8 * (int)(reinterpret_cast<uintptr_t>(p) & 7u);
            const uint64_t *const at = reinterpret_cast<const uint64_t *>(p - shift / 8);
            const uint64_t x = __ldg(at), y = shift ? __ldg(at + 1) : 0u;
            w = shift ? (x >> shift) | (y << (64 - shift)) : x;
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i >= lo && i < hi) w |= (uint64_t)__ldg(p + i) << (8 * i);
        }
        float v[kVec];
        q8_values4((uint32_t)w, 1.f, v);
        q8_values4((uint32_t)(w >> 32), 1.f, v + 4);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = q8_operand<F16>(v[i] * (i < left ? step0 : step1));
        if (whole) {
            *reinterpret_cast<uint4 *>(to + c) = pack8x16<F16>(v);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i >= lo && i < hi) to[c + i] = (uint16_t)to16<F16>(v[i]);
        }
    }
}

template <bool F16>
__global__ void __launch_bounds__(kThreads, kBlocks) copy16_kernel(const __grid_constant__ CopyArgs a) {
    const CopyArgs::One &j = a.job[blockIdx.z];
    const Item it(j.walk, (int64_t)blockIdx.x * kThreads + threadIdx.x);
    pdl_trigger();
    pdl_wait();
    if (j.wide) return unpack_wide<F16>(j, it);
    if (j.odd) return unpack_odd<F16>(j, it);
    if (j.from.scale)
        copy_any<F16, true>(j, it);
    else
        copy_any<F16, false>(j, it);
}

// A walk of pieces of `cols` columns over rows of k, by threads or by warps, in
// blocks that are all resident at once.
struct WalkPlan {
    int per_row, workers;  // of a block
    int64_t items;
    unsigned blocks(int sms) const {
        return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + workers - 1) / workers, (int64_t)kBlocks * sms));
    }
    Walk walk(unsigned blocks) const {
        const int64_t all = (int64_t)blocks * workers;
        return {per_row, all / per_row, (int)(all % per_row)};
    }
};
WalkPlan walk_plan(int64_t rows, int64_t k, int cols, int workers, bool even) {
    int64_t per_row = (k + cols - 1) / cols;
    if (even) per_row = (per_row + 1) / 2 * 2;
    return {(int)per_row, workers, rows * per_row};
}

}  // namespace

int slope_slices(int m, int n, int sms) {
    return n > 0 ? std::max(slope_shape(m, n, sms, true, true).slices, slope_shape(m, n, sms, true, false).slices) : 1;
}

cudaError_t launch_slope(emtk_type type, int act, int m, int n, const emtk_matrix &dy, const emtk_matrix &pre,
                         void *dz, int64_t dz_ld, float *db, float *partial, SlopeRange *range, int sms, cudaStream_t s) {
    SlopeArgs a{};
    a.dy = source_of(dy);
    if (act != EMTK_ACT_NONE) a.gate = source_of(pre);
    a.dg = static_cast<uint16_t *>(dz);
    a.d_ld = dz_ld;
    a.range = range;
    a.m = m;
    a.n = n;
    return run_slope<false>(type, act, a, partial, db, nullptr, sms, s);
}

cudaError_t launch_gated_slope(emtk_type type, int act, int m, int f, const emtk_matrix &dh, const emtk_matrix &gate,
                               const emtk_matrix &up, void *dg, void *du, int64_t d_ld, const emtk_matrix &h,
                               float *db_gate, float *db_up, float *partial, SlopeRange *range, int sms, cudaStream_t s) {
    SlopeArgs a{};
    a.dy = source_of(dh);
    a.gate = source_of(gate);
    a.up = source_of(up);
    a.dg = static_cast<uint16_t *>(dg);
    a.du = static_cast<uint16_t *>(du);
    a.d_ld = d_ld;
    a.h = static_cast<uint16_t *>(h.d);
    a.h_ld = h.ld;
    a.range = range;
    a.m = m;
    a.n = f;
    return run_slope<true>(type, act, a, partial, db_gate, db_up, sms, s);
}

cudaError_t launch_pack8(emtk_type type, int m, int k, const emtk_matrix &x, const emtk_matrix &q, int sms,
                         cudaStream_t s) {
    if (m == 0 || k == 0) return cudaSuccess;
    const bool wide = k % kVec == 0 && wide_matrix(x.d, 2 * x.ld, 16) && wide_matrix(q.d, q.ld, 8);
    const bool whole = k % kPackCols == 0 && wide_matrix(q.d, q.ld, 16);
    const bool f16 = type == EMTK_TYPE_F16;
    // wide: an even number of pieces a row, so that a block's two threads are neighbours
    int lanes_log2 = 5;
    while (lanes_log2 > 2 && (kVec << (lanes_log2 - 1)) >= k) --lanes_log2;
    const WalkPlan plan = wide ? walk_plan(m, k, kPackCols, kThreads, true)
                               : walk_plan(m, k, kVec << lanes_log2, kThreads >> lanes_log2, false);
    const unsigned blocks = plan.blocks(sms);
    const PackArgs a{source_of(x), static_cast<uint8_t *>(q.d), q.d_scale, q.ld, q.ld_scale, m, k, plan.walk(blocks), whole, lanes_log2};
    return launch_pdl(wide ? (f16 ? pack8_kernel<true> : pack8_kernel<false>)
                           : (f16 ? pack8_any_kernel<true> : pack8_any_kernel<false>),
                      dim3(blocks), dim3(kThreads), 0, s, a);
}

cudaError_t launch_copy16(emtk_type type, const Copy16 *copies, int n, int sms, cudaStream_t s) {
    CopyArgs a{};
    WalkPlan plans[kMaxCopies];
    unsigned jobs = 0, blocks = 0;
    for (int i = 0; i < n; ++i) {
        const Copy16 &c = copies[i];
        if (c.rows == 0 || c.cols == 0) continue;
        const Source from = source_of(c.from);
        const bool odd = !wide_matrix(c.to.d, 2 * c.to.ld, 16);  // a caller's values: the workspace's rows never are
        if (odd && !from.scale) return cudaErrorInvalidValue;    // unpack_odd reads the scales
        const bool wide = from.scale && !odd && wide_source(from, c.cols);
        plans[jobs] = walk_plan(c.rows, (int64_t)c.cols + (odd ? kVec - 1 : 0), kVec, kThreads, false);
        blocks = std::max(blocks, plans[jobs].blocks(sms));
        a.job[jobs++] = {from, static_cast<uint16_t *>(c.to.d), c.to.ld, c.rows, c.cols, wide, odd, Walk{}};
    }
    if (jobs == 0) return cudaSuccess;
    for (unsigned i = 0; i < jobs; ++i) a.job[i].walk = plans[i].walk(blocks);
    return launch_pdl(type == EMTK_TYPE_F16 ? copy16_kernel<true> : copy16_kernel<false>, dim3(blocks, 1, jobs),
                      dim3(kThreads), 0, s, a);
}

}  // namespace emtk
