// The layers' matrix products on the tcgen05 tensor cores.
//
// out[M][N] = sum over the contraction of a and b, in tiles of 256 rows by TN
// columns, each computed by a pair of CTAs (cta_group::2): every CTA stages 128
// rows of a and half of the columns' b through shared memory by TMA, one thread
// of the leader issues the MMAs for both, and each CTA's TMEM holds the sums of
// its own 128 rows in fp32.  Roles of a CTA's 12 warps: TMA producer, MMA issuer
// (leader), TMEM owner, and 8 epilogue warps that turn one accumulator into
// output while the next tile is summed in the other.
//
// An operand may lie along the contraction (x, w of the forward pass) or across
// it (w of dx, both operands of dw): the same 128-byte-swizzled boxes, K-major
// or MN-major descriptors, so no operand is ever transposed in memory.
//
// The gated block's tile holds TN/2 columns of each projection: the pair's first
// CTA stages w_gate's rows, the second w_up's, so one MMA makes g and u of the
// same columns side by side in TMEM and the epilogue multiplies them there.
//
// Outputs of few tiles and a long contraction are split along it (nn_plan.cu): each
// part leaves fp32 sums in the workspace and a second kernel adds them in order and
// applies the epilogue, so results do not depend on timing.  A backward call's two or
// three products are one launch.
//
// What bounds it.  A chunk of 64 steps of a 256-wide tile is 512 cycles of the
// tensor pipe and takes 519 (bf16, measured in the loop); its 32 KB a CTA from L2
// come just as fast, so a 128-wide tile's chunk, 24 KB, is bound by L2 (420 cycles
// against 256 of the pipe).  16384 x 4096 -> 4096 with residual, bf16: 293 us, 1.88
// PFLOP/s, tensor pipe 88% active (342 in a row, at the power limit).  8192 x 4096 -> 2 x 10240 gated: 693 us, 1.98
// PFLOP/s.  20000 x 512 -> 2304 (dx) with 512 x 20000 x 2304 (dw): 60 us, 1.57
// PFLOP/s; there the epilogue's 92 MB of stores take about as long as the MMAs.
// A few tiles: 4 us for one, then about 0.2 us a chunk.
//
// All waits on barriers are bounded and end in an error status; TMEM allocation and
// the cluster barriers at the start and the end are the hardware's own, which every
// thread of the pair reaches.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_math.cuh"
#include "nn_ptx.cuh"

namespace emtk {
namespace {

constexpr int kTileM = kMmTileRows;       // rows of a pair's tile
constexpr int kStep = kMmStep;           // contraction steps of a stage: 128 bytes
constexpr int kABytes = 128 * kStep * 2;  // a CTA's rows of a stage
constexpr int kEpiWarps = 8;
constexpr int kFirstEpiWarp = 4;
constexpr int kThreads = 32 * (kFirstEpiWarp + kEpiWarps);

// Which epilogue a kernel has: gradients' (nothing but the sums), a dense layer's, a
// gated block's, and those that keep z or g and u as well.  Each is a variant of its
// own: unrolled over a block's columns, the others' code, jumped over, costs as much as
// the stores, in instruction fetches or spilled registers (bf16, 20000 x 512 -> 2304
// with the dense layer's code as well: 60 us, 41 when split off; 8192 x 64 -> 4096
// with a residual, with the kept z's: 42, 37 when split off).  An epilogue warp turns blocks of 32
// rows by kBlock columns into output through kStageRow-byte rows of shared memory; the
// gradients' blocks are twice as wide, which halves the latencies that their stores
// wait out.
enum Kind : int { kPlain, kDense, kGated, kDenseKept, kGatedKept };
constexpr bool is_gated(Kind k) { return k == kGated || k == kGatedKept; }
constexpr bool keeps(Kind k) { return k == kDenseKept || k == kGatedKept; }
template <Kind KIND>
struct Epi {
    static constexpr int kBlock = KIND == kPlain ? 64 : 32;
    static constexpr int kStageRow = KIND == kPlain ? 128 : 64;
    static constexpr int kBiasBytes = KIND == kPlain ? 0 : 128 * 4;  // of the warp's columns
    static constexpr int kWarpBytes = 32 * kStageRow + kBiasBytes;
};

template <int TN, Kind KIND>
struct Shape {
    static constexpr int kBBytes = TN / 2 * kStep * 2;
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = TN == 256 ? 6 : 8;
    static constexpr int kTmemCols = 2 * TN;
    // the stages on 1024 bytes, the epilogue's rows, the barriers
    static constexpr int kSmem = 1024 + kStages * kStageBytes + kEpiWarps * Epi<KIND>::kWarpBytes + 512;
};
static_assert(Shape<256, kPlain>::kSmem <= 227 * 1024 && Shape<128, kPlain>::kSmem <= 227 * 1024 &&
              Shape<256, kGated>::kSmem <= 227 * 1024 && Shape<128, kGated>::kSmem <= 227 * 1024, "shared memory of an SM");

// Where a job's tiles lie: in groups of 8 tile rows, along the rows first, so that
// the pairs at work share operand panels in L2.
struct Raster {
    int tiles_m, tiles_n;
    Divisor by_group, by_last;  // tiles of 8 tile rows; tile rows of the last group
    __device__ __forceinline__ void tile(int t, int cols, int &m0, int &n0) const {
        const int group = by_group.of(t);
        const int in = t - group * 8 * tiles_n;
        const int rows = min(8, tiles_m - 8 * group);
        const int column = rows == 8 ? in >> 3 : by_last.of(in);
        m0 = (8 * group + in - column * rows) * kTileM;
        n0 = column * cols;
    }
};

struct MmWork {  // one piece of the plan
    CUtensorMap a[2], b[2];
    MmEpilogue epi;
    float *partial;  // not null: [tile of the piece][part][256][TN] fp32 sums
    int M, N;
    int a_across, b_across;
    Raster raster;
    int tile0, tiles, parts;
    int chunks, total;     // of one term, of all
    int chunks_per_part;
    int units, pair_lo, pair_count;  // unit u is pair pair_lo + u % pair_count's
    Divisor by_parts;
};
struct MmParams {
    MmWork piece[kMaxPieces];
    int pieces;
    int *status;
    SlopeRange *range;  // to be reset, or null
    int64_t timeout_ns;
    int debug_stall;
};

struct Unit {
    int piece, tile, m0, n0, part, c0, c1;  // tile: of the piece
};

// A pair's way through its units: the pieces in order.
struct Cursor {
    int piece = -1, u = 0;
    __device__ __forceinline__ bool advance(const MmParams &p, int pair) {
        if (piece >= 0) {
            u += p.piece[piece].pair_count;
            if (u < p.piece[piece].units) return true;
        }
        while (++piece < p.pieces) {
            const MmWork &w = p.piece[piece];
            u = pair - w.pair_lo;
            if (u >= 0 && u < w.pair_count && u < w.units) return true;
        }
        return false;
    }
};

// The cursor's unit: a tile's parts are adjacent.
__device__ __forceinline__ Unit unit_of(const MmParams &p, const Cursor &at, int cols) {
    Unit r;
    r.piece = at.piece;
    const int u = at.u;
    const MmWork &w = p.piece[r.piece];
    r.tile = w.by_parts.of(u);
    r.part = u - r.tile * w.parts;
    w.raster.tile(w.tile0 + r.tile, cols, r.m0, r.n0);
    r.c0 = r.part * w.chunks_per_part;
    r.c1 = min(r.c0 + w.chunks_per_part, w.total);
    return r;
}

// The rows' alignment: 0 on 16 bytes, a multiple of 4 on words.
__device__ __forceinline__ uint32_t row_bits(const void *p, int64_t ld, int elem) {
    return (uint32_t)(reinterpret_cast<uintptr_t>(p) | (uint64_t)(ld * elem)) & 15u;
}

// 16-byte piece c of staged row r: the pieces are permuted so that neither a lane to
// a row nor the lanes of a row meet in a bank.
template <int ROW>
__device__ __forceinline__ uint32_t staged(int r, int c) {
    return (uint32_t)(r * ROW + (ROW == 128 ? (c ^ r) & 7 : (c ^ (r >> 1)) & 3) * 16);
}

// nr staged rows of nc elements to `to`, neighbours in memory by neighbouring lanes.
template <typename T, int ROW>
__device__ __forceinline__ void store_elements(T *to, int64_t ld, int nr, int nc, const uint8_t *stage, int lane) {
    constexpr int kCols = ROW / (int)sizeof(T), kAcross = kCols < 32 ? kCols : 32, kDown = 32 / kAcross;
    const int first = lane / kAcross;
#pragma unroll
    for (int c = lane % kAcross; c < kCols; c += kAcross) {
        if (c >= nc) continue;
        const int at = c * (int)sizeof(T) / 16, in = c * (int)sizeof(T) % 16;
        T *g = to + first * ld + c;
        for (int r = first; r < nr; r += 4 * kDown, g += 4 * kDown * ld) {
            T x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (r + i * kDown < nr) x[i] = *reinterpret_cast<const T *>(stage + staged<ROW>(r + i * kDown, at) + in);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (r + i * kDown < nr) g[i * kDown * ld] = x[i];
        }
    }
}

// Stores rows r0 .. r0 + 31 (below `rows`), columns c0 .. c0 + ROW / sizeof(T) - 1 (below
// `cols`) of a matrix from the warp's staged rows: 16-byte pieces, ROW / 16 lanes to a
// row, where they fit; else words or elements (8192 x 64 -> n, bf16: 15 us at n = 4096,
// 21 at 4090, 30 at 4095).  low: row_bits of the matrix.
template <typename T, int ROW>
__device__ __forceinline__ void store_block(T *base, int64_t ld, int64_t r0, int64_t rows, int64_t c0, int64_t cols,
                                            uint32_t low, const uint8_t *stage, int lane) {
    constexpr int kPiece = 16 / sizeof(T), kCols = ROW / sizeof(T), kLanes = ROW / 16, kRows = 32 / kLanes;
    const int nr = (int)min((int64_t)32, rows - r0), nc = (int)min((int64_t)kCols, cols - c0);
    T *const to = base + r0 * ld + c0;
    if (low == 0 && nc == kCols) {
        const int r_first = lane / kLanes, piece = lane % kLanes;
        T *g = to + r_first * ld + piece * kPiece;
#pragma unroll
        for (int it = 0; it < kLanes; ++it, g += kRows * ld) {
            if (r_first + it * kRows >= nr) continue;
            *reinterpret_cast<uint4 *>(g) = *reinterpret_cast<const uint4 *>(stage + staged<ROW>(r_first + it * kRows, piece));
        }
    } else if (sizeof(T) == 2 && (low & 3u) == 0 && nc % 2 == 0) {
        store_elements<uint32_t, ROW>(reinterpret_cast<uint32_t *>(to), ld / 2, nr, nc / 2, stage, lane);
    } else {
        store_elements<T, ROW>(to, ld, nr, nc, stage, lane);
    }
}

// What the epilogue of one warp needs of its tile, in registers: its 32 rows, its
// staged rows, and of the job what every block of 32 columns uses.
struct Rows {
    int64_t r0, rows;  // first row, rows of the matrix
    uint8_t *stage;
    int lane;
    int act;
    bool has_bias, out_f32;
    float unscale;  // of fp16 slopes' sums, else 1
    uint32_t out_low, residual_low;  // row_bits
    void *out, *residual;
    int64_t out_ld, residual_ld;
    __device__ __forceinline__ void take(const MmEpilogue &e) {
        act = e.act;
        has_bias = e.bias[0] != nullptr;
        out_f32 = e.out_f32 != 0;
        unscale = e.range ? __ldcg(&e.range->unscale) : 1.f;
        out = e.out.d;
        out_ld = e.out.ld;
        out_low = row_bits(out, out_ld, out_f32 ? 4 : 2);
        residual = e.residual.d;
        residual_ld = e.residual.ld;
        residual_low = row_bits(residual, residual_ld, 2);
    }
};

// A lane's N columns (of its row) in 16 bits.
template <bool F16, int N>
__device__ __forceinline__ void store16(void *base, int64_t ld, uint32_t low, const Rows &w, int64_t c0, int64_t cols,
                                        const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i)
        *reinterpret_cast<uint4 *>(w.stage + staged<2 * N>(w.lane, i)) =
            make_uint4(pack16<F16>(v[8 * i], v[8 * i + 1]), pack16<F16>(v[8 * i + 2], v[8 * i + 3]),
                       pack16<F16>(v[8 * i + 4], v[8 * i + 5]), pack16<F16>(v[8 * i + 6], v[8 * i + 7]));
    __syncwarp();
    store_block<uint16_t, 2 * N>(static_cast<uint16_t *>(base), ld, w.r0, w.rows, c0, cols, low, w.stage, w.lane);
    __syncwarp();
}

// A lane's N columns as they are, N / 2 at a time.
template <int N>
__device__ __forceinline__ void store32(float *base, int64_t ld, uint32_t low, const Rows &w, int64_t c0, int64_t cols,
                                        const float (&v)[N]) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const int j = N / 2 * half + 4 * i;
            *reinterpret_cast<float4 *>(w.stage + staged<2 * N>(w.lane, i)) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        }
        __syncwarp();
        if (c0 + N / 2 * half < cols)
            store_block<float, 2 * N>(base, ld, w.r0, w.rows, c0 + N / 2 * half, cols, low, w.stage, w.lane);
        __syncwarp();
    }
}

// A row's 32 columns as one checkpoint block.  Rows of codes on 16 bytes: a lane writes
// its row's sector.  Others go through the staged rows so that a store of the warp falls
// into few sectors: 8 lanes to a row by words, or all 32 by bytes.  (By bytes from its own
// row's lane, 32 sectors a store, 1981 x 648 -> 2 x 3032 took 138 us where this takes
// 30.)
__device__ __forceinline__ void store_q8(const emtk_matrix &m, const Rows &w, int64_t c0, int64_t cols,
                                         const float (&v)[32]) {
    const int nc = (int)min((int64_t)32, cols - c0);
    float x[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = i < nc ? v[i] : 0.f;
    bool all_finite;
    const uint32_t b = q8_scale(finite_top(x, all_finite));
    const float inverse = q8_inverse(b);
    const int64_t r = w.r0 + w.lane;
    if (r < w.rows) m.d_scale[r * m.ld_scale + c0 / kQ8Block] = (uint8_t)b;
    uint8_t *const base = static_cast<uint8_t *>(m.d) + w.r0 * m.ld + c0;
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = q8_codes4(x + 4 * i, inverse, all_finite);
    const uint32_t low = (uint32_t)(reinterpret_cast<uintptr_t>(m.d) | (uintptr_t)m.ld);
    if (nc == 32 && (low & 15u) == 0) {
        uint4 *p = reinterpret_cast<uint4 *>(base + w.lane * m.ld);
        if (r >= w.rows) return;
        p[0] = make_uint4(q[0], q[1], q[2], q[3]);
        p[1] = make_uint4(q[4], q[5], q[6], q[7]);
        return;
    }
    constexpr int kRow = 36;  // bytes of a staged row: a word off 32, so that lanes meet in no bank
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint32_t *>(w.stage + w.lane * kRow + 4 * i) = q[i];
    __syncwarp();
    const int nr = (int)min((int64_t)32, w.rows - w.r0);
    if (nc % 4 == 0 && (low & 3u) == 0) {
        const int first = w.lane / 8, c = w.lane % 8 * 4;
#pragma unroll
        for (int i = first; i < 32; i += 4)
            if (i < nr && c < nc)
                *reinterpret_cast<uint32_t *>(base + i * m.ld + c) = *reinterpret_cast<const uint32_t *>(w.stage + i * kRow + c);
    } else if (w.lane < nc) {
#pragma unroll 8
        for (int i = 0; i < nr; ++i) base[i * m.ld + w.lane] = w.stage[i * kRow + w.lane];
    }
    __syncwarp();
}

template <bool F16>
__device__ __forceinline__ void store_saved(const emtk_matrix &m, const Rows &w, int64_t c0, int64_t cols,
                                            const float (&v)[32]) {
    if (m.d_scale)
        store_q8(m, w, c0, cols, v);
    else
        store16<F16>(m.d, m.ld, row_bits(m.d, m.ld, 2), w, c0, cols, v);
}

template <bool F16>
__device__ __forceinline__ float bias_at(const MmEpilogue &e, int which, int64_t n, int64_t cols) {
    if (e.bias[which] == nullptr || n >= cols) return 0.f;
    return e.bias_f32 ? __ldg(static_cast<const float *>(e.bias[which]) + n)
                      : from16<F16>(__ldg(static_cast<const uint16_t *>(e.bias[which]) + n));
}

__device__ __forceinline__ void add_bias(const float *bias, float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 b = reinterpret_cast<const float4 *>(bias)[i];
        v[4 * i] += b.x;
        v[4 * i + 1] += b.y;
        v[4 * i + 2] += b.z;
        v[4 * i + 3] += b.w;
    }
}

// Gradients: nothing but the sums.
template <bool F16, int N>
__device__ __forceinline__ void finish_plain(const Rows &w, int64_t c0, int64_t cols, float (&v)[N]) {
    if (F16 && w.unscale != 1.f) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= w.unscale;
    }
    if (w.out_f32)
        store32(static_cast<float *>(w.out), w.out_ld, w.out_low, w, c0, cols, v);
    else
        store16<F16>(w.out, w.out_ld, w.out_low, w, c0, cols, v);
}

// The residual's block on its way into the warp's staged rows: 16-byte pieces
// or words asynchronously, without registers that the wait would hold, else elements.
__device__ __forceinline__ void fetch_residual(const Rows &w, int64_t c0, int64_t cols) {
    const int nr = (int)min((int64_t)32, w.rows - w.r0), nc = (int)min((int64_t)32, cols - c0);
    const uint16_t *const base = static_cast<const uint16_t *>(w.residual) + w.r0 * w.residual_ld + c0;
    if (w.residual_low == 0 && nc == 32) {
        const int first = w.lane / 4, piece = w.lane % 4;
#pragma unroll
        for (int it = 0; it < 4; ++it)
            if (first + 8 * it < nr)
                copy_async_16(smem_u32(w.stage + staged<64>(first + 8 * it, piece)),
                              base + (first + 8 * it) * w.residual_ld + 8 * piece);
    } else if ((w.residual_low & 3u) == 0 && nc % 2 == 0) {
        const int first = w.lane / 16, c = w.lane % 16;
#pragma unroll
        for (int it = 0; it < 16; ++it)
            if (first + 2 * it < nr && 2 * c < nc)
                copy_async_4(smem_u32(w.stage + staged<64>(first + 2 * it, c / 4) + c % 4 * 4),
                             base + (first + 2 * it) * w.residual_ld + 2 * c);
    } else if (w.lane < nc) {
        const uint16_t *g = base + w.lane;
        for (int r = 0; r < nr; r += 8, g += 8 * w.residual_ld) {  // eight rows' elements in flight
            uint16_t x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r + i < nr) x[i] = g[i * w.residual_ld];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r + i < nr) *reinterpret_cast<uint16_t *>(w.stage + staged<64>(r + i, w.lane / 8) + w.lane % 8 * 2) = x[i];
        }
    }
}

// Sums of a dense tile's 32 columns (z without its bias, which is in `bias`).
template <bool F16, bool KEEP>
__device__ __forceinline__ void finish_dense(const MmEpilogue &e, const Rows &w, int64_t c0, int64_t cols,
                                             const float *bias, bool fetched, float (&v)[32]) {
    if (w.has_bias) add_bias(bias, v);
    if constexpr (KEEP) store_saved<F16>(e.saved[0], w, c0, cols, v);
    apply_act(w.act, v);
    if (w.residual) {
        if (!fetched) fetch_residual(w, c0, cols);
        copy_async_wait();
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 q = *reinterpret_cast<const uint4 *>(w.stage + staged<64>(w.lane, i));
            const uint32_t x[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[8 * i + 2 * j] += from16<F16>(x[j] & 0xffffu);
                v[8 * i + 2 * j + 1] += from16<F16>(x[j] >> 16);
            }
        }
        __syncwarp();
    }
    store16<F16>(w.out, w.out_ld, w.out_low, w, c0, cols, v);
}

template <bool F16, bool KEEP>
__device__ __forceinline__ void finish_gated(const MmEpilogue &e, const Rows &w, int64_t c0, int64_t cols,
                                             const float *bias_g, const float *bias_u, float (&g)[32],
                                             float (&u)[32]) {
    if (w.has_bias) {
        add_bias(bias_g, g);
        add_bias(bias_u, u);
    }
    if constexpr (KEEP) {
        store_saved<F16>(e.saved[0], w, c0, cols, g);
        store_saved<F16>(e.saved[1], w, c0, cols, u);
    }
    apply_act(w.act, g);
#pragma unroll
    for (int i = 0; i < 32; ++i) g[i] *= u[i];
    store16<F16>(w.out, w.out_ld, w.out_low, w, c0, cols, g);
}

enum Bar : int { kBarFull = 0, kBarEmpty = 8, kBarAccFull = 16, kBarAccEmpty = 18, kBarDrain = 20, kBarStall = 21, kBars = 22 };

template <bool F16, Kind KIND, int TN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    mm_kernel(const __grid_constant__ MmParams p) {
    using S = Shape<TN, KIND>;
    using E = Epi<KIND>;
    constexpr bool GATED = is_gated(KIND);
    constexpr int kCols = GATED ? TN / 2 : TN;  // output columns of a tile
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    uint8_t *const base = smem_raw + ((1024u - (raw & 1023u)) & 1023u);
    const uint32_t stages = smem_u32(base);
    uint8_t *const tail = base + S::kStages * S::kStageBytes;
    uint64_t *const bars = reinterpret_cast<uint64_t *>(tail + kEpiWarps * E::kWarpBytes);
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(bars + kBars);
    volatile uint32_t *const abort_flag = tmem_slot + 1;
    auto bar = [&](int i) { return smem_u32(bars + i); };

    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const Guard guard{abort_flag, p.status, p.timeout_ns};
    const int pair = (int)blockIdx.x / 2;
    Cursor cursor;

    pdl_trigger();

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(bar(kBarFull + s), 1);
            mbar_init(bar(kBarEmpty + s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(kBarAccFull + i), 1);
            mbar_init(bar(kBarAccEmpty + i), 2 * kEpiWarps);
        }
        mbar_init(bar(kBarDrain), 1);
        mbar_init(bar(kBarStall), 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 2) tmem_alloc_pair(smem_u32(tmem_slot), S::kTmemCols);
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();
    if (KIND == kPlain && F16 && p.range && blockIdx.x == 0 && threadIdx.x < 2) p.range->peak[threadIdx.x] = 0u;

    if (warp == 0) {
        // ---------------------------------------------------- TMA producer
        // The warp runs the loop together and one lane issues (here and in the MMA
        // warp): descriptors and addresses stay in uniform registers.
        bool ok = !(p.debug_stall && !warp_wait(bar(kBarStall), 0u, guard, lane));
        const uint32_t full0 = cluster_addr(bar(kBarFull), 0);
        int s = 0;
        uint32_t phase = 1;  // a fresh barrier's previous phase counts as complete
        while (ok && cursor.advance(p, pair)) {
            const Unit t = unit_of(p, cursor, kCols);
            const int ra = t.m0 + 128 * (int)rank, rb = t.n0 + (GATED ? 0 : TN / 2 * (int)rank);
            const MmWork &w = p.piece[t.piece];
            // Where the pairs share no rows of a, each tile starts at another chunk and wraps
            // around: in step, all would read the same few address bits of b's rows at a time.
            int at = t.c0;
            if (w.raster.tiles_m == 1) at += t.n0 / kCols * 5 % max(1, t.c1 - t.c0);
            for (int c = t.c0; c < t.c1; ++c) {
                if (!warp_wait_all(bar(kBarEmpty + s), phase, guard, lane)) {
                    ok = false;
                    break;
                }
                const int term = at >= w.chunks ? 1 : 0, k0 = (at - term * w.chunks) * kStep;
                if (elect_one()) {
                    const uint32_t sa = stages + s * S::kStageBytes, sb = sa + kABytes;
                    const uint32_t full = full0 + 8 * s;
                    if (rank == 0) mbar_expect_tx_relaxed(bar(kBarFull + s), 2 * S::kStageBytes);
                    const CUtensorMap *ma = &w.a[GATED ? 0 : term];
                    if (w.a_across) {
                        tma_load_2d_pair(sa, ma, full, ra, k0);
                        tma_load_2d_pair(sa + 64 * 128, ma, full, ra + 64, k0);
                    } else {
                        tma_load_2d_pair(sa, ma, full, k0, ra);
                    }
                    const CUtensorMap *mb = &w.b[GATED ? (int)rank : term];
                    if (w.b_across) {
#pragma unroll
                        for (int j = 0; j < TN / 128; ++j) tma_load_2d_pair(sb + j * 64 * 128, mb, full, rb + 64 * j, k0);
                    } else {
                        tma_load_2d_pair(sb, mb, full, k0, rb);
                    }
                }
                __syncwarp();
                if (++at == t.c1) at = t.c0;
                if (++s == S::kStages) {
                    s = 0;
                    phase ^= 1;
                }
            }
        }
        // The last commits' arrivals at this CTA's stages (at unused ones the wait is none).
        for (int i = 0; ok && i < S::kStages; ++i) {
            ok = warp_wait_all(bar(kBarEmpty + s), phase, guard, lane);
            if (++s == S::kStages) {
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
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------ MMA issuer
        bool ok = true;
        int s = 0, tile = 0;
        uint32_t phase = 0;
        for (; ok && cursor.advance(p, pair); ++tile) {
            const Unit t = unit_of(p, cursor, kCols);
            const MmWork &w = p.piece[t.piece];
            const uint32_t idesc = make_idesc_major(kTileM, TN, F16, w.a_across != 0, w.b_across != 0);
            const uint64_t da = w.a_across ? sw128_desc_across(stages, 64 * 128) : sw128_desc(stages);
            const uint64_t db = w.b_across ? sw128_desc_across(stages + kABytes, 64 * 128) : sw128_desc(stages + kABytes);
            // 16 contraction steps: 32 bytes along a K-major row, 16 rows of an MN-major box
            const uint64_t step_a = w.a_across ? 2048 >> 4 : 32 >> 4, step_b = w.b_across ? 2048 >> 4 : 32 >> 4;
            const int ab = tile & 1;
            if (tile >= 2 && !warp_wait_all(bar(kBarAccEmpty + ab), (uint32_t)(tile / 2 - 1) & 1u, guard, lane)) break;
            tc_fence_after();
            const uint32_t acc = tmem + (uint32_t)(ab * TN);
            for (int c = t.c0; c < t.c1; ++c) {
                if (!warp_wait_all(bar(kBarFull + s), phase, guard, lane)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t off = (uint64_t)(s * S::kStageBytes) >> 4;
#pragma unroll
                    for (int i = 0; i < kStep / 16; ++i)
                        mma_pair(acc, da + off + i * step_a, db + off + i * step_b, idesc,
                                 (i > 0 || c > t.c0) ? 1u : 0u);
                    mma_commit_pair(bar(kBarEmpty + s));
                }
                __syncwarp();
                if (++s == S::kStages) {
                    s = 0;
                    phase ^= 1;
                }
            }
            if (ok && elect_one()) mma_commit_pair(bar(kBarAccFull + ab));
            __syncwarp();
        }
        if (elect_one()) mma_commit_pair(bar(kBarDrain));
        __syncwarp();
    } else if (warp >= kFirstEpiWarp) {
        // ---------------------------------------------------- epilogue
        // Warp e reads TMEM lanes 32 (e % 4) .. (the hardware's rule: a warp's index in
        // its group of four) and half of the tile's columns.
        const int e = warp - kFirstEpiWarp;
        const int q = e & 3, half = e >> 2;
        constexpr int kMine = kCols / 2;  // output columns of a warp
        float *const bias = reinterpret_cast<float *>(tail + e * E::kWarpBytes + 32 * E::kStageRow);
        Rows w{};
        w.stage = tail + e * E::kWarpBytes;
        w.lane = lane;
        int tile = 0, taken = -1;
        for (; cursor.advance(p, pair); ++tile) {
            const Unit t = unit_of(p, cursor, kCols);
            const MmWork &job = p.piece[t.piece];
            const int ab = tile & 1;
            if (t.piece != taken) {
                w.take(job.epi);
                w.rows = job.M;
                taken = t.piece;
            }
            w.r0 = t.m0 + 128 * (int64_t)rank + 32 * q;
            const int64_t n0 = t.n0 + half * kMine;
            __syncwarp();
            float *const partial = job.partial;
            const int N = job.N;
            if (KIND != kPlain && partial == nullptr && w.has_bias) {
                for (int j = lane; j < kMine; j += 32) {
                    bias[j] = bias_at<F16>(job.epi, 0, n0 + j, N);
                    if (GATED) bias[kMine + j] = bias_at<F16>(job.epi, 1, n0 + j, N);
                }
            }
            // the residual of a block comes while the one before is finished, the first one's
            // while the tile is summed (a z to be kept needs the staged rows first)
            const bool early = KIND == kDense && partial == nullptr && w.residual && w.r0 < w.rows;
            if (early && n0 < N) {
                fetch_residual(w, n0, N);
                if (w.r0 + lane < w.rows) {  // the other blocks of the lane's row: into L2 meanwhile
                    const uint16_t *g = static_cast<const uint16_t *>(w.residual) + (w.r0 + lane) * w.residual_ld + n0;
#pragma unroll
                    for (int j = E::kBlock; j < kMine; j += 64) prefetch_l2(g + min((int64_t)j, N - 1 - n0));
                    prefetch_l2(g + min((int64_t)kMine, N - n0) - 1);
                }
            }
            if (!warp_wait(bar(kBarAccFull + ab), (uint32_t)(tile / 2) & 1u, guard, lane)) break;
            tc_fence_after();
            const uint32_t acc = tmem + (uint32_t)(ab * TN) + ((uint32_t)(32 * q) << 16);
            const bool rows_in = w.r0 < w.rows;
#pragma unroll 1
            for (int j = 0; j < kMine; j += E::kBlock) {
                const int64_t c0 = n0 + j;
                float v[E::kBlock], x[GATED ? 32 : 1];
                const bool in = rows_in && c0 < N;
                if (in && t.c0 < t.c1) {
                    tmem_ld(acc + (uint32_t)(half * kMine + j), v);
                    if constexpr (GATED) tmem_ld(acc + (uint32_t)(TN / 2 + half * kMine + j), x);
                } else {
#pragma unroll
                    for (int i = 0; i < E::kBlock; ++i) {
                        v[i] = 0.f;
                        if constexpr (GATED) x[i] = 0.f;
                    }
                }
                if (j + E::kBlock == kMine) {  // this warp has read all of its sums
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(cluster_addr(bar(kBarAccEmpty + ab), 0));
                }
                if (!in) continue;
                if (partial != nullptr) {
                    Rows whole = w;  // a tile of the workspace
                    whole.r0 = 128 * (int64_t)rank + 32 * q;
                    whole.rows = kTileM;
                    float *const part = partial + ((int64_t)t.tile * job.parts + t.part) * (kTileM * TN);
                    store32(part, TN, 0u, whole, half * kMine + j, TN, v);
                    if constexpr (GATED) store32(part, TN, 0u, whole, TN / 2 + half * kMine + j, TN, x);
                } else if constexpr (KIND == kPlain) {
                    finish_plain<F16>(w, c0, N, v);
                } else if constexpr (GATED) {
                    finish_gated<F16, keeps(KIND)>(job.epi, w, c0, N, bias + j, bias + kMine + j, v, x);
                } else {
                    finish_dense<F16, keeps(KIND)>(job.epi, w, c0, N, bias + j, early, v);
                    if (early && j + E::kBlock < kMine && c0 + E::kBlock < N) fetch_residual(w, c0 + E::kBlock, N);
                }
            }
        }
        if (KIND == kDense) copy_async_wait();  // a wait that gave up left a residual's copies in flight
    }
    tc_fence_before();
    __syncthreads();
    // Every MMA issued is complete, and both CTAs have seen the arrival that says so:
    // neither may leave, nor release TMEM, while one is on its way to its shared memory.
    // (The accumulators' arrivals are seen by the epilogues, the stages' by the producers.)
    if (warp == 1) {
        const uint64_t t0 = global_timer_ns();
        while (!__all_sync(0xffffffffu, mbar_try_wait(bar(kBarDrain), 0u)) &&
               __any_sync(0xffffffffu, (int64_t)(global_timer_ns() - t0) < p.timeout_ns)) {
        }
        __syncwarp();
    }
    cluster_sync();  // no arrival or MMA of the pair is outstanding
    tc_fence_after();
    if (warp == 2) tmem_free_pair(tmem, S::kTmemCols);
}

// Eight columns of a row, of which the first n exist.
template <bool F16>
__device__ __forceinline__ void store8(uint16_t *p, int n, const float (&v)[8]) {
    if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack16<F16>(v[0], v[1]), pack16<F16>(v[2], v[3]), pack16<F16>(v[4], v[5]),
                                                   pack16<F16>(v[6], v[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = (uint16_t)to16<F16>(v[j]);
    }
}

// Adds the parts' sums and applies the epilogue: 2^lanes_log2 neighbouring
// threads take 8 columns of a row, each every so-manieth part, and join their
// sums in a fixed tree; four such groups hold a checkpoint block (8 threads each
// at most, then: the four share a warp).
template <bool F16, Kind KIND, int TN>
__global__ void __launch_bounds__(256) parts_kernel(const __grid_constant__ MmEpilogue e, const __grid_constant__ Raster raster,
                                                    const float *partial, int tile0, int tiles, int parts, int M, int N,
                                                    int lanes_log2) {
    constexpr bool GATED = KIND == kGated;
    constexpr int kCols = GATED ? TN / 2 : TN, kGroups = kCols / 8;
    const int64_t tid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int lanes = 1 << lanes_log2, mine = threadIdx.x & (lanes - 1);
    const int64_t idx = tid >> lanes_log2;  // a tile's groups are a multiple of four
    const int tile = (int)(idx / (kTileM * kGroups)), row = (int)(idx / kGroups % kTileM), col = (int)(idx % kGroups) * 8;
    int m0 = 0, n0 = 0;
    if (tile < tiles) raster.tile(tile0 + tile, kCols, m0, n0);
    const int64_t r = m0 + row;
    const int c = n0 + col;
    const bool in = tile < tiles && r < M && c < N;
    float v[GATED ? 2 : 1][8] = {};
    pdl_trigger();
    pdl_wait();
    if (in) {
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h) {
            constexpr int kPart = kTileM * TN;
            const float *p = partial + ((int64_t)tile * parts + mine) * kPart + row * TN + col + h * (TN / 2);
#pragma unroll 4
            for (int i = mine; i < parts; i += lanes, p += lanes * kPart) {
                const float4 lo = *reinterpret_cast<const float4 *>(p);
                const float4 hi = *(reinterpret_cast<const float4 *>(p) + 1);
                const float x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int j = 0; j < 8; ++j) v[h][j] += x[j];
            }
        }
    }
    for (int d = lanes >> 1; d > 0; d >>= 1)
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[h][j] += __shfl_xor_sync(0xffffffffu, v[h][j], d);
    if (KIND == kPlain && F16 && e.range) {
        const float unscale = __ldcg(&e.range->unscale);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[0][j] *= unscale;
    }
    const bool writes = in && mine == 0;
#pragma unroll
    for (int h = 0; h < (GATED ? 2 : 1); ++h) {
        if (in) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[h][j] += bias_at<F16>(e, h, c + j, N);
        }
        const emtk_matrix &m = e.saved[h];
        if (m.d == nullptr) continue;
        if (m.d_scale) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = in && c + j < N ? v[h][j] : 0.f;
            bool all_finite;
            float top = finite_top(x, all_finite);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, lanes));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2 * lanes));
            const uint32_t b = q8_scale(top);
            if (!writes) continue;
            if (c % kQ8Block == 0) m.d_scale[r * m.ld_scale + c / kQ8Block] = (uint8_t)b;
            const uint32_t q[2] = {q8_codes4(x, q8_inverse(b), all_finite), q8_codes4(x + 4, q8_inverse(b), all_finite)};
            uint8_t *const codes = static_cast<uint8_t *>(m.d) + r * m.ld + c;
            if (c + 8 <= N && (reinterpret_cast<uintptr_t>(codes) & 7u) == 0) {
                *reinterpret_cast<uint2 *>(codes) = make_uint2(q[0], q[1]);
            } else {
                for (int j = 0; j < 8; ++j)
                    if (c + j < N) codes[j] = (uint8_t)(q[j / 4] >> (8 * (j % 4)));
            }
        } else if (writes) {
            store8<F16>(static_cast<uint16_t *>(m.d) + r * m.ld + c, N - c, v[h]);
        }
    }
    if (!writes) return;
    apply_act(e.act, v[0]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float y = v[0][j];
        if (GATED) y *= v[GATED ? 1 : 0][j];
        if (!GATED && e.residual.d && c + j < N)
            y += from16<F16>(static_cast<const uint16_t *>(e.residual.d)[r * e.residual.ld + c + j]);
        v[0][j] = y;
    }
    if (e.out_f32) {
        float *o = static_cast<float *>(e.out.d) + r * e.out.ld + c;
        for (int j = 0; j < 8; ++j)
            if (c + j < N) o[j] = v[0][j];
    } else {
        store8<F16>(static_cast<uint16_t *>(e.out.d) + r * e.out.ld + c, N - c, v[0]);
    }
}

// ---------------------------------------------------------------- host
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

template <bool F16, Kind KIND, int TN>
cudaError_t run(const MmParams &p, const MmPlan &plan, cudaStream_t s) {
    constexpr Kind kJoin = is_gated(KIND) ? kGated : KIND == kPlain ? kPlain : kDense;  // it keeps what there is to keep
    cudaError_t e = launch_pdl(mm_kernel<F16, KIND, TN>, dim3(2 * plan.pairs), dim3(kThreads), Shape<TN, KIND>::kSmem, s, p);
    for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
        const MmWork &w = p.piece[i];
        if (w.parts == 1) continue;
        const int64_t groups = (int64_t)w.tiles * kTileM * (is_gated(KIND) ? TN / 16 : TN / 8);
        int lanes_log2 = 0;  // while the parts and the idle threads last, and a checkpoint's block fits a warp
        const int most = w.epi.saved[0].d_scale || w.epi.saved[1].d_scale ? 3 : 5;
        while (lanes_log2 < most && (2 << lanes_log2) <= w.parts && (groups << lanes_log2) < 2 * 2048 * plan.pairs)
            ++lanes_log2;
        e = launch_pdl(parts_kernel<F16, kJoin, TN>, dim3((unsigned)(((groups << lanes_log2) + 255) / 256)), dim3(256), 0,
                       s, w.epi, w.raster, static_cast<const float *>(w.partial), w.tile0, w.tiles, w.parts, w.M, w.N,
                       lanes_log2);
    }
    return e;
}

}  // namespace

bool encode_operand(const emtk_nn *nn, CUtensorMap *map, const MmOperand &o, int rows, int K, int box_rows) {
    const int64_t lines = o.across ? K : rows;
    const cuuint64_t dims[2] = {(cuuint64_t)(o.across ? rows : K), (cuuint64_t)lines};
    const cuuint64_t strides[1] = {(cuuint64_t)(lines > 1 ? 2 * o.ld : (2 * (int64_t)dims[0] + 15) / 16 * 16)};
    const cuuint32_t box[2] = {64u, (cuuint32_t)(o.across ? kStep : box_rows)};
    const cuuint32_t one[2] = {1u, 1u};
    return reinterpret_cast<EncodeTiled>(nn->encode)(
               map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void *>(o.p), dims, strides, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool mm_operand_ok(const void *p, int64_t ld, int64_t rows) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || (ld * 2) % 16 == 0);
}

cudaError_t init_mm_kernels() {
    cudaError_t e = cudaSuccess;
#define EMTK_MM_ATTR(F16, KIND, TN)                                                                       \
    if (e == cudaSuccess)                                                                                 \
        e = cudaFuncSetAttribute(mm_kernel<F16, KIND, TN>, cudaFuncAttributeMaxDynamicSharedMemorySize, \
                                 Shape<TN, KIND>::kSmem);
#define EMTK_MM_ATTRS(KIND)        \
    EMTK_MM_ATTR(false, KIND, 256) \
    EMTK_MM_ATTR(true, KIND, 256)  \
    EMTK_MM_ATTR(false, KIND, 128) \
    EMTK_MM_ATTR(true, KIND, 128)
    EMTK_MM_ATTRS(kPlain)
    EMTK_MM_ATTRS(kDense)
    EMTK_MM_ATTRS(kGated)
    EMTK_MM_ATTRS(kDenseKept)
    EMTK_MM_ATTRS(kGatedKept)
#undef EMTK_MM_ATTRS
#undef EMTK_MM_ATTR
    return e == cudaSuccess ? init_skinny_kernels() : e;
}

namespace {
template <bool F16, Kind KIND>
cudaError_t run(const MmParams &p, const MmPlan &plan, cudaStream_t s) {
    return plan.tn == 256 ? run<F16, KIND, 256>(p, plan, s) : run<F16, KIND, 128>(p, plan, s);
}
template <bool F16>
cudaError_t run(const MmParams &p, const MmPlan &plan, Kind kind, cudaStream_t s) {
    switch (kind) {
        case kPlain: return run<F16, kPlain>(p, plan, s);
        case kDense: return run<F16, kDense>(p, plan, s);
        case kGated: return run<F16, kGated>(p, plan, s);
        case kDenseKept: return run<F16, kDenseKept>(p, plan, s);
        default: return run<F16, kGatedKept>(p, plan, s);
    }
}
}  // namespace

cudaError_t launch_mm(const MmJob *jobs, int n, const MmPlan &plan, const emtk_nn *nn, void *partial,
                      cudaStream_t s) {
    const bool gated = jobs[0].kind == kMmGated, f16 = jobs[0].type == EMTK_TYPE_F16;
    MmParams p;
    for (int i = 0; i < plan.pieces; ++i) {
        const MmPlan::Piece &c = plan.piece[i];
        const MmPlan::Job &t = plan.job[c.job];
        const MmJob &j = jobs[c.job];
        MmWork &w = p.piece[i];
        if (j.K > 0) {
            bool ok = true;
            for (int k = 0; k < j.terms; ++k) ok = ok && encode_operand(nn, &w.a[k], j.a[k], j.M, j.K, 128);
            for (int k = 0; k < (gated ? 2 : j.terms); ++k) ok = ok && encode_operand(nn, &w.b[k], j.b[k], j.N, j.K, plan.tn / 2);
            if (!ok) return cudaErrorInvalidValue;
        }
        w.epi = j.epi;
        w.partial = c.parts > 1 ? static_cast<float *>(partial) + c.part_at : nullptr;
        w.M = j.M;
        w.N = j.N;
        w.a_across = j.a[0].across;
        w.b_across = j.b[0].across;
        w.raster = {t.tiles_m, t.tiles_n, Divisor((uint32_t)(8 * t.tiles_n)), Divisor((uint32_t)std::max(1, t.tiles_m % 8))};
        w.tile0 = c.tile0;
        w.tiles = c.tiles;
        w.parts = c.parts;
        w.chunks = t.chunks;
        w.total = t.total;
        w.chunks_per_part = c.chunks_per_part;
        w.units = c.units;
        w.pair_lo = c.pair_lo;
        w.pair_count = c.pair_count;
        w.by_parts = Divisor((uint32_t)c.parts);
    }
    p.pieces = plan.pieces;
    p.status = nn->status;
    p.range = jobs[0].epi.range ? nn->range : nullptr;
    p.timeout_ns = nn->timeout_ns;
    p.debug_stall = nn->debug_stall;
    bool plain = !gated, kept = false;
    for (int i = 0; i < n; ++i) {
        const MmEpilogue &e = jobs[i].epi;
        kept = kept || e.saved[0].d;
        plain = plain && e.act == EMTK_ACT_NONE && !e.bias[0] && !e.residual.d && !kept;
    }
    const Kind kind = plain ? kPlain : gated ? (kept ? kGatedKept : kGated) : (kept ? kDenseKept : kDense);
    return f16 ? run<true>(p, plan, kind, s) : run<false>(p, plan, kind, s);
}

}  // namespace emtk
