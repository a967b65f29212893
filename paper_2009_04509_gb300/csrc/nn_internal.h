// Declarations shared by the dense / gated / checkpoint layers' files
// (nn_api.cu, nn_mm.cu, nn_pointwise.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/emtk.h"

#ifdef __CUDACC__
#define EMTK_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define EMTK_HOST_DEVICE inline
#endif

namespace emtk {
struct SlopeRange;
}

struct emtk_nn {
    int device = 0;
    int sm_count = 0;
    int64_t timeout_ns = 0;
    int debug_stall = 0;
    int *status = nullptr;   // device status word, as a context's
    emtk::SlopeRange *range = nullptr;  // beside it: of the running backward call's slopes
    float2 *far_sums = nullptr;         // and [sm_count * kCutRows]: rows' sums that a gradient of logits takes again
    void *ws = nullptr;      // workspace of the running call
    size_t ws_bytes = 0;
    bool captured = false;   // a graph holds the workspace's address
    struct Outgrown {        // workspaces that graphs hold, kept until the handle goes
        void *ws;
        Outgrown *next;
    } *outgrown = nullptr;
    void *encode = nullptr;  // cuTensorMapEncodeTiled
};

namespace emtk {

constexpr int kCutRows = 4;   // for each SM, of a gradient of logits whose rows go to several blocks
constexpr int kQ8Block = 32;  // columns that share a checkpoint scale
constexpr int kMaxNormWidth = 16384;  // of residual norms: a row is held in a block's registers

// Size of a workspace that has to hold `need` bytes: a quarter more, so that slowly
// growing calls seldom wait, unless the device has little left beside it.
inline size_t workspace_size(size_t need, size_t device_free) {
    const size_t ample = need + need / 4;
    return ample <= device_free - device_free / 16 ? ample : need;
}

// Operand of a matrix product: element (i, t) of the contraction t is
// p[i * ld + t], or p[t * ld + i] if `across` (i runs along memory).
struct MmOperand {
    const void *p;
    int64_t ld;
    bool across;
};

// Slopes dz (dg and du) in fp16: their largest finite magnitudes (zero between calls:
// the products, which come last, reset them), and the inverse of the power of two by
// which they are stored (nn_math.cuh), which the products' sums take.  Kernels in a row
// write and read the one line that this is in, so they read it from L2.
struct SlopeRange {
    uint32_t peak[2];
    float unscale;
};

// What becomes of the sums.
//   plain: z = sum + bias[0]; out = act(z) + residual; saved[0] = z
//   gated: g = sum0 + bias[0], u = sum1 + bias[1]; out = act(g) u;
//          saved[0] = g, saved[1] = u
// Absent parts have null pointers.  out is fp32 if out_f32.  range (of a gradient: no other
// parts): the sums are of scaled slopes.
struct MmEpilogue {
    int act;
    int bias_f32;
    int out_f32;
    const void *bias[2];
    emtk_matrix residual, out, saved[2];
    const SlopeRange *range;
};

// out[M][N] from the contraction over K of a[i] and b[i] (rows M and N):
//   kMmSum:   a[0] b[0]^T (+ a[1] b[1]^T if terms == 2)
//   kMmGated: sum0 = a[0] b[0]^T and sum1 = a[0] b[1]^T, gated epilogue
// Both operands' types are `type`; sums are fp32.
enum MmKind { kMmSum = 0, kMmGated = 1 };
struct MmJob {
    MmKind kind;
    emtk_type type;
    int M, N, K;
    int terms;
    MmOperand a[2], b[2];
    MmEpilogue epi;
};
// Whether a matrix of 16-bit elements can be an operand as it lies: TMA wants
// its address and row distance on 16 bytes.  (Others are copied first.)
bool mm_operand_ok(const void *p, int64_t ld, int64_t rows);
// Tensor map of an operand: rows of index i (M or N), K contraction steps, boxes
// of 128 bytes along memory by box_rows (or 64, where i runs along memory).
bool encode_operand(const emtk_nn *nn, CUtensorMap *map, const MmOperand &o, int rows, int K, int box_rows);
// Tensor map of a matrix of 16-bit elements: boxes of box_cols (64 bytes to 256 columns) by
// box_rows as they lie, unswizzled.
bool encode_rows(const emtk_nn *nn, CUtensorMap *map, const emtk_matrix &m, int rows, int cols, int box_cols, int box_rows);
constexpr int kMmTileRows = 256, kMmStep = 64;  // rows of a tile, contraction steps of a chunk

// Division by a fixed d > 0 of 0 <= n < 2^31, as a product: floor(n m / 2^(31 + s)) with
// 2^(s - 1) < d <= 2^s and m = ceil(2^(31 + s) / d) < 2^32 is exact there.  The integer
// unit's own division would keep each tile's first MMA waiting.
struct Divisor {
    uint32_t mul, shift;
    Divisor() = default;
    explicit Divisor(uint32_t d) {
        uint32_t s = 0;
        while ((1u << s) < d) ++s;
        mul = (uint32_t)(((1ull << (31 + s)) + d - 1) / d);
        shift = 31 + s;
    }
    EMTK_HOST_DEVICE int of(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
};

// Up to kMaxJobs jobs of one kind and type in one launch (nn_mm.cu); the plan
// says how they are cut, and how much workspace `partial` it needs.  A piece is a
// run of a job's tiles whose contraction is cut into equally many parts, dealt in
// turn to pair_count of the launch's CTA pairs from pair_lo on.
constexpr int kMaxJobs = 3, kMaxPieces = 8;
struct MmPlan {
    int tn, pairs, units, pieces;
    struct Job {
        int tiles_m, tiles_n, chunks, total;
    } job[kMaxJobs];
    struct Piece {
        int job, tile0, tiles, parts, chunks_per_part, units, pair_lo, pair_count;
        int64_t part_at;
    } piece[kMaxPieces];
    size_t workspace;
};
MmPlan plan_mm(const MmJob *jobs, int n, int sms);
cudaError_t launch_mm(const MmJob *jobs, int n, const MmPlan &plan, const emtk_nn *nn, void *partial, cudaStream_t s);
cudaError_t init_mm_kernels();  // once per device
// The forward pass of 1 to 4 rows (nn_rows.cu), operands anywhere.
bool few_rows(const MmJob &job);
cudaError_t launch_rows(const MmJob &job, int sms, cudaStream_t s);
// The forward pass of up to 128 rows (nn_skinny.cu).
bool skinny(const MmJob &job, int sms);
cudaError_t launch_skinny(const MmJob &job, const emtk_nn *nn, cudaStream_t s);
cudaError_t init_skinny_kernels();  // once per device

// ---- pointwise passes (nn_pointwise.cu)
// dz = dy act'(pre) as a 16-bit matrix dz (or none), and its column sums db
// (or null).  partial: fp32 [slope_slices(m, n, sms)][n] scratch when db is wanted.
// range (fp16, or null): dz is stored by a power of two that keeps it in fp16's range.
int slope_slices(int m, int n, int sms);
cudaError_t launch_slope(emtk_type type, int act, int m, int n, const emtk_matrix &dy, const emtk_matrix &pre,
                         void *dz, int64_t dz_ld, float *db, float *partial, SlopeRange *range, int sms, cudaStream_t s);
// dg, du, h and the column sums of the gated block; partial: twice as large.
cudaError_t launch_gated_slope(emtk_type type, int act, int m, int f, const emtk_matrix &dh, const emtk_matrix &gate,
                               const emtk_matrix &up, void *dg, void *du, int64_t d_ld, const emtk_matrix &h,
                               float *db_gate, float *db_up, float *partial, SlopeRange *range, int sms, cudaStream_t s);
cudaError_t launch_pack8(emtk_type type, int m, int k, const emtk_matrix &x, const emtk_matrix &q, int sms,
                         cudaStream_t s);
// to = the values of from (a checkpoint, or a 16-bit matrix as it is), for up
// to kMaxCopies matrices in one launch.  A 16-bit matrix goes to rows on 16 bytes alone
// (else cudaErrorInvalidValue); dropout of nothing copies one to any rows.
constexpr int kMaxCopies = 4;
struct Copy16 {
    emtk_matrix from, to;
    int rows, cols;
};
cudaError_t launch_copy16(emtk_type type, const Copy16 *copies, int n, int sms, cudaStream_t s);

// ---- around the products: argument structs as they came, checked
cudaError_t launch_dropout(emtk_type type, int m, int n, const emtk_matrix &x, const emtk_matrix &y, const emtk_drop &drop,
                           int sms, cudaStream_t s);  // nn_dropout.cu
cudaError_t init_norm_kernels();  // once per device
cudaError_t launch_residual_norm(const emtk_residual_norm_args &p, const emtk_nn *nn, cudaStream_t s);  // nn_norm.cu
size_t residual_norm_workspace(const emtk_residual_norm_grad_args &p, int sms);
cudaError_t launch_residual_norm_grad(const emtk_residual_norm_grad_args &p, void *workspace, const emtk_nn *nn, cudaStream_t s);
cudaError_t launch_logprobs(const emtk_logprobs_args &p, int sms, cudaStream_t s);  // nn_logprob.cu
cudaError_t launch_logprobs_grad(const emtk_logprobs_grad_args &p, const emtk_nn *nn, cudaStream_t s);
cudaError_t init_recur_kernels();  // once per device
// Whether a recurrence reads its input m from a copy.
bool recurrence_copies(const emtk_matrix &m, int rows, int n, int seqs, bool uniform, int sms);
size_t recurrence_workspace(int rows, int n, int seqs, bool uniform, bool tma, int sms);  // uniform: without offsets
cudaError_t launch_recurrence(const emtk_recurrence_args &p, void *workspace, const emtk_nn *nn, cudaStream_t s);  // nn_recur.cu
cudaError_t launch_recurrence_grad(const emtk_recurrence_grad_args &p, void *workspace, const emtk_nn *nn, cudaStream_t s);

}  // namespace emtk
