// Dropout with a mask that is never stored (nn_pieces.cuh has the generator).
//
// A lane takes pieces of 8 columns, neighbouring lanes neighbouring pieces of a row; HBM
// bounds large ones (4 bytes a value), the call small ones: 16384 x 10240 in bf16 118 us, 5.7 TB/s, with
// the generator's 20 wide products to a piece beside it (the math pipes are what warps wait for most);
// 235 x 333 2.3 us.  A worker's next run is found by adding: with two divisions a run 139 us.
#include <algorithm>

#include "emtk_internal.h"
#include "nn_internal.h"
#include "nn_pieces.cuh"

namespace emtk {
namespace {

constexpr int kThreads = 256;
constexpr int kFlight = 2;  // pieces of a thread whose loads are in flight together (4: 65536 x 333 53 us; 2: 48)

struct DropoutArgs {
    Rows16 x, y;
    Drop drop;
    int m, n, lanes_log2;
    int runs;                        // of a row
    int64_t step_rows;               // from a worker's run to its next, without a division
    int step_runs;
};

template <bool F16, bool ANY>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const __grid_constant__ DropoutArgs a) {
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t first = (int64_t)blockIdx.x * (kThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
    int64_t row = first / a.runs;
    int run = (int)(first - row * a.runs);
    pdl_trigger();
    pdl_wait();
    const uint64_t offset = drop_offset(a.drop);
    while (__any_sync(0xffffffffu, row < a.m)) {
        Piece16<ANY> w[kFlight];
        int r[kFlight], c[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            r[i] = row < a.m ? (int)row : -1;
            c[i] = run * (kPiece << a.lanes_log2);
            w[i].clear();
            if (r[i] >= 0 && c[i] + kPiece * lane < a.n) w[i].load(a.x, r[i], c[i] + kPiece * lane, a.m, a.n);
            row += a.step_rows;
            run += a.step_runs;
            if (run >= a.runs) {
                run -= a.runs;
                ++row;
            }
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            Eight v = w[i].template values<F16>();
            uint32_t q[4];
            dropped(a.drop, offset, (uint32_t)r[i], (uint32_t)(c[i] / kPiece + lane), v);
            words8<F16>(v, q);
            store_run<ANY>(r[i] >= 0 ? a.y.row(r[i]) + c[i] : nullptr, r[i] >= 0 ? min(a.n - c[i], kPiece << a.lanes_log2) : 0, q,
                           lanes, lane);
        }
    }
}

}  // namespace

cudaError_t launch_dropout(emtk_type type, int m, int n, const emtk_matrix &x, const emtk_matrix &y, const emtk_drop &drop,
                           int sms, cudaStream_t s) {
    if (m == 0 || n == 0) return cudaSuccess;
    DropoutArgs a{};
    a.x = rows16_of(x);
    a.y = rows16_of(y);
    a.drop = drop_of(drop);
    a.m = m;
    a.n = n;
    a.lanes_log2 = 5;  // lanes beyond a short row would idle
    while (a.lanes_log2 > 2 && (kPiece << (a.lanes_log2 - 1)) >= n) --a.lanes_log2;
    const int64_t cols = kPiece << a.lanes_log2;
    a.runs = (int)((n + cols - 1) / cols);
    const int64_t all = (int64_t)m * a.runs, per_block = kThreads >> a.lanes_log2;
    const unsigned blocks = (unsigned)std::min<int64_t>((all + per_block - 1) / per_block, 16ll * sms);
    a.step_rows = blocks * per_block / a.runs;
    a.step_runs = (int)(blocks * per_block % a.runs);
    const bool any = !on_grid(x, m) || !on_grid(y, m), f16 = type == EMTK_TYPE_F16;
    return launch_pdl(any ? (f16 ? dropout_kernel<true, true> : dropout_kernel<false, true>)
                          : (f16 ? dropout_kernel<true, false> : dropout_kernel<false, false>),
                      dim3(blocks), dim3(kThreads), 0, s, a);
}

}  // namespace emtk
