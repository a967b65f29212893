// C ABI of the dense layers, gated blocks and 8-bit checkpoints
// (include/emtk.h): argument checks, workspace and the launches of each call.
#include <cuda.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <new>

#include "emtk_internal.h"
#include "nn_internal.h"

using namespace emtk;

namespace {

struct DeviceGuard {  // restores the caller's current device
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        ok = prev == dev || cudaSetDevice(dev) == cudaSuccess;
        if (prev == dev) prev = -1;
    }
    ~DeviceGuard() {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

struct Range {  // NVTX range on the host thread
    explicit Range(const char *name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
};

emtk_status status_of(cudaError_t e) {
    if (e == cudaSuccess) return EMTK_OK;
    cudaGetLastError();  // reported here; not left for a later launch to find
    return e == cudaErrorMemoryAllocation ? EMTK_ERR_OOM : EMTK_ERR_CUDA;
}

bool type16(int t) { return t == EMTK_TYPE_BF16 || t == EMTK_TYPE_F16; }
bool act_known(int a) { return a >= EMTK_ACT_NONE && a <= EMTK_ACT_SIGMOID; }
constexpr int32_t kMaxSize = 1 << 30;
bool sizes_ok(int32_t a, int32_t b, int32_t c) { return std::min({a, b, c}) >= 0 && std::max({a, b, c}) <= kMaxSize; }
size_t align_up(size_t v) { return (v + 255) / 256 * 256; }

// Collects the first argument error of a call.
struct Checks {
    emtk_status st = EMTK_OK;
    void fail(emtk_status s) {
        if (st == EMTK_OK) st = s;
    }
    void need(bool ok) {
        if (!ok) fail(EMTK_ERR_ARG);
    }
    // A matrix of rows x cols elements of elem bytes; q8: a checkpoint is allowed too.
    void matrix(const emtk_matrix &m, int64_t rows, int64_t cols, bool required, bool q8, size_t elem = 2) {
        if (m.d_scale && !q8) return fail(EMTK_ERR_ARG);
        if (!m.d) {
            if (m.d_scale || (required && rows > 0 && cols > 0)) fail(EMTK_ERR_ARG);
            return;
        }
        if (m.ld < cols) return fail(EMTK_ERR_ARG);
        if (m.d_scale) {
            if (m.ld_scale < (cols + kQ8Block - 1) / kQ8Block) fail(EMTK_ERR_ARG);
            return;
        }
        if (reinterpret_cast<uintptr_t>(m.d) % elem) fail(EMTK_ERR_ALIGN);
    }
    void vector(const void *p, size_t elem) {
        if (reinterpret_cast<uintptr_t>(p) % elem) fail(EMTK_ERR_ALIGN);
    }
};

// Workspace of one call, laid out front to back: a first pass adds up the
// sizes, ensure() makes room, a second pass hands out the addresses.  A workspace
// whose address a captured call holds is kept when it is outgrown: the graph may
// be replayed at any time.
struct CallSpace {
    emtk_nn *nn;
    size_t used = 0;
    bool dry = true;
    void *take(size_t bytes) {
        void *p = dry ? nullptr : static_cast<uint8_t *>(nn->ws) + used;
        used += align_up(bytes);
        return p;
    }
    emtk_status ensure(cudaStream_t s) {
        dry = false;
        const size_t bytes = used;
        used = 0;
        if (bytes == 0) return EMTK_OK;
        cudaStreamCaptureStatus capture;
        cudaError_t e = cudaStreamIsCapturing(s, &capture);
        if (e != cudaSuccess) return status_of(e);
        const bool capturing = capture != cudaStreamCaptureStatusNone;
        if (bytes <= nn->ws_bytes) {
            nn->captured = nn->captured || capturing;
            return EMTK_OK;
        }
        if (capturing) return EMTK_ERR_CUDA;  // refused before it would spoil the capture
        if (nn->captured) {
            emtk_nn::Outgrown *const kept = new (std::nothrow) emtk_nn::Outgrown{nn->ws, nn->outgrown};
            if (!kept) return EMTK_ERR_OOM;
            nn->outgrown = kept;
            nn->captured = false;
        } else {
            e = cudaStreamSynchronize(s);  // earlier calls may still use the old one
            if (e != cudaSuccess) return status_of(e);
            e = dev_free(nn->ws);
        }
        nn->ws = nullptr;
        nn->ws_bytes = 0;
        size_t device_free = 0, device_total = 0;
        if (e == cudaSuccess) e = cudaMemGetInfo(&device_free, &device_total);
        const size_t size = workspace_size(bytes, device_free);
        if (e == cudaSuccess) e = dev_alloc(&nn->ws, size);
        if (e != cudaSuccess) return status_of(e);
        nn->ws_bytes = size;
        return EMTK_OK;
    }
};

// Operands of a call's products that cannot be read where they lie (a
// checkpoint, or rows off the 16-byte grid): each gets a copy in the workspace.
struct Staging {
    CallSpace &ws;
    Copy16 copies[kMaxCopies];
    int n = 0;
    emtk_matrix operator()(const emtk_matrix &m, int rows, int cols);
};

int64_t ld16(int64_t cols) { return (cols + 7) / 8 * 8; }  // rows of 16-byte multiples

emtk_matrix Staging::operator()(const emtk_matrix &m, int rows, int cols) {
    if (rows == 0 || cols == 0 || (!m.d_scale && mm_operand_ok(m.d, m.ld, rows))) return m;
    Copy16 &c = copies[n++];
    c = {m, {ws.take(2 * (size_t)rows * ld16(cols)), ld16(cols), nullptr, 0}, rows, cols};
    return c.to;
}

MmOperand rows_of(const emtk_matrix &m) { return {m.d, m.ld, false}; }
MmOperand cols_of(const emtk_matrix &m) { return {m.d, m.ld, true}; }

// The forward pass of a layer: x [M][K] and one or two weights [N][K].
emtk_status forward(emtk_nn *nn, MmJob &j, const emtk_matrix &x, const emtk_matrix *w, cudaStream_t s) {
    const int nw = j.kind == kMmGated ? 2 : 1;
    j.terms = 1;
    j.a[0] = rows_of(x);
    for (int i = 0; i < nw; ++i) j.b[i] = rows_of(w[i]);
    if (few_rows(j)) return status_of(launch_rows(j, nn->sm_count, s));
    const bool thin = skinny(j, nn->sm_count);
    const MmPlan plan = thin ? MmPlan{} : plan_mm(&j, 1, nn->sm_count);
    CallSpace ws{nn};
    Staging stage{ws};
    void *partial = nullptr;
    for (int pass = 0; pass < 2; ++pass) {
        stage.n = 0;
        j.a[0] = rows_of(stage(x, j.M, j.K));
        for (int i = 0; i < nw; ++i) j.b[i] = rows_of(stage(w[i], j.N, j.K));
        partial = ws.take(plan.workspace);
        if (pass == 0) {
            const emtk_status st = ws.ensure(s);
            if (st != EMTK_OK) return st;
        }
    }
    cudaError_t e = launch_copy16(j.type, stage.copies, stage.n, nn->sm_count, s);
    if (e == cudaSuccess) e = thin ? launch_skinny(j, nn, s) : launch_mm(&j, 1, plan, nn, partial, s);
    return status_of(e);
}

// The status of a backward call.  Where a launch failed, the products have not reset the
// slopes' range.
emtk_status finished(cudaError_t e, SlopeRange *range, cudaStream_t s) {
    const emtk_status st = status_of(e);
    if (st != EMTK_OK && range) status_of(cudaMemsetAsync(range, 0, sizeof(SlopeRange), s));
    return st;
}

}  // namespace

extern "C" {

emtk_status emtk_nn_create(int device, int64_t workspace_bytes, int64_t wait_timeout_ns, int32_t debug_stall,
                           emtk_nn **out) {
    if (out) *out = nullptr;
    if (!out || device < 0 || workspace_bytes < 0 || wait_timeout_ns <= 0 || (debug_stall != 0 && debug_stall != 1))
        return EMTK_ERR_ARG;
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || device >= ndev) return EMTK_ERR_CUDA;
    DeviceGuard g(device);
    if (!g.ok) return EMTK_ERR_CUDA;
    cudaDeviceProp prop;
    if (cudaGetDeviceProperties(&prop, device) != cudaSuccess) return EMTK_ERR_CUDA;
    if (!(prop.major == 10 && prop.minor == 3)) return EMTK_ERR_UNSUPPORTED;  // built for sm_103a only
    emtk_nn *nn = new (std::nothrow) emtk_nn;
    if (!nn) return EMTK_ERR_OOM;
    nn->device = device;
    nn->sm_count = prop.multiProcessorCount;
    nn->timeout_ns = wait_timeout_ns;
    nn->debug_stall = debug_stall;
    void *status = nullptr;
    cudaDriverEntryPointQueryResult found;
    cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &nn->encode, 12000, cudaEnableDefault,
                                                     &found);
    if (e == cudaSuccess && (nn->encode == nullptr || found != cudaDriverEntryPointSuccess)) e = cudaErrorNotSupported;
    if (e == cudaSuccess) e = init_mm_kernels();
    if (e == cudaSuccess) e = dev_alloc(&status, sizeof(int) + sizeof(SlopeRange));
    nn->status = static_cast<int *>(status);
    nn->range = reinterpret_cast<SlopeRange *>(nn->status + 1);
    if (e == cudaSuccess) e = cudaMemset(nn->status, 0, sizeof(int) + sizeof(SlopeRange));
    if (e == cudaSuccess && workspace_bytes > 0) {
        e = dev_alloc(&nn->ws, (size_t)workspace_bytes);
        if (e == cudaSuccess) nn->ws_bytes = (size_t)workspace_bytes;
    }
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        emtk_nn_destroy(nn);
        return status_of(e);
    }
    *out = nn;
    return EMTK_OK;
}

emtk_status emtk_nn_destroy(emtk_nn *nn) {
    if (!nn) return EMTK_OK;
    DeviceGuard g(nn->device);
    cudaError_t e = cudaDeviceSynchronize();
    dev_free(nn->ws);
    while (emtk_nn::Outgrown *const o = nn->outgrown) {
        dev_free(o->ws);
        nn->outgrown = o->next;
        delete o;
    }
    dev_free(nn->status);
    delete nn;
    return e == cudaSuccess ? EMTK_OK : EMTK_ERR_CUDA;
}

emtk_status emtk_nn_check(emtk_nn *nn, emtk_stream stream) {
    if (!nn) return EMTK_ERR_ARG;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    if (cudaStreamSynchronize(reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess) return EMTK_ERR_CUDA;
    int status = 0;
    if (cudaMemcpy(&status, nn->status, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess) return EMTK_ERR_CUDA;
    if (status == 0) return EMTK_OK;
    return cudaMemset(nn->status, 0, sizeof(int)) == cudaSuccess ? EMTK_ERR_TIMEOUT : EMTK_ERR_CUDA;
}

emtk_status emtk_dense(emtk_nn *nn, const emtk_dense_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_dense_args &a = *p;
    Checks c;
    c.need(sizes_ok(a.m, a.n, a.k) && act_known(a.act) && type16(a.type));
    if (a.bias) c.need(a.bias_type == a.type || a.bias_type == EMTK_TYPE_F32);
    if (c.st != EMTK_OK) return c.st;
    c.matrix(a.x, a.m, a.k, true, false);
    c.matrix(a.w, a.n, a.k, true, false);
    c.matrix(a.y, a.m, a.n, true, false);
    c.matrix(a.residual, a.m, a.n, false, false);
    c.matrix(a.pre, a.m, a.n, false, true);
    c.vector(a.bias, a.bias_type == EMTK_TYPE_F32 ? 4 : 2);
    if (c.st != EMTK_OK || a.m == 0 || a.n == 0) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk dense");
    MmJob j{};
    j.kind = kMmSum;
    j.type = (emtk_type)a.type;
    j.M = a.m;
    j.N = a.n;
    j.K = a.k;
    j.epi.act = a.act;
    j.epi.bias[0] = a.bias;
    j.epi.bias_f32 = a.bias_type == EMTK_TYPE_F32;
    j.epi.residual = a.residual;
    j.epi.out = a.y;
    j.epi.saved[0] = a.pre;
    return forward(nn, j, a.x, &a.w, reinterpret_cast<cudaStream_t>(stream));
}

emtk_status emtk_dense_backward(emtk_nn *nn, const emtk_dense_grad_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_dense_grad_args &a = *p;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    Checks c;
    c.need(sizes_ok(a.m, a.n, a.k) && act_known(a.act) && type16(a.type));
    if (a.dw.d) c.need(a.dw_type == a.type || a.dw_type == EMTK_TYPE_F32);
    if (c.st != EMTK_OK) return c.st;
    c.matrix(a.dy, a.m, a.n, true, false);
    c.matrix(a.x, a.m, a.k, a.dw.d != nullptr, true);
    c.matrix(a.w, a.n, a.k, a.dx.d != nullptr, false);
    c.matrix(a.pre, a.m, a.n, a.act != EMTK_ACT_NONE, true);
    c.matrix(a.dx, a.m, a.k, false, false);
    c.matrix(a.dw, a.n, a.k, false, false, a.dw_type == EMTK_TYPE_F32 ? 4 : 2);
    c.vector(a.db, 4);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk dense backward");
    const emtk_type type = (emtk_type)a.type;
    const bool dx = a.dx.d && a.m > 0 && a.k > 0, dw = a.dw.d && a.n > 0 && a.k > 0;
    const bool own_dz = a.act != EMTK_ACT_NONE && (dx || dw);
    CallSpace ws{nn};
    Staging stage{ws};
    MmJob jobs[2]{};
    int n = 0;
    for (MmJob &j : jobs) {
        j.kind = kMmSum;
        j.type = type;
        j.terms = 1;
        j.N = a.k;
    }
    MmJob &jx = jobs[n], &jw = jobs[n + (dx ? 1 : 0)];
    if (dx) {
        jx.M = a.m;
        jx.K = a.n;
        jx.epi.out = a.dx;
        ++n;
    }
    if (dw) {
        jw.M = a.n;
        jw.K = a.m;
        jw.epi.out = a.dw;
        jw.epi.out_f32 = a.dw_type == EMTK_TYPE_F32;
        ++n;
    }
    MmPlan plan{};
    if (n > 0) plan = plan_mm(jobs, n, nn->sm_count);
    emtk_matrix dz{};
    float *sums = nullptr;
    void *partial = nullptr;
    for (int pass = 0; pass < 2; ++pass) {
        stage.n = 0;
        if (own_dz)
            dz = emtk_matrix{ws.take(2 * (size_t)a.m * ld16(a.n)), ld16(a.n), nullptr, 0};
        else if (n > 0)
            dz = stage(a.dy, a.m, a.n);
        if (dx) {
            jx.a[0] = rows_of(dz);
            jx.b[0] = cols_of(stage(a.w, a.n, a.k));
        }
        if (dw) {
            jw.a[0] = cols_of(dz);
            jw.b[0] = cols_of(stage(a.x, a.m, a.k));
        }
        partial = ws.take(plan.workspace);
        if (a.db) sums = static_cast<float *>(ws.take(4 * (size_t)slope_slices(a.m, a.n, nn->sm_count) * a.n));
        if (pass == 0) {
            const emtk_status st = ws.ensure(s);
            if (st != EMTK_OK) return st;
        }
    }
    // (ReLU's dz is dy or 0 and rounds nothing.)
    SlopeRange *const kept_in = own_dz && type == EMTK_TYPE_F16 && a.act != EMTK_ACT_RELU ? nn->range : nullptr;
    for (MmJob &j : jobs) j.epi.range = kept_in;
    cudaError_t e = cudaSuccess;
    if (own_dz || a.db)
        e = launch_slope(type, a.act, a.m, a.n, a.dy, a.pre, own_dz ? dz.d : nullptr, dz.ld, a.db, sums, kept_in,
                         nn->sm_count, s);
    if (e == cudaSuccess) e = launch_copy16(type, stage.copies, stage.n, nn->sm_count, s);
    if (e == cudaSuccess && n > 0) e = launch_mm(jobs, n, plan, nn, partial, s);
    return finished(e, kept_in, s);
}

emtk_status emtk_gated(emtk_nn *nn, const emtk_gated_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_gated_args &a = *p;
    Checks c;
    c.need(sizes_ok(a.m, a.f, a.k) && act_known(a.act) && type16(a.type));
    c.need((a.bias_gate == nullptr) == (a.bias_up == nullptr) && (a.gate.d == nullptr) == (a.up.d == nullptr));
    if (a.bias_gate) c.need(a.bias_type == a.type || a.bias_type == EMTK_TYPE_F32);
    if (c.st != EMTK_OK) return c.st;
    c.matrix(a.x, a.m, a.k, true, false);
    c.matrix(a.w_gate, a.f, a.k, true, false);
    c.matrix(a.w_up, a.f, a.k, true, false);
    c.matrix(a.h, a.m, a.f, true, false);
    c.matrix(a.gate, a.m, a.f, false, true);
    c.matrix(a.up, a.m, a.f, false, true);
    for (const void *b : {a.bias_gate, a.bias_up}) c.vector(b, a.bias_type == EMTK_TYPE_F32 ? 4 : 2);
    if (c.st != EMTK_OK || a.m == 0 || a.f == 0) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk gated");
    MmJob j{};
    j.kind = kMmGated;
    j.type = (emtk_type)a.type;
    j.M = a.m;
    j.N = a.f;
    j.K = a.k;
    j.epi.act = a.act;
    j.epi.bias[0] = a.bias_gate;
    j.epi.bias[1] = a.bias_up;
    j.epi.bias_f32 = a.bias_type == EMTK_TYPE_F32;
    j.epi.out = a.h;
    j.epi.saved[0] = a.gate;
    j.epi.saved[1] = a.up;
    const emtk_matrix w[2] = {a.w_gate, a.w_up};
    return forward(nn, j, a.x, w, reinterpret_cast<cudaStream_t>(stream));
}

emtk_status emtk_gated_backward(emtk_nn *nn, const emtk_gated_grad_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_gated_grad_args &a = *p;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    Checks c;
    c.need(sizes_ok(a.m, a.f, a.k) && act_known(a.act) && type16(a.type));
    c.need((a.dw_gate.d == nullptr) == (a.dw_up.d == nullptr) && (a.db_gate == nullptr) == (a.db_up == nullptr));
    c.need((a.gate.d_scale == nullptr) == (a.up.d_scale == nullptr));
    if (a.dw_gate.d) c.need(a.dw_type == a.type || a.dw_type == EMTK_TYPE_F32);
    if (c.st != EMTK_OK) return c.st;
    const size_t dw_elem = a.dw_type == EMTK_TYPE_F32 ? 4 : 2;
    c.matrix(a.dh, a.m, a.f, true, false);
    c.matrix(a.gate, a.m, a.f, true, true);
    c.matrix(a.up, a.m, a.f, true, true);
    c.matrix(a.x, a.m, a.k, a.dw_gate.d != nullptr, true);
    c.matrix(a.w_gate, a.f, a.k, a.dx.d != nullptr, false);
    c.matrix(a.w_up, a.f, a.k, a.dx.d != nullptr, false);
    c.matrix(a.dx, a.m, a.k, false, false);
    c.matrix(a.dw_gate, a.f, a.k, false, false, dw_elem);
    c.matrix(a.dw_up, a.f, a.k, false, false, dw_elem);
    c.matrix(a.h, a.m, a.f, false, false);
    c.vector(a.db_gate, 4);
    c.vector(a.db_up, 4);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk gated backward");
    const emtk_type type = (emtk_type)a.type;
    const bool dx = a.dx.d && a.m > 0 && a.k > 0, dw = a.dw_gate.d && a.f > 0 && a.k > 0;
    CallSpace ws{nn};
    Staging stage{ws};
    MmJob jobs[3]{};
    int n = 0;
    for (MmJob &j : jobs) {
        j.kind = kMmSum;
        j.type = type;
        j.terms = 1;
        j.N = a.k;
    }
    MmJob &jx = jobs[0];
    MmJob *const jw = jobs + (dx ? 1 : 0);  // of w_gate and w_up
    if (dx) {
        jx.terms = 2;
        jx.M = a.m;
        jx.K = a.f;
        jx.epi.out = a.dx;
        ++n;
    }
    for (int w = 0; w < 2 && dw; ++w) {
        jw[w].M = a.f;
        jw[w].K = a.m;
        jw[w].epi.out = w ? a.dw_up : a.dw_gate;
        jw[w].epi.out_f32 = a.dw_type == EMTK_TYPE_F32;
        ++n;
    }
    MmPlan plan{};
    if (n > 0) plan = plan_mm(jobs, n, nn->sm_count);
    emtk_matrix dg{}, du{};
    float *sums = nullptr;
    void *partial = nullptr;
    for (int pass = 0; pass < 2; ++pass) {
        stage.n = 0;
        if (n > 0) {
            dg = emtk_matrix{ws.take(2 * (size_t)a.m * ld16(a.f)), ld16(a.f), nullptr, 0};
            du = emtk_matrix{ws.take(2 * (size_t)a.m * ld16(a.f)), ld16(a.f), nullptr, 0};
        }
        if (dx) {
            jx.a[0] = rows_of(dg);
            jx.a[1] = rows_of(du);
            jx.b[0] = cols_of(stage(a.w_gate, a.f, a.k));
            jx.b[1] = cols_of(stage(a.w_up, a.f, a.k));
        }
        if (dw) {
            jw[0].a[0] = cols_of(dg);
            jw[1].a[0] = cols_of(du);
            jw[0].b[0] = jw[1].b[0] = cols_of(stage(a.x, a.m, a.k));
        }
        partial = ws.take(plan.workspace);
        if (a.db_gate) sums = static_cast<float *>(ws.take(8 * (size_t)slope_slices(a.m, a.f, nn->sm_count) * a.f));
        if (pass == 0) {
            const emtk_status st = ws.ensure(s);
            if (st != EMTK_OK) return st;
        }
    }
    SlopeRange *const kept_in = n > 0 && type == EMTK_TYPE_F16 ? nn->range : nullptr;
    for (MmJob &j : jobs) j.epi.range = kept_in;
    cudaError_t e = cudaSuccess;
    if (n > 0 || a.db_gate || a.h.d)
        e = launch_gated_slope(type, a.act, a.m, a.f, a.dh, a.gate, a.up, dg.d, du.d, ld16(a.f), a.h, a.db_gate,
                               a.db_up, sums, kept_in, nn->sm_count, s);
    if (e == cudaSuccess) e = launch_copy16(type, stage.copies, stage.n, nn->sm_count, s);
    if (e == cudaSuccess && n > 0) e = launch_mm(jobs, n, plan, nn, partial, s);
    return finished(e, kept_in, s);
}

emtk_status emtk_pack8(emtk_nn *nn, int32_t m, int32_t k, emtk_type type, const emtk_matrix *x, const emtk_matrix *q,
                       emtk_stream stream) {
    if (!nn || !x || !q || !sizes_ok(m, k, 0) || !type16(type)) return EMTK_ERR_ARG;
    Checks c;
    c.matrix(*x, m, k, true, false);
    c.matrix(*q, m, k, true, true);
    if (m > 0 && k > 0) c.need(q->d_scale != nullptr);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk pack8");
    return status_of(launch_pack8(type, m, k, *x, *q, nn->sm_count, reinterpret_cast<cudaStream_t>(stream)));
}

emtk_status emtk_unpack8(emtk_nn *nn, int32_t m, int32_t k, emtk_type type, const emtk_matrix *q, const emtk_matrix *x,
                         emtk_stream stream) {
    if (!nn || !x || !q || !sizes_ok(m, k, 0) || !type16(type)) return EMTK_ERR_ARG;
    Checks c;
    c.matrix(*x, m, k, true, false);
    c.matrix(*q, m, k, true, true);
    if (m > 0 && k > 0) c.need(q->d_scale != nullptr);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk unpack8");
    const Copy16 copy{*q, *x, m, k};
    return status_of(launch_copy16(type, &copy, 1, nn->sm_count, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
