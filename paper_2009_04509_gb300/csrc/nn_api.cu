// C ABI of the layers and of what stands around them (include/emtk.h): argument
// checks, workspace and the launches of each call.
#include <cuda.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
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
    // Two matrices share no element, or all of them (the same address and ld).
    void whole_or_apart(const emtk_matrix &a, const emtk_matrix &b, bool may_be_same) {
        if (a.d && a.d == b.d && (a.ld != b.ld || !may_be_same)) fail(EMTK_ERR_ARG);
    }
    void norm(const emtk_norm &n, int type) {
        need(n.kind >= EMTK_NORM_NONE && n.kind <= EMTK_NORM_LAYER);
        if (n.kind == EMTK_NORM_NONE) return need(!n.weight && !n.bias);
        need(n.eps >= 0.f && n.eps < INFINITY);
        if (!n.weight && !n.bias) return;
        need(n.param_type == type || n.param_type == EMTK_TYPE_F32);
        for (const void *p : {n.weight, n.bias}) vector(p, n.param_type == EMTK_TYPE_F32 ? 4 : 2);
    }
    // > 0, and log2(e) / temperature, which the kernels scale logits by, finite.
    void temperature(float t) { need(t > 0.f && t < INFINITY && 1.4426950408889634f * (1.f / t) < INFINITY); }
    void drop(const emtk_drop &d) {
        need(d.p >= 0.f && d.p < 1.f);
        vector(d.d_offset, 8);
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

// The workspace of a recurrence's call, which begins with what its kernels leave each other;
// inputs that are to be read from a copy there become that copy.
template <typename Args>
emtk_status recurrence_inputs(emtk_nn *nn, const Args &a, std::initializer_list<emtk_matrix *> inputs, cudaStream_t s) {
    const bool uniform = a.offsets == nullptr;
    bool tma = true;  // what is not copied lies on its grid
    for (const emtk_matrix *m : inputs)
        tma = tma && (!m->d || mm_operand_ok(m->d, m->ld, a.rows) || recurrence_copies(*m, a.rows, a.n, a.seqs, uniform, nn->sm_count));
    const size_t kept = recurrence_workspace(a.rows, a.n, a.seqs, uniform, tma, nn->sm_count);
    CallSpace ws{nn};
    Staging stage{ws};
    for (int pass = 0; pass < 2; ++pass) {
        stage.n = 0;
        ws.take(kept);
        for (emtk_matrix *m : inputs) {
            if (!recurrence_copies(*m, a.rows, a.n, a.seqs, uniform, nn->sm_count)) continue;
            const emtk_matrix there = stage(*m, a.rows, a.n);
            if (pass == 1) *m = there;
        }
        if (pass == 0) {
            const emtk_status st = ws.ensure(s);
            if (st != EMTK_OK) return st;
        }
    }
    return status_of(launch_copy16((emtk_type)a.type, stage.copies, stage.n, nn->sm_count, s));
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

int64_t gate_rows(int32_t m, int32_t every) { return std::max<int64_t>(1, ((int64_t)m + every - 1) / every); }

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
    if (e == cudaSuccess) e = init_norm_kernels();
    if (e == cudaSuccess) e = init_recur_kernels();
    const size_t head = align_up(sizeof(int) + sizeof(SlopeRange));
    if (e == cudaSuccess) e = dev_alloc(&status, head + sizeof(float2) * kCutRows * nn->sm_count);
    nn->status = static_cast<int *>(status);
    nn->range = reinterpret_cast<SlopeRange *>(nn->status + 1);
    nn->far_sums = reinterpret_cast<float2 *>(static_cast<uint8_t *>(status) + head);
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

emtk_status emtk_dropout(emtk_nn *nn, int32_t m, int32_t n, emtk_type type, const emtk_matrix *x, const emtk_matrix *y,
                         const emtk_drop *drop, emtk_stream stream) {
    if (!nn || !x || !y || !drop || !sizes_ok(m, n, 0) || !type16(type)) return EMTK_ERR_ARG;
    Checks c;
    c.matrix(*x, m, n, true, false);
    c.matrix(*y, m, n, true, false);
    c.whole_or_apart(*x, *y, true);
    c.drop(*drop);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk dropout");
    return status_of(launch_dropout(type, m, n, *x, *y, *drop, nn->sm_count, reinterpret_cast<cudaStream_t>(stream)));
}

emtk_status emtk_residual_norm(emtk_nn *nn, const emtk_residual_norm_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_residual_norm_args &a = *p;
    Checks c;
    c.need(sizes_ok(a.m, a.n, 0) && a.n <= kMaxNormWidth && type16(a.type));
    c.need(!a.gate.d || a.gate_every > 0);
    if (c.st != EMTK_OK) return c.st;
    c.norm(a.post, a.type);
    c.norm(a.pre, a.type);
    c.drop(a.drop);
    if (a.m > 0 && a.n > 0) {  // what has no elements may have no address
        c.need(a.block.d || (a.post.kind == EMTK_NORM_NONE && !a.gate.d && a.drop.p == 0.f));
        c.need((a.residual.d || a.block.d) && (a.y.d || a.h.d) && (a.h.d != nullptr) == (a.pre.kind != EMTK_NORM_NONE));
    }
    c.matrix(a.residual, a.m, a.n, false, false);
    c.matrix(a.block, a.m, a.n, false, false);
    if (c.st == EMTK_OK && a.gate.d) c.matrix(a.gate, gate_rows(a.m, a.gate_every), a.n, false, false);
    c.matrix(a.y, a.m, a.n, false, false);
    c.matrix(a.h, a.m, a.n, false, false);
    c.whole_or_apart(a.y, a.residual, true);
    for (const emtk_matrix *in : {&a.block, &a.gate}) c.whole_or_apart(a.y, *in, false);
    for (const emtk_matrix *in : {&a.block, &a.gate, &a.residual, &a.y}) c.whole_or_apart(a.h, *in, false);
    if (c.st != EMTK_OK || a.m == 0 || a.n == 0) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk residual norm");
    return status_of(launch_residual_norm(a, nn, reinterpret_cast<cudaStream_t>(stream)));
}

emtk_status emtk_residual_norm_backward(emtk_nn *nn, const emtk_residual_norm_grad_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    emtk_residual_norm_grad_args a = *p;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    Checks c;
    c.need(sizes_ok(a.m, a.n, 0) && a.n <= kMaxNormWidth && type16(a.type));
    if (!a.gate.d && !a.d_gate.d) a.gate_every = std::max(1, a.m);
    c.need(a.gate_every > 0);
    if (c.st != EMTK_OK) return c.st;
    const bool pre = a.pre.kind != EMTK_NORM_NONE, post = a.post.kind != EMTK_NORM_NONE;
    const int64_t gates = gate_rows(a.m, a.gate_every);
    c.norm(a.post, a.type);
    c.norm(a.pre, a.type);
    c.drop(a.drop);
    if (a.m > 0 && a.n > 0) {
        c.need((a.dh.d != nullptr) == pre && (a.dy.d || a.dh.d));
        c.need(a.block.d || (!post && !a.gate.d && a.drop.p == 0.f));
    }
    c.need(pre || (!a.dw_pre && !a.db_pre));
    c.need(post || (!a.dw_post && !a.db_post));
    c.matrix(a.dy, a.m, a.n, false, false);
    c.matrix(a.dh, a.m, a.n, pre, false);
    c.matrix(a.y, a.m, a.n, pre, false);
    c.matrix(a.block, a.m, a.n, a.d_block.d || a.d_gate.d || a.dw_post || a.db_post, false);
    c.matrix(a.gate, gates, a.n, false, false);
    c.matrix(a.d_residual, a.m, a.n, false, false);
    c.matrix(a.d_block, a.m, a.n, false, false);
    c.matrix(a.d_gate, gates, a.n, false, false, 4);
    for (const void *v : {a.dw_pre, a.db_pre, a.dw_post, a.db_post}) c.vector(v, 4);
    c.whole_or_apart(a.d_residual, a.dy, true);
    c.whole_or_apart(a.d_block, a.d_residual, false);
    for (const emtk_matrix *in : {&a.dh, &a.y, &a.block, &a.gate}) c.whole_or_apart(a.d_residual, *in, false);
    for (const emtk_matrix *in : {&a.dy, &a.dh, &a.y, &a.block, &a.gate}) c.whole_or_apart(a.d_block, *in, false);
    if (c.st != EMTK_OK || a.n == 0) return c.st;
    if (!a.d_block.d && !a.d_gate.d && !a.dw_post && !a.db_post) a.block.d = nullptr;  // nothing needs it
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk residual norm backward");
    // The sums past the block's norm read dy after d_residual is written: where that takes its place, a
    // copy, which lies alike, so that the sums are the same.
    const bool copied = a.m > 0 && a.dy.d && a.dy.d == a.d_residual.d && (a.d_gate.d || a.dw_post || a.db_post);
    emtk_matrix copy{nullptr, ld16(a.n) + a.dy.ld % 8, nullptr, 0};
    CallSpace ws{nn};
    void *space = nullptr;
    for (int pass = 0; pass < 2; ++pass) {
        space = ws.take(residual_norm_workspace(a, nn->sm_count));
        if (copied) copy.d = ws.take(16 + 2 * (size_t)a.m * copy.ld);
        const emtk_status st = pass == 0 ? ws.ensure(s) : EMTK_OK;
        if (st != EMTK_OK) return st;
    }
    if (copied) {
        copy.d = static_cast<uint8_t *>(copy.d) + reinterpret_cast<uintptr_t>(a.dy.d) % 16;
        const cudaError_t e = launch_dropout((emtk_type)a.type, a.m, a.n, a.dy, copy, emtk_drop{}, nn->sm_count, s);  // of nothing: a copy to any rows
        if (e != cudaSuccess) return status_of(e);
        a.dy = copy;
    }
    return status_of(launch_residual_norm_grad(a, space, nn, s));
}

emtk_status emtk_logprobs(emtk_nn *nn, const emtk_logprobs_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_logprobs_args &a = *p;
    Checks c;
    c.need(sizes_ok(a.m, a.v, 0) && (type16(a.type) || a.type == EMTK_TYPE_F32));
    c.need(a.top >= 0 && a.top <= std::min(32, a.v));
    c.temperature(a.temperature);
    c.need((a.tokens == nullptr) == (a.logprob == nullptr));
    c.need((a.top > 0) == (a.top_logprob != nullptr) && (a.top > 0) == (a.top_index != nullptr));
    if (c.st != EMTK_OK) return c.st;
    c.matrix(a.logits, a.m, a.v, true, false, a.type == EMTK_TYPE_F32 ? 4 : 2);
    for (const void *v : {(const void *)a.tokens, (const void *)a.logprob, (const void *)a.entropy, (const void *)a.lse,
                          (const void *)a.top_logprob, (const void *)a.top_index})
        c.vector(v, 4);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk logprobs");
    return status_of(launch_logprobs(a, nn->sm_count, reinterpret_cast<cudaStream_t>(stream)));
}

emtk_status emtk_logprobs_backward(emtk_nn *nn, const emtk_logprobs_grad_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_logprobs_grad_args &a = *p;
    const size_t elem = a.type == EMTK_TYPE_F32 ? 4 : 2;
    Checks c;
    c.need(sizes_ok(a.m, a.v, 0) && (type16(a.type) || a.type == EMTK_TYPE_F32));
    c.temperature(a.temperature);
    c.need(a.m == 0 || a.lse);
    c.need(!a.d_logprob || a.tokens);
    c.need(!a.d_entropy || a.entropy);
    if (c.st != EMTK_OK) return c.st;
    c.matrix(a.logits, a.m, a.v, true, false, elem);
    c.matrix(a.d_logits, a.m, a.v, true, false, elem);
    c.whole_or_apart(a.d_logits, a.logits, true);
    for (const void *v : {(const void *)a.tokens, (const void *)a.lse, (const void *)a.entropy, (const void *)a.d_logprob,
                          (const void *)a.d_entropy})
        c.vector(v, 4);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk logprobs backward");
    return status_of(launch_logprobs_grad(a, nn, reinterpret_cast<cudaStream_t>(stream)));
}

emtk_status emtk_recurrence(emtk_nn *nn, const emtk_recurrence_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_recurrence_args &a = *p;
    Checks c;
    c.need(sizes_ok(a.rows, a.n, a.seqs) && act_known(a.act) && type16(a.type));
    if (c.st != EMTK_OK) return c.st;
    c.need(a.offsets || (a.seqs > 0 ? a.rows % a.seqs == 0 : a.rows == 0));
    const bool some = a.rows > 0 && a.n > 0;  // what has no elements may have no address
    c.need(!some || a.o.d || a.act == EMTK_ACT_NONE);
    c.matrix(a.f, a.rows, a.n, true, false);
    c.matrix(a.x, a.rows, a.n, true, false);
    c.matrix(a.o, a.rows, a.n, false, false);
    c.matrix(a.y, a.rows, a.n, true, false);
    for (const emtk_matrix *in : {&a.f, &a.x, &a.o}) c.whole_or_apart(a.y, *in, false);
    for (const void *v : {(const void *)a.offsets, (const void *)a.state, (const void *)a.last, (const void *)a.states})
        c.vector(v, 4);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk recurrence");
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    emtk_recurrence_args b = a;
    const emtk_status st = recurrence_inputs(nn, a, {&b.f, &b.x, &b.o}, s);
    return st != EMTK_OK ? st : status_of(launch_recurrence(b, nn->ws, nn, s));
}

emtk_status emtk_recurrence_backward(emtk_nn *nn, const emtk_recurrence_grad_args *p, emtk_stream stream) {
    if (!nn || !p) return EMTK_ERR_ARG;
    const emtk_recurrence_grad_args &a = *p;
    Checks c;
    c.need(sizes_ok(a.rows, a.n, a.seqs) && act_known(a.act) && type16(a.type));
    if (c.st != EMTK_OK) return c.st;
    c.need(a.offsets || (a.seqs > 0 ? a.rows % a.seqs == 0 : a.rows == 0));
    const bool some = a.rows > 0 && a.n > 0;
    c.need(!some || a.o.d || (a.act == EMTK_ACT_NONE && !a.d_o.d));
    c.need(!some || a.states || a.seqs == 0);
    const emtk_matrix *const in[] = {&a.dy, &a.f, &a.x, &a.o}, *const out[] = {&a.df, &a.dx, &a.d_o};
    for (const emtk_matrix *i : in) c.matrix(*i, a.rows, a.n, i != &a.o, false);
    for (const emtk_matrix *o : out) c.matrix(*o, a.rows, a.n, false, false);
    for (const emtk_matrix *o : out)
        for (const emtk_matrix *i : in) c.whole_or_apart(*o, *i, false);
    c.whole_or_apart(a.df, a.dx, false);
    for (const emtk_matrix *o : {&a.df, &a.dx}) c.whole_or_apart(a.d_o, *o, false);
    for (const void *v : {(const void *)a.offsets, (const void *)a.states, (const void *)a.d_last, (const void *)a.d_state})
        c.vector(v, 4);
    if (c.st != EMTK_OK) return c.st;
    DeviceGuard g(nn->device);
    if (!g.ok) return EMTK_ERR_CUDA;
    Range range("emtk recurrence backward");
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    emtk_recurrence_grad_args b = a;
    const emtk_status st = recurrence_inputs(nn, a, {&b.f, &b.x, &b.o, &b.dy}, s);
    return st != EMTK_OK ? st : status_of(launch_recurrence_grad(b, nn->ws, nn, s));
}

}  // extern "C"
