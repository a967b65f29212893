"""Thin ctypes binding of libemtk.so (include/emtk.h), same names as the C ABI.

Only argument marshalling lives here: torch tensors are passed as device
pointers and the current torch stream as the CUDA stream.  Every step of the
hot path runs in the library's kernels.  If the library is not built, loading
fails loudly; there is no other implementation to fall back to.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libemtk.so")

EMTK_OK, EMTK_ERR_ARG, EMTK_ERR_ALIGN, EMTK_ERR_OOM, EMTK_ERR_CUDA, EMTK_ERR_TIMEOUT, EMTK_ERR_UNSUPPORTED = range(7)
EMTK_FP32, EMTK_TF32, EMTK_BF16, EMTK_FP16, EMTK_FP8 = 0, 1, 2, 3, 4
EMTK_PATCH_F32, EMTK_PATCH_BF16, EMTK_PATCH_F16 = 0, 1, 2
PRECISIONS = {"fp32": EMTK_FP32, "tf32": EMTK_TF32, "bf16": EMTK_BF16, "fp16": EMTK_FP16, "fp8": EMTK_FP8}
PATCH_FORMATS = {"f32": EMTK_PATCH_F32, "bf16": EMTK_PATCH_BF16, "fp16": EMTK_PATCH_F16}
EMTK_TYPE_BF16, EMTK_TYPE_F16, EMTK_TYPE_F32 = 0, 1, 2
NORMS = {"none": 0, "rms": 1, "layer": 2}
EMTK_RECURRENCE_STEP = 128
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "sigmoid": 4}
KERNELS = ("intervals", "gather", "network", "head", "convert", "hitfind")

EXPORTED = ("emtk_default_options", "emtk_create", "emtk_destroy", "emtk_infer", "emtk_infer_batch",
            "emtk_extract_patches", "emtk_infer_patches", "emtk_check", "emtk_get_stats",
            "emtk_status_string", "emtk_extract_patches_static", "emtk_batcher_create", "emtk_batcher_submit",
            "emtk_batcher_wait", "emtk_batcher_stats", "emtk_batcher_destroy", "emtk_get_fp8_scales",
            "emtk_find_hits", "emtk_infer_batch_host", "emtk_debug_fail_alloc", "emtk_debug_alloc_counts",
            "emtk_debug_batcher_stall", "emtk_nn_create", "emtk_nn_destroy", "emtk_nn_check", "emtk_dense",
            "emtk_dense_backward", "emtk_gated", "emtk_gated_backward", "emtk_pack8", "emtk_unpack8", "emtk_dropout", "emtk_residual_norm",
            "emtk_residual_norm_backward", "emtk_logprobs", "emtk_logprobs_backward", "emtk_recurrence",
            "emtk_recurrence_backward")
EMTK_STATIC_SCRATCH_BYTES = 4 << 20

_vp = ctypes.c_void_p
_fp = ctypes.POINTER(ctypes.c_float)


class emtk_weights(ctypes.Structure):
    _fields_ = [(k, _fp) for k in ("conv_w", "conv_b", "fc1_w", "fc1_b", "fc2_w", "fc2_b", "cls_w", "cls_b",
                                   "mic_w", "mic_b")]


class emtk_options(ctypes.Structure):
    _fields_ = [("precision", ctypes.c_int), ("max_hits", ctypes.c_int32), ("debug_logits", ctypes.c_int32),
                ("wait_timeout_ns", ctypes.c_int64), ("debug_stall", ctypes.c_int32), ("profile", ctypes.c_int32)]


class emtk_request(ctypes.Structure):
    _fields_ = [("d_adc", _vp), ("nwires", ctypes.c_int32), ("nticks", ctypes.c_int32), ("ld", ctypes.c_int64),
                ("d_hits", _vp), ("nhits", ctypes.c_int32), ("d_scores", _vp)]


class emtk_stats(ctypes.Structure):
    _fields_ = [("calls", ctypes.c_uint64), ("hits", ctypes.c_uint64), ("launches", ctypes.c_uint64),
                ("chunks", ctypes.c_uint64), ("batch_hist", ctypes.c_uint64 * 8),
                ("kernel_launches", ctypes.c_uint64 * 6), ("kernel_ms", ctypes.c_double * 6)]


class emtk_hitfind_request(ctypes.Structure):
    _fields_ = [("d_adc", _vp), ("nwires", ctypes.c_int32), ("nticks", ctypes.c_int32), ("ld", ctypes.c_int64),
                ("threshold", ctypes.c_float), ("capacity", ctypes.c_int32), ("d_hits", _vp), ("d_info", _vp),
                ("n_found", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class emtk_matrix(ctypes.Structure):
    _fields_ = [("d", _vp), ("ld", ctypes.c_int64), ("d_scale", _vp), ("ld_scale", ctypes.c_int64)]


class emtk_drop(ctypes.Structure):
    _fields_ = [("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("d_offset", _vp), ("p", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


class emtk_norm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("param_type", ctypes.c_int32), ("eps", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("weight", _vp), ("bias", _vp)]


def _args_struct(name, ints, matrices, pointers, floats="", parts=()):
    """An argument struct of the layers: int32 fields (those in `floats` fp32), other structs, matrices, pointers."""
    fields = [(f, ctypes.c_float if f in floats.split() else ctypes.c_int32) for f in ints.split()] + list(parts) + \
        [(f, emtk_matrix) for f in matrices.split()] + [(f, _vp) for f in pointers.split()]
    return type(name, (ctypes.Structure,), {"_fields_": fields})


emtk_dense_args = _args_struct("emtk_dense_args", "m n k act type bias_type", "x w y residual pre", "bias")
emtk_dense_grad_args = _args_struct("emtk_dense_grad_args", "m n k act type dw_type", "dy x w pre dx dw", "db")
emtk_gated_args = _args_struct("emtk_gated_args", "m f k act type bias_type", "x w_gate w_up h gate up",
                               "bias_gate bias_up")
emtk_gated_grad_args = _args_struct("emtk_gated_grad_args", "m f k act type dw_type",
                                    "dh gate up x w_gate w_up dx dw_gate dw_up h", "db_gate db_up")
_SEAM_PARTS = (("post", emtk_norm), ("pre", emtk_norm), ("drop", emtk_drop))
emtk_residual_norm_args = _args_struct("emtk_residual_norm_args", "m n type gate_every scale reserved",
                                       "residual block gate y h", "", "scale", _SEAM_PARTS)
emtk_residual_norm_grad_args = _args_struct("emtk_residual_norm_grad_args", "m n type gate_every scale reserved",
                                            "dy dh y block gate d_residual d_block d_gate",
                                            "dw_pre db_pre dw_post db_post", "scale", _SEAM_PARTS)
emtk_logprobs_args = _args_struct("emtk_logprobs_args", "m v type top temperature reserved", "logits",
                                  "tokens logprob entropy lse top_logprob top_index", "temperature")
emtk_logprobs_grad_args = _args_struct("emtk_logprobs_grad_args", "m v type reserved0 temperature reserved",
                                       "logits d_logits", "tokens lse entropy d_logprob d_entropy", "temperature")
emtk_recurrence_args = _args_struct("emtk_recurrence_args", "rows n seqs act type reserved", "f x o y",
                                    "offsets state last states")
emtk_recurrence_grad_args = _args_struct("emtk_recurrence_grad_args", "rows n seqs act type reserved",
                                         "dy f x o df dx d_o", "offsets states d_last d_state")


class EmtkError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


_lib = None


def load_library(path: str | None = None):
    """The ctypes handle of libemtk.so; raises if it was not built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with __graft_entry__.build() "
                           "(there is no CPU fallback)")
    lib = ctypes.CDLL(p)
    lib.emtk_default_options.argtypes = [ctypes.POINTER(emtk_options)]
    lib.emtk_default_options.restype = None
    lib.emtk_create.argtypes = [ctypes.POINTER(emtk_weights), ctypes.POINTER(emtk_options), ctypes.c_int,
                                ctypes.POINTER(_vp)]
    lib.emtk_destroy.argtypes = [_vp]
    lib.emtk_infer.argtypes = [_vp, _vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, _vp, ctypes.c_int32,
                               _vp, _vp]
    lib.emtk_infer_batch.argtypes = [_vp, ctypes.POINTER(emtk_request), ctypes.c_int32, _vp]
    lib.emtk_extract_patches.argtypes = [_vp, _vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, _vp,
                                         ctypes.c_int32, _vp, ctypes.c_int, _vp]
    lib.emtk_infer_patches.argtypes = [_vp, _vp, ctypes.c_int32, _vp, _vp]
    lib.emtk_check.argtypes = [_vp, _vp]
    lib.emtk_get_stats.argtypes = [_vp, ctypes.POINTER(emtk_stats)]
    lib.emtk_extract_patches_static.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, _vp,
                                                ctypes.c_int32, _vp, ctypes.c_int, _vp]
    lib.emtk_extract_patches_static.restype = ctypes.c_int
    lib.emtk_batcher_create.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, ctypes.POINTER(_vp)]
    lib.emtk_batcher_submit.argtypes = [_vp, ctypes.POINTER(emtk_request), ctypes.POINTER(ctypes.c_uint64)]
    lib.emtk_batcher_wait.argtypes = [_vp, ctypes.c_uint64, ctypes.c_int64]
    lib.emtk_batcher_stats.argtypes = [_vp, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64),
                                       ctypes.POINTER(ctypes.c_int64)]
    lib.emtk_batcher_destroy.argtypes = [_vp]
    lib.emtk_get_fp8_scales.argtypes = [_vp, _fp, _fp]
    lib.emtk_get_fp8_scales.restype = ctypes.c_int
    lib.emtk_find_hits.argtypes = [_vp, ctypes.POINTER(emtk_hitfind_request), ctypes.c_int32, _vp]
    lib.emtk_infer_batch_host.argtypes = [_vp, ctypes.POINTER(emtk_request), ctypes.c_int32, _vp]
    lib.emtk_infer_batch_host.restype = ctypes.c_int
    lib.emtk_find_hits.restype = ctypes.c_int
    lib.emtk_debug_fail_alloc.argtypes = [ctypes.c_int64]
    lib.emtk_debug_fail_alloc.restype = None
    lib.emtk_debug_alloc_counts.argtypes = [ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
    lib.emtk_debug_alloc_counts.restype = None
    lib.emtk_debug_batcher_stall.argtypes = [_vp, ctypes.c_int32]
    lib.emtk_debug_batcher_stall.restype = ctypes.c_int
    for name in ("emtk_batcher_create", "emtk_batcher_submit", "emtk_batcher_wait", "emtk_batcher_stats",
                 "emtk_batcher_destroy"):
        getattr(lib, name).restype = ctypes.c_int
    lib.emtk_nn_create.argtypes = [ctypes.c_int, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(_vp)]
    lib.emtk_nn_destroy.argtypes = [_vp]
    lib.emtk_nn_check.argtypes = [_vp, _vp]
    packed = ("emtk_dense", "emtk_dense_backward", "emtk_gated", "emtk_gated_backward", "emtk_residual_norm",
              "emtk_residual_norm_backward", "emtk_logprobs", "emtk_logprobs_backward", "emtk_recurrence",
              "emtk_recurrence_backward")
    for name in packed:
        getattr(lib, name).argtypes = [_vp, ctypes.c_char_p, _vp]  # a packed argument struct
    for name in ("emtk_pack8", "emtk_unpack8"):
        getattr(lib, name).argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int, ctypes.c_char_p,
                                       ctypes.c_char_p, _vp]
    lib.emtk_dropout.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int, ctypes.c_char_p, ctypes.c_char_p,
                                 ctypes.c_char_p, _vp]
    for name in packed + ("emtk_nn_create", "emtk_nn_destroy", "emtk_nn_check", "emtk_pack8", "emtk_unpack8", "emtk_dropout"):
        getattr(lib, name).restype = ctypes.c_int
    lib.emtk_status_string.argtypes = [ctypes.c_int]
    lib.emtk_status_string.restype = ctypes.c_char_p
    for name in ("emtk_create", "emtk_destroy", "emtk_infer", "emtk_infer_batch", "emtk_extract_patches",
                 "emtk_infer_patches", "emtk_check", "emtk_get_stats"):
        getattr(lib, name).restype = ctypes.c_int
    if path is None:
        _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().emtk_status_string(int(status)).decode()


def emtk_status_string(status: int) -> str:
    return status_string(status)


def _check(rc: int, what: str) -> int:
    if rc != EMTK_OK:
        raise EmtkError(rc, what)
    return rc


def _ptr(t) -> int:
    """Device pointer of a torch tensor (or a raw int)."""
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _stream(stream) -> int:
    import torch
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def emtk_default_options() -> emtk_options:
    o = emtk_options()
    load_library().emtk_default_options(ctypes.byref(o))
    return o


def emtk_create(weights: dict, precision: str = "bf16", device: int = 0, max_hits: int | None = None,
                debug_logits: bool = False, wait_timeout_ns: int | None = None, debug_stall: bool = False,
                profile: bool = False):
    """Creates a context from host fp32 weights (a dict of numpy arrays in the
    layouts of include/emtk.h).  Returns an opaque handle (int)."""
    lib = load_library()
    keep = {k: np.ascontiguousarray(weights[k], dtype=np.float32) for k, _ in emtk_weights._fields_}
    w = emtk_weights(**{k: v.ctypes.data_as(_fp) for k, v in keep.items()})
    o = emtk_default_options()
    o.precision = PRECISIONS[precision] if isinstance(precision, str) else int(precision)
    if max_hits is not None:
        o.max_hits = int(max_hits)
    o.debug_logits = int(bool(debug_logits))
    if wait_timeout_ns is not None:
        o.wait_timeout_ns = int(wait_timeout_ns)
    o.debug_stall = int(bool(debug_stall))
    o.profile = int(bool(profile))
    h = _vp()
    _check(lib.emtk_create(ctypes.byref(w), ctypes.byref(o), int(device), ctypes.byref(h)), "emtk_create")
    return h.value


def emtk_destroy(ctx) -> None:
    _check(load_library().emtk_destroy(ctx), "emtk_destroy")


def emtk_infer(ctx, adc, nticks: int, hits, scores, stream=None) -> None:
    """adc: float32 [nwires][ld] CUDA tensor; hits: int32 [n][2]; scores:
    float32 [n][4] (or [n][8] with debug logits)."""
    nwires, ld = adc.shape
    _check(load_library().emtk_infer(ctx, _ptr(adc), int(nwires), int(nticks), int(ld), _ptr(hits),
                                     int(hits.shape[0]), _ptr(scores), _stream(stream)), "emtk_infer")


def make_requests(items) -> ctypes.Array:
    """items: iterable of (adc, nticks, hits, scores) tensors."""
    items = list(items)
    arr = (emtk_request * max(1, len(items)))()
    for i, (adc, nticks, hits, scores) in enumerate(items):
        arr[i] = emtk_request(_ptr(adc), int(adc.shape[0]), int(nticks), int(adc.shape[1]), _ptr(hits),
                              int(hits.shape[0]), _ptr(scores))
    return arr


def emtk_infer_batch(ctx, items, stream=None) -> None:
    items = list(items)
    reqs = make_requests(items)
    _check(load_library().emtk_infer_batch(ctx, reqs, len(items), _stream(stream)), "emtk_infer_batch")


def emtk_infer_batch_host(ctx, items, stream=None) -> None:
    """emtk_infer_batch with host (CPU) tensors: (adc, nticks, hits, scores) per
    request.  Returns once the work is enqueued; the scores are final when the
    stream has completed, and the tensors must stay alive until then."""
    items = list(items)
    reqs = make_requests(items)
    _check(load_library().emtk_infer_batch_host(ctx, reqs, len(items), _stream(stream)), "emtk_infer_batch_host")


def emtk_extract_patches(ctx, adc, nticks: int, hits, patches, fmt: str = "f32", stream=None) -> None:
    nwires, ld = adc.shape
    _check(load_library().emtk_extract_patches(ctx, _ptr(adc), int(nwires), int(nticks), int(ld), _ptr(hits),
                                               int(hits.shape[0]), _ptr(patches), PATCH_FORMATS[fmt],
                                               _stream(stream)), "emtk_extract_patches")


def emtk_extract_patches_static(adc, nticks: int, hits, patches, fmt: str = "f32", stream=None) -> None:
    """The patch cut without a context and without any device allocation, for
    callers that cannot allocate; its scratch is a fixed 4 MiB array in the
    library (see include/emtk.h for the size limit and the sharing rules)."""
    nwires, ld = adc.shape
    _check(load_library().emtk_extract_patches_static(_ptr(adc), int(nwires), int(nticks), int(ld), _ptr(hits),
                                                      int(hits.shape[0]), _ptr(patches), PATCH_FORMATS[fmt],
                                                      _stream(stream)), "emtk_extract_patches_static")


def emtk_infer_patches(ctx, patches, scores, stream=None) -> None:
    _check(load_library().emtk_infer_patches(ctx, _ptr(patches), int(patches.shape[0]), _ptr(scores),
                                             _stream(stream)), "emtk_infer_patches")


def emtk_check(ctx, stream=None) -> int:
    """Returns the status code (does not raise on EMTK_ERR_TIMEOUT)."""
    return int(load_library().emtk_check(ctx, _stream(stream)))


def emtk_get_stats(ctx) -> dict:
    s = emtk_stats()
    _check(load_library().emtk_get_stats(ctx, ctypes.byref(s)), "emtk_get_stats")
    return dict(calls=s.calls, hits=s.hits, launches=s.launches, chunks=s.chunks, batch_hist=list(s.batch_hist),
                kernel_launches=dict(zip(KERNELS, s.kernel_launches)), kernel_ms=dict(zip(KERNELS, s.kernel_ms)))


def emtk_find_hits(ctx, planes, stream=None) -> list:
    """Hit finding (see include/emtk.h) on several planes in one call.
    ``planes``: list of (adc [nwires][ld] float32 device tensor, nticks, threshold,
    hits [capacity][2] int32 device tensor, info [capacity][4] int32 device tensor
    or None).  info columns: start, end, then peak and charge as float32 bits
    (``info[:, 2:].view(torch.float32)``).  Returns the number of hits found per
    plane (which may exceed a plane's capacity); the call synchronises the stream."""
    reqs = (emtk_hitfind_request * max(1, len(planes)))()
    for i, (adc, nticks, thr, hits, info) in enumerate(planes):
        q = reqs[i]
        q.d_adc = _ptr(adc)
        q.nwires, q.ld = adc.shape
        q.nticks = int(nticks)
        q.threshold = float(thr)
        q.capacity = hits.shape[0]
        q.d_hits = _ptr(hits)
        q.d_info = _ptr(info) if info is not None else None
    _check(load_library().emtk_find_hits(ctx, reqs, len(planes), _stream(stream)), "emtk_find_hits")
    return [int(reqs[i].n_found) for i in range(len(planes))]


def emtk_get_fp8_scales(ctx) -> tuple:
    """(s_a, s_w): the dense-1 operand scales of an "fp8" context, (1, 1) otherwise."""
    a, w = ctypes.c_float(), ctypes.c_float()
    _check(load_library().emtk_get_fp8_scales(ctx, ctypes.byref(a), ctypes.byref(w)), "emtk_get_fp8_scales")
    return float(a.value), float(w.value)


# ------------------------------------------------------------------ batcher
def emtk_batcher_create(ctx, nstreams: int = 4, max_hits: int = 65536, max_delay_us: int = 200):
    """Request batcher over `ctx` (see include/emtk.h).  Returns a handle (int)."""
    out = _vp()
    _check(load_library().emtk_batcher_create(ctx, int(nstreams), int(max_hits), int(max_delay_us),
                                              ctypes.byref(out)), "emtk_batcher_create")
    return out.value


# (batcher, ticket) -> the request's tensors.  The batcher reads and writes them on its
# own streams after submit returns; holding them here until the ticket is waited for (or
# the batcher destroyed) keeps torch from freeing and reusing their memory meanwhile.
_batcher_refs = {}


def emtk_batcher_submit(b, adc, nticks: int, hits, scores) -> int:
    """Queues one request (a plane, its hits and its output); returns its ticket.  The tensors
    must stay unchanged until emtk_batcher_wait has returned for the ticket; this binding
    keeps them alive until then."""
    req = make_requests([(adc, nticks, hits, scores)])
    t = ctypes.c_uint64()
    _check(load_library().emtk_batcher_submit(b, req, ctypes.byref(t)), "emtk_batcher_submit")
    _batcher_refs[(b, t.value)] = (adc, hits, scores)
    return t.value


def emtk_batcher_wait(b, ticket: int, timeout_ms: int = -1) -> int:
    """Blocks until the ticket's scores are complete; returns the status (EMTK_ERR_TIMEOUT when
    timeout_ms ran out first, without consuming the ticket)."""
    rc = load_library().emtk_batcher_wait(b, int(ticket), int(timeout_ms))
    if rc != EMTK_ERR_TIMEOUT:  # the ticket is done with (or was never issued)
        _batcher_refs.pop((b, int(ticket)), None)
    return rc


def emtk_batcher_stats(b) -> dict:
    n = [ctypes.c_int64() for _ in range(3)]
    _check(load_library().emtk_batcher_stats(b, *[ctypes.byref(x) for x in n]), "emtk_batcher_stats")
    return dict(batches=n[0].value, requests=n[1].value, hits=n[2].value)


def emtk_batcher_destroy(b) -> None:
    _check(load_library().emtk_batcher_destroy(b), "emtk_batcher_destroy")
    for key in [k for k in _batcher_refs if k[0] == b]:
        del _batcher_refs[key]


# ------------------------------------------- dense, gated, 8-bit checkpoints
class Q8(NamedTuple):
    """An 8-bit checkpoint of a matrix [m][k] (emtk_matrix in include/emtk.h): int8
    codes [m][k] and uint8 scales [m][ceil(k / 32)], CUDA tensors with unit column
    stride.  Where an argument below is a matrix that may be kept in 8 bits, it is
    either a 16-bit tensor or a Q8."""
    codes: "object"
    scales: "object"


def emtk_q8_empty(m: int, k: int, device="cuda") -> Q8:
    """An 8-bit checkpoint's tensors for an [m][k] matrix, contents undefined."""
    import torch
    return Q8(torch.empty((m, k), dtype=torch.int8, device=device),
              torch.empty((m, (k + 31) // 32), dtype=torch.uint8, device=device))


# The argument structs of include/emtk.h as bytes: packing one takes a fraction of
# filling a ctypes.Structure, and a call for one row is short.
_MATRIX = "QqQq"
_PACK_MATRIX = struct.Struct("<" + _MATRIX)
_PACK_DENSE = struct.Struct("<6i" + 5 * _MATRIX + "Q")
_PACK_DENSE_GRAD = struct.Struct("<6i" + 6 * _MATRIX + "Q")
_PACK_GATED = struct.Struct("<6i" + 6 * _MATRIX + "2Q")
_PACK_GATED_GRAD = struct.Struct("<6i" + 10 * _MATRIX + "2Q")
_ABSENT = (0, 0, 0, 0)
_TYPES = {}  # torch dtype -> emtk_type
_F32 = _I32 = None  # torch's float32 and int32, once torch is here


def _load_types() -> None:
    global _F32, _I32
    import torch
    _TYPES.update({torch.bfloat16: EMTK_TYPE_BF16, torch.float16: EMTK_TYPE_F16, torch.float32: EMTK_TYPE_F32})
    _F32, _I32 = torch.float32, torch.int32


def _type_of(t, what: str, f32: bool = False) -> int:
    if not _TYPES:
        _load_types()
    v = _TYPES.get(t.dtype, -1)
    if v < 0 or (v == EMTK_TYPE_F32 and not f32):
        raise ValueError(f"{what}: dtype {t.dtype} is not supported")
    return v


def _mat(on, t, rows: int, cols: int, dtype, what: str) -> tuple:
    """(d, ld, d_scale, ld_scale) of a [rows][cols] tensor of dtype on CUDA device `on`; absent for None."""
    if t is None:
        return _ABSENT
    if t.dtype is dtype and t.shape == (rows, cols) and t.get_device() == on:
        ld, unit = t.stride()
        if unit == 1 and ld >= cols:
            return (t.data_ptr(), ld, 0, 0)
        if (unit == 1 or cols <= 1) and (ld >= cols or rows <= 1):
            return (t.data_ptr(), max(ld, cols), 0, 0)  # one row or column: its stride says nothing
        raise ValueError(f"{what}: strides {t.stride()}: a row's elements must be neighbours and rows apart")
    raise ValueError(f"{what}: expected a tensor {(rows, cols)} of {dtype} on CUDA device {on}, got {tuple(t.shape)} of {t.dtype} on {t.device}")


def _mat8(on, t, rows: int, cols: int, dtype, what: str) -> tuple:
    """_mat of a tensor that may be a Q8."""
    if not isinstance(t, Q8):
        return _mat(on, t, rows, cols, dtype, what)
    import torch
    d, ld, _, _ = _mat(on, t.codes, rows, cols, torch.int8, what)
    s, lds, _, _ = _mat(on, t.scales, rows, (cols + 31) // 32, torch.uint8, what)
    return (d, ld, s, lds)


def _vec(on, t, n: int, what: str, f32: bool = False) -> int:
    if t is None:
        return 0
    if t.shape != (n,) or t.get_device() != on or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: expected a contiguous vector of {n} on CUDA device {on}, got {tuple(t.shape)} on {t.device}")
    if f32 and _type_of(t, what, True) != EMTK_TYPE_F32:
        raise ValueError(f"{what}: dtype {t.dtype}, expected float32")
    return t.data_ptr()


_raw_stream = None


def _current(t, stream) -> int:
    """The stream argument, or the current stream of t's device."""
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            import torch
            _raw_stream = torch._C._cuda_getCurrentRawStream  # torch.cuda.current_stream() without its object
        return _raw_stream(t.get_device())
    return _stream(stream)


_nn_devices = {}  # layer handle -> its device


def _device_of(nn, t) -> int:
    """The device that a call's tensors must be on: the handle's (of a handle made elsewhere, t's)."""
    device = _nn_devices.get(nn)
    if device is None:
        device = t.get_device()
        if device < 0:
            raise ValueError(f"expected CUDA tensors, got one on {t.device}")
    return device


def _act_code(act: str) -> int:
    if act not in ACTS:
        raise ValueError(f"act: {act!r} is none of {tuple(ACTS)}")
    return ACTS[act]


def emtk_nn_create(device: int = 0, workspace_bytes: int = 0, wait_timeout_ns: int = 2_000_000_000,
                   debug_stall: bool = False):
    """A layer handle (see include/emtk.h), an int.  The tensors of its calls are on ``device``."""
    out = _vp()
    _check(load_library().emtk_nn_create(int(device), int(workspace_bytes), int(wait_timeout_ns),
                                         int(bool(debug_stall)), ctypes.byref(out)), "emtk_nn_create")
    _nn_devices[out.value] = int(device)
    return out.value


def emtk_nn_destroy(nn) -> None:
    _nn_devices.pop(nn, None)
    _check(load_library().emtk_nn_destroy(nn), "emtk_nn_destroy")


def emtk_nn_check(nn, stream=None) -> int:
    """Returns the status code (does not raise on EMTK_ERR_TIMEOUT)."""
    return int(load_library().emtk_nn_check(nn, _stream(stream)))


def emtk_dense(nn, x, w, y, bias=None, act: str = "none", residual=None, pre=None, stream=None) -> None:
    """y = act(x w^T + bias) + residual.  x [m][k], w [n][k], y and residual [m][n]: bf16 or fp16 tensors of
    one dtype, rows any distance apart; bias [n] of that dtype or float32; pre [m][n] (tensor or Q8) receives
    the activation's input for emtk_dense_backward."""
    (m, k), n = x.shape, w.shape[0]
    dt = x.dtype
    on = _device_of(nn, x)
    args = _PACK_DENSE.pack(m, n, k, _act_code(act), _type_of(x, "x"),
                            0 if bias is None else _type_of(bias, "bias", True),
                            *_mat(on, x, m, k, dt, "x"), *_mat(on, w, n, k, dt, "w"), *_mat(on, y, m, n, dt, "y"),
                            *_mat(on, residual, m, n, dt, "residual"), *_mat8(on, pre, m, n, dt, "pre"),
                            _vec(on, bias, n, "bias"))
    _check(load_library().emtk_dense(nn, args, _current(x, stream)), "emtk_dense")


def emtk_dense_backward(nn, dy, x, w, act: str = "none", pre=None, dx=None, dw=None, db=None, stream=None) -> None:
    """Gradients of emtk_dense from dy [m][n]: dx [m][k], dw [n][k] (x's dtype or float32), db [n] float32,
    each optional.  x and pre may be Q8; x may be None without dw, w None without dx."""
    (m, n), dt = dy.shape, dy.dtype
    on = _device_of(nn, dy)
    like = w if w is not None else dw if dw is not None else x.codes if isinstance(x, Q8) else x
    k = 0 if like is None else like.shape[1]
    args = _PACK_DENSE_GRAD.pack(m, n, k, _act_code(act), _type_of(dy, "dy"),
                                 0 if dw is None else _type_of(dw, "dw", True),
                                 *_mat(on, dy, m, n, dt, "dy"), *_mat8(on, x, m, k, dt, "x"), *_mat(on, w, n, k, dt, "w"),
                                 *_mat8(on, pre, m, n, dt, "pre"), *_mat(on, dx, m, k, dt, "dx"),
                                 *_mat(on, dw, n, k, None if dw is None else dw.dtype, "dw"),
                                 _vec(on, db, n, "db", True))
    _check(load_library().emtk_dense_backward(nn, args, _current(dy, stream)), "emtk_dense_backward")


def emtk_gated(nn, x, w_gate, w_up, h, bias_gate=None, bias_up=None, act: str = "silu", gate=None, up=None,
               stream=None) -> None:
    """h = act(x w_gate^T + bias_gate) * (x w_up^T + bias_up): x [m][k], weights [f][k], h [m][f]; gate and up
    [m][f] (tensors or Q8s) receive the two factors' inputs for emtk_gated_backward."""
    (m, k), f = x.shape, w_gate.shape[0]
    dt = x.dtype
    on = _device_of(nn, x)
    bias_type = 0 if bias_gate is None else _type_of(bias_gate, "bias_gate", True)
    if bias_gate is not None and bias_up is not None and bias_gate.dtype is not bias_up.dtype:
        raise ValueError("bias_up: its dtype must be bias_gate's")
    args = _PACK_GATED.pack(m, f, k, _act_code(act), _type_of(x, "x"), bias_type,
                            *_mat(on, x, m, k, dt, "x"), *_mat(on, w_gate, f, k, dt, "w_gate"), *_mat(on, w_up, f, k, dt, "w_up"),
                            *_mat(on, h, m, f, dt, "h"), *_mat8(on, gate, m, f, dt, "gate"),
                            *_mat8(on, up, m, f, dt, "up"), _vec(on, bias_gate, f, "bias_gate"),
                            _vec(on, bias_up, f, "bias_up"))
    _check(load_library().emtk_gated(nn, args, _current(x, stream)), "emtk_gated")


def emtk_gated_backward(nn, dh, gate, up, x, w_gate, w_up, act: str = "silu", dx=None, dw_gate=None, dw_up=None,
                        db_gate=None, db_up=None, h=None, stream=None) -> None:
    """Gradients of emtk_gated from dh [m][f] and the gate and up it kept: dx [m][k], dw_gate and dw_up [f][k]
    (x's dtype or float32), db_gate and db_up [f] float32, and h [m][f] once more; each optional."""
    (m, f), dt = dh.shape, dh.dtype
    on = _device_of(nn, dh)
    like = w_gate if w_gate is not None else dw_gate if dw_gate is not None else x.codes if isinstance(x, Q8) else x
    k = 0 if like is None else like.shape[1]
    if dw_gate is not None and dw_up is not None and dw_gate.dtype is not dw_up.dtype:
        raise ValueError("dw_up: its dtype must be dw_gate's")
    dwt = None if dw_gate is None else dw_gate.dtype
    args = _PACK_GATED_GRAD.pack(m, f, k, _act_code(act), _type_of(dh, "dh"),
                                 0 if dw_gate is None else _type_of(dw_gate, "dw_gate", True),
                                 *_mat(on, dh, m, f, dt, "dh"), *_mat8(on, gate, m, f, dt, "gate"),
                                 *_mat8(on, up, m, f, dt, "up"), *_mat8(on, x, m, k, dt, "x"),
                                 *_mat(on, w_gate, f, k, dt, "w_gate"), *_mat(on, w_up, f, k, dt, "w_up"),
                                 *_mat(on, dx, m, k, dt, "dx"), *_mat(on, dw_gate, f, k, dwt, "dw_gate"),
                                 *_mat(on, dw_up, f, k, dwt, "dw_up"), *_mat(on, h, m, f, dt, "h"),
                                 _vec(on, db_gate, f, "db_gate", True), _vec(on, db_up, f, "db_up", True))
    _check(load_library().emtk_gated_backward(nn, args, _current(dh, stream)), "emtk_gated_backward")


def emtk_pack8(nn, x, q: Q8, stream=None) -> None:
    """Keeps x [m][k] (bf16 or fp16) in the 8-bit checkpoint q."""
    (m, k), dt = x.shape, x.dtype
    on = _device_of(nn, x)
    _check(load_library().emtk_pack8(nn, m, k, _type_of(x, "x"), _PACK_MATRIX.pack(*_mat(on, x, m, k, dt, "x")),
                                     _PACK_MATRIX.pack(*_mat8(on, q, m, k, dt, "q")), _current(x, stream)), "emtk_pack8")


def emtk_unpack8(nn, q: Q8, x, stream=None) -> None:
    """The values that the 8-bit checkpoint q stands for, into x [m][k] (bf16 or fp16)."""
    (m, k), dt = x.shape, x.dtype
    on = _device_of(nn, x)
    _check(load_library().emtk_unpack8(nn, m, k, _type_of(x, "x"), _PACK_MATRIX.pack(*_mat8(on, q, m, k, dt, "q")),
                                       _PACK_MATRIX.pack(*_mat(on, x, m, k, dt, "x")), _current(x, stream)), "emtk_unpack8")


# ------------------- residual norms, dropout, log probabilities, recurrence
class Drop(NamedTuple):
    """Dropout (emtk_drop in include/emtk.h): the share dropped, and what the random numbers are made of.  The
    backward pass takes the same one.  ``offset_tensor``: a CUDA tensor of one int64 that is added to ``offset``
    on the device, so that a captured call takes other numbers at each replay."""
    p: float
    seed: int
    offset: int = 0
    offset_tensor: "object" = None


class Norm(NamedTuple):
    """A norm over a row (emtk_norm in include/emtk.h): "rms" or "layer", its weight and bias (vectors of the
    call's dtype or float32, or None for 1 and 0) and the eps beside the variance."""
    kind: str
    weight: "object" = None
    bias: "object" = None
    eps: float = 1e-6


_NORM, _DROP = "iif4xQQ", "QQQf4x"
_PACK_DROP = struct.Struct("<" + _DROP)
_PACK_SEAM = struct.Struct("<4if4x" + 2 * _NORM + _DROP + 5 * _MATRIX)
_PACK_SEAM_GRAD = struct.Struct("<4if4x" + 2 * _NORM + _DROP + 8 * _MATRIX + "4Q")
_PACK_LOGPROBS = struct.Struct("<4if4x" + _MATRIX + "6Q")
_PACK_LOGPROBS_GRAD = struct.Struct("<3i4xf4x" + 2 * _MATRIX + "5Q")
_PACK_RECURRENCE = struct.Struct("<5i4x" + 4 * _MATRIX + "4Q")
_PACK_RECURRENCE_GRAD = struct.Struct("<5i4x" + 7 * _MATRIX + "4Q")
_NO_NORM = (0, 0, 0.0, 0, 0)
_NO_DROP = (0, 0, 0, 0.0)
_WORD = (1 << 64) - 1


def _drop(on, d) -> tuple:
    """The fields of emtk_drop; absent for None."""
    if d is None:
        return _NO_DROP
    p, seed, offset, t = d
    if t is not None:
        import torch
        if t.dtype is not torch.int64 or t.numel() != 1 or t.get_device() != on:
            raise ValueError(f"offset_tensor: expected one int64 on CUDA device {on}, got {tuple(t.shape)} of {t.dtype} on {t.device}")
        t = t.data_ptr()
    return (seed & _WORD, offset & _WORD, t or 0, p)


def _norm(on, v, n: int, what: str) -> tuple:
    """The fields of emtk_norm; absent for None."""
    if v is None:
        return _NO_NORM
    kind, weight, bias, eps = v
    code = NORMS.get(kind, 0)
    if not code:
        raise ValueError(f"{what}: {kind!r} is none of {tuple(NORMS)[1:]}")
    if bias is None:
        if weight is None:
            return (code, 0, eps, 0, 0)
        return (code, _type_of(weight, what, True), eps, _vec(on, weight, n, what), 0)
    if weight is not None and weight.dtype is not bias.dtype:
        raise ValueError(f"{what}: its bias' dtype must be its weight's")
    return (code, _type_of(bias, what, True), eps, _vec(on, weight, n, what), _vec(on, bias, n, what))


def _whole(on, t, shape: tuple, dtype, what: str) -> int:
    """A contiguous tensor of a shape and dtype on CUDA device `on`; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != on or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor {shape} of {dtype} on CUDA device {on}, got {tuple(t.shape)} of "
                         f"{t.dtype} on {t.device}")
    return t.data_ptr()


def _gate(on, gate, m: int, n: int, every, dtype, what: str) -> tuple:
    """(matrix, rows to a gate row) of a gate: [n], one row for all, or [ceil(m / every)][n]."""
    every = max(1, m) if every is None else int(every)
    if gate is None:
        return _ABSENT, every
    if gate.dim() == 1:
        gate = gate[None]
    if every <= 0:
        raise ValueError(f"gate_every: {every} is not positive")
    return _mat(on, gate, max(1, -(-m // every)), n, dtype, what), every


def emtk_dropout(nn, x, y, drop: Drop, stream=None) -> None:
    """y = x under dropout, [m][n] of bf16 or fp16; dx from dy is the same call.  y may be x."""
    (m, n), dt = x.shape, x.dtype
    on = _device_of(nn, x)
    _check(load_library().emtk_dropout(nn, m, n, _type_of(x, "x"), _PACK_MATRIX.pack(*_mat(on, x, m, n, dt, "x")),
                                       _PACK_MATRIX.pack(*_mat(on, y, m, n, dt, "y")), _PACK_DROP.pack(*_drop(on, drop)),
                                       _current(x, stream)), "emtk_dropout")


def emtk_residual_norm(nn, residual=None, block=None, y=None, h=None, post: Norm = None, pre: Norm = None, gate=None,
                       gate_every: int = None, scale: float = 1.0, drop: Drop = None, stream=None) -> None:
    """y = scale * residual + gate * dropout(post(block)) and h = pre(y), [m][n] of bf16 or fp16, n <= 16384, each part
    optional.  gate: [n], or [ceil(m / gate_every)][n] with row i taking row i // gate_every.  y may be residual."""
    like = block if block is not None else residual
    if like is None:
        raise ValueError("residual, block: one must be given")
    (m, n), dt = like.shape, like.dtype
    on = _device_of(nn, like)
    g, every = _gate(on, gate, m, n, gate_every, dt, "gate")
    args = _PACK_SEAM.pack(m, n, _type_of(like, "block" if like is block else "residual"), every, scale, *_norm(on, post, n, "post"),
                           *_norm(on, pre, n, "pre"), *_drop(on, drop), *_mat(on, residual, m, n, dt, "residual"),
                           *_mat(on, block, m, n, dt, "block"), *g, *_mat(on, y, m, n, dt, "y"), *_mat(on, h, m, n, dt, "h"))
    _check(load_library().emtk_residual_norm(nn, args, _current(like, stream)), "emtk_residual_norm")


def emtk_residual_norm_backward(nn, dy=None, dh=None, y=None, block=None, d_residual=None, d_block=None, post: Norm = None,
                                pre: Norm = None, gate=None, gate_every: int = None, scale: float = 1.0, drop: Drop = None,
                                d_gate=None, dw_pre=None, db_pre=None, dw_post=None, db_post=None, stream=None) -> None:
    """Gradients of emtk_residual_norm from dy (of y's other uses) and dh, with the y that it wrote: d_residual and
    d_block [m][n], d_gate (gate's shape), dw_pre, db_pre, dw_post, db_post [n] float32; each optional.  d_residual may
    be dy."""
    like = dh if dh is not None else dy
    if like is None:
        raise ValueError("dy, dh: one must be given")
    (m, n), dt = like.shape, like.dtype
    on, code = _device_of(nn, like), _type_of(like, "dh" if like is dh else "dy")
    g, every = _gate(on, gate, m, n, gate_every, dt, "gate")
    dg, _ = _gate(on, d_gate, m, n, gate_every, _F32, "d_gate")
    args = _PACK_SEAM_GRAD.pack(m, n, code, every, scale, *_norm(on, post, n, "post"),
                                *_norm(on, pre, n, "pre"), *_drop(on, drop), *_mat(on, dy, m, n, dt, "dy"),
                                *_mat(on, dh, m, n, dt, "dh"), *_mat(on, y, m, n, dt, "y"), *_mat(on, block, m, n, dt, "block"), *g,
                                *_mat(on, d_residual, m, n, dt, "d_residual"), *_mat(on, d_block, m, n, dt, "d_block"), *dg,
                                _vec(on, dw_pre, n, "dw_pre", True), _vec(on, db_pre, n, "db_pre", True),
                                _vec(on, dw_post, n, "dw_post", True), _vec(on, db_post, n, "db_post", True))
    _check(load_library().emtk_residual_norm_backward(nn, args, _current(like, stream)), "emtk_residual_norm_backward")


def emtk_logprobs(nn, logits, tokens=None, logprob=None, entropy=None, lse=None, top_logprob=None, top_index=None,
                  temperature: float = 1.0, stream=None) -> None:
    """Of logits [m][v] (bf16, fp16 or float32), float32 and contiguous, each optional: logprob [m] of tokens [m] (int32;
    negative: none), entropy [m], lse [m] for the backward call, top_logprob [m][top] and top_index [m][top] (int32) of
    the largest `top` <= 32."""
    (m, v), on, code = logits.shape, _device_of(nn, logits), _type_of(logits, "logits", True)
    some = top_logprob if top_logprob is not None else top_index
    top = 0 if some is None else some.shape[1]
    args = _PACK_LOGPROBS.pack(m, v, code, top, temperature, *_mat(on, logits, m, v, logits.dtype, "logits"),
                               _whole(on, tokens, (m,), _I32, "tokens"), _whole(on, logprob, (m,), _F32, "logprob"),
                               _whole(on, entropy, (m,), _F32, "entropy"), _whole(on, lse, (m,), _F32, "lse"),
                               _whole(on, top_logprob, (m, top), _F32, "top_logprob"), _whole(on, top_index, (m, top), _I32, "top_index"))
    _check(load_library().emtk_logprobs(nn, args, _current(logits, stream)), "emtk_logprobs")


def emtk_logprobs_backward(nn, logits, lse, d_logits, tokens=None, d_logprob=None, entropy=None, d_entropy=None,
                           temperature: float = 1.0, stream=None) -> None:
    """The gradient of logits, of their dtype, from d_logprob [m] (with the tokens) and d_entropy [m] (with the entropy
    that emtk_logprobs wrote), each optional, and its lse.  d_logits may be logits."""
    (m, v), dt, on, code = logits.shape, logits.dtype, _device_of(nn, logits), _type_of(logits, "logits", True)
    args = _PACK_LOGPROBS_GRAD.pack(m, v, code, temperature, *_mat(on, logits, m, v, dt, "logits"),
                                    *_mat(on, d_logits, m, v, dt, "d_logits"), _whole(on, tokens, (m,), _I32, "tokens"),
                                    _whole(on, lse, (m,), _F32, "lse"), _whole(on, entropy, (m,), _F32, "entropy"),
                                    _whole(on, d_logprob, (m,), _F32, "d_logprob"), _whole(on, d_entropy, (m,), _F32, "d_entropy"))
    _check(load_library().emtk_logprobs_backward(nn, args, _current(logits, stream)), "emtk_logprobs_backward")


def emtk_recurrence_states(rows: int, n: int, seqs: int, device="cuda"):
    """The tensor in which emtk_recurrence keeps what its backward call needs, contents undefined."""
    import torch
    return torch.empty((rows // EMTK_RECURRENCE_STEP + seqs, n), dtype=torch.float32, device=device)


def emtk_recurrence(nn, f, x, y, o=None, act: str = "none", seqs: int = 1, offsets=None, state=None, last=None, states=None,
                    stream=None) -> None:
    """h_t = h_(t-1) + (x_t - h_(t-1)) / (1 + exp(f_t)) along each sequence and y = act(o) h (y = h without o), [rows][n]
    of bf16 or fp16.  Sequences lie one after another: offsets [seqs + 1] (int32) says where, or each has rows / seqs
    rows.  state and last [seqs][n] float32: the states before and after (last may be state); states
    (emtk_recurrence_states) is for the backward call."""
    (rows, n), dt, on, code, seqs = f.shape, f.dtype, _device_of(nn, f), _type_of(f, "f"), int(seqs)
    args = _PACK_RECURRENCE.pack(rows, n, seqs, _act_code(act), code, *_mat(on, f, rows, n, dt, "f"),
                                 *_mat(on, x, rows, n, dt, "x"), *_mat(on, o, rows, n, dt, "o"), *_mat(on, y, rows, n, dt, "y"),
                                 _whole(on, offsets, (seqs + 1,), _I32, "offsets"), _whole(on, state, (seqs, n), _F32, "state"),
                                 _whole(on, last, (seqs, n), _F32, "last"),
                                 _whole(on, states, (rows // EMTK_RECURRENCE_STEP + seqs, n), _F32, "states"))
    _check(load_library().emtk_recurrence(nn, args, _current(f, stream)), "emtk_recurrence")


def emtk_recurrence_backward(nn, dy, f, x, states, df=None, dx=None, o=None, act: str = "none", seqs: int = 1, offsets=None,
                             d_last=None, d_o=None, d_state=None, stream=None) -> None:
    """Gradients of emtk_recurrence from dy and d_last [seqs][n] float32 (None: 0), with the states that it kept: df, dx,
    d_o [rows][n] and d_state [seqs][n] float32, each optional."""
    (rows, n), dt, on, code, seqs = f.shape, f.dtype, _device_of(nn, f), _type_of(f, "f"), int(seqs)
    args = _PACK_RECURRENCE_GRAD.pack(rows, n, seqs, _act_code(act), code, *_mat(on, dy, rows, n, dt, "dy"),
                                      *_mat(on, f, rows, n, dt, "f"), *_mat(on, x, rows, n, dt, "x"), *_mat(on, o, rows, n, dt, "o"),
                                      *_mat(on, df, rows, n, dt, "df"), *_mat(on, dx, rows, n, dt, "dx"),
                                      *_mat(on, d_o, rows, n, dt, "d_o"), _whole(on, offsets, (seqs + 1,), _I32, "offsets"),
                                      _whole(on, states, (rows // EMTK_RECURRENCE_STEP + seqs, n), _F32, "states"),
                                      _whole(on, d_last, (seqs, n), _F32, "d_last"), _whole(on, d_state, (seqs, n), _F32, "d_state"))
    _check(load_library().emtk_recurrence_backward(nn, args, _current(f, stream)), "emtk_recurrence_backward")


# ------------------------------------------------------------- test hooks
def emtk_debug_fail_alloc(after: int) -> None:
    """The allocation after ``after`` more successful ones fails, once (< 0 disarms)."""
    load_library().emtk_debug_fail_alloc(int(after))


def emtk_debug_alloc_counts() -> tuple:
    """(device, pinned host) allocations of the library alive now."""
    d, h = ctypes.c_int64(), ctypes.c_int64()
    load_library().emtk_debug_alloc_counts(ctypes.byref(d), ctypes.byref(h))
    return d.value, h.value


def emtk_debug_batcher_stall(b, stall: bool) -> None:
    _check(load_library().emtk_debug_batcher_stall(b, int(bool(stall))), "emtk_debug_batcher_stall")
