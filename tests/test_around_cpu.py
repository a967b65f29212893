"""Host-side checks, without a GPU, of the C ABI around the products (residual norms, dropout, log probabilities, the
gated recurrence): struct layouts, packed argument formats, refusals before the device is touched, tensors of another
device."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2009_04509_gb300 import emtk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKERS = dict(emtk_drop="_PACK_DROP", emtk_residual_norm_args="_PACK_SEAM", emtk_residual_norm_grad_args="_PACK_SEAM_GRAD",
               emtk_logprobs_args="_PACK_LOGPROBS", emtk_logprobs_grad_args="_PACK_LOGPROBS_GRAD",
               emtk_recurrence_args="_PACK_RECURRENCE", emtk_recurrence_grad_args="_PACK_RECURRENCE_GRAD")
STRUCTS = tuple(PACKERS) + ("emtk_norm",)


@pytest.fixture(scope="module")
def lib():
    from paper_2009_04509_gb300 import build
    build.build()
    return emtk.load_library()


def test_struct_layouts_match_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "emtk.h"', "int main(void) {"]
    for name in STRUCTS:
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        for f, _ in getattr(emtk, name)._fields_:
            lines.append(f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));')
    lines.append('printf("step %d\\n", EMTK_RECURRENCE_STEP);')
    lines.append("return 0; }")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    want = dict(line.split() for line in out.splitlines())
    for name in STRUCTS:
        st = getattr(emtk, name)
        assert ctypes.sizeof(st) == int(want[name]), name
        for f, _ in st._fields_:
            assert getattr(st, f).offset == int(want[f"{name}.{f}"]), f"{name}.{f}"
    assert int(want["step"]) == emtk.EMTK_RECURRENCE_STEP


def _values(st):
    """A struct's values in order, its padding fields left out."""
    out = []
    for f, kind in st._fields_:
        if f.startswith("reserved"):
            continue
        v = getattr(st, f)
        out += _values(v) if isinstance(v, ctypes.Structure) else [v]
    return out


def test_packed_bytes_fill_the_structs():
    for name, packer in PACKERS.items():
        st, pack = getattr(emtk, name), getattr(emtk, packer)
        assert pack.size == ctypes.sizeof(st), name
        n = len(pack.unpack(bytes(pack.size)))
        assert _values(st.from_buffer_copy(pack.pack(*range(1, n + 1)))) == list(range(1, n + 1)), name


def test_generator_gives_the_published_numbers():
    """The tests' generator has the known answers that were published with Philox4x32-10."""
    pytest.importorskip("torch")
    from tests.test_gpu_around import philox
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert philox((0xffffffff,) * 4, (0xffffffff,) * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert philox((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) == \
        [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


@pytest.fixture
def handle(tmp_path):
    """A handle's bytes, all 0: its device is 0, and no call gets as far as using it."""
    return ctypes.create_string_buffer(256)


M = emtk._PACK_MATRIX.size
A = 1 << 20  # an address that nothing follows


def mat(d=A, ld=16):
    return (d, ld, 0, 0)


def seam(**c):
    d = dict(m=4, n=16, type=0, every=1, scale=1.0, post=emtk._NO_NORM, pre=(1, 0, 1e-6, 0, 0), drop=emtk._NO_DROP, residual=mat(A), block=mat(A + 4096),
             gate=(0, 0, 0, 0), y=mat(A + 8192), h=mat(A + 12288))
    d.update(c)
    return emtk._PACK_SEAM.pack(d["m"], d["n"], d["type"], d["every"], d["scale"], *d["post"], *d["pre"], *d["drop"], *d["residual"], *d["block"],
                                *d["gate"], *d["y"], *d["h"])


def seam_grad(**c):
    none = (0, 0, 0, 0)
    d = dict(m=4, n=16, type=0, every=1, scale=1.0, post=(2, 0, 1e-6, 0, 0), pre=(1, 0, 1e-6, 0, 0), drop=emtk._NO_DROP, dy=mat(A), dh=mat(A + 4096),
             y=mat(A + 8192), block=mat(A + 12288), gate=none, dr=mat(A + 16384), db=mat(A + 20480), dg=none, sums=(0, 0, 0, 0))
    d.update(c)
    return emtk._PACK_SEAM_GRAD.pack(d["m"], d["n"], d["type"], d["every"], d["scale"], *d["post"], *d["pre"], *d["drop"], *d["dy"], *d["dh"], *d["y"],
                                     *d["block"], *d["gate"], *d["dr"], *d["db"], *d["dg"], *d["sums"])


def logprobs(**c):
    d = dict(m=4, v=16, type=0, top=0, t=1.0, logits=mat(), tokens=A, logprob=A, entropy=0, lse=0, tl=0, ti=0)
    d.update(c)
    return emtk._PACK_LOGPROBS.pack(d["m"], d["v"], d["type"], d["top"], d["t"], *d["logits"], d["tokens"], d["logprob"], d["entropy"], d["lse"], d["tl"], d["ti"])


def logprobs_grad(**c):
    d = dict(m=4, v=16, type=0, t=1.0, logits=mat(), dz=mat(), tokens=A, lse=A, entropy=A, dl=A, dh=A)
    d.update(c)
    return emtk._PACK_LOGPROBS_GRAD.pack(d["m"], d["v"], d["type"], d["t"], *d["logits"], *d["dz"], d["tokens"], d["lse"], d["entropy"], d["dl"], d["dh"])


def recurrence(**c):
    d = dict(rows=4, n=16, seqs=2, act=0, type=0, f=mat(A), x=mat(A + 4096), o=(0, 0, 0, 0), y=mat(A + 8192), offsets=0, state=0, last=0, states=0)
    d.update(c)
    return emtk._PACK_RECURRENCE.pack(d["rows"], d["n"], d["seqs"], d["act"], d["type"], *d["f"], *d["x"], *d["o"], *d["y"], d["offsets"], d["state"], d["last"], d["states"])


def recurrence_grad(**c):
    none = (0, 0, 0, 0)
    d = dict(rows=4, n=16, seqs=2, act=0, type=0, dy=mat(A), f=mat(A + 4096), x=mat(A + 8192), o=none, df=mat(A + 12288), dx=none, do=none, offsets=0,
             states=A, dlast=0, dstate=0)
    d.update(c)
    return emtk._PACK_RECURRENCE_GRAD.pack(d["rows"], d["n"], d["seqs"], d["act"], d["type"], *d["dy"], *d["f"], *d["x"], *d["o"], *d["df"], *d["dx"], *d["do"],
                                           d["offsets"], d["states"], d["dlast"], d["dstate"])


NAN, INF = float("nan"), float("inf")
REFUSED = [
    ("emtk_residual_norm", seam, emtk.EMTK_ERR_ARG, [
        dict(m=-1), dict(n=-1), dict(n=16385, pre=emtk._NO_NORM, h=(0, 0, 0, 0)), dict(type=2), dict(type=9), dict(y=mat(A, 15)), dict(h=(0, 0, 0, 0)), dict(pre=emtk._NO_NORM),
        dict(pre=(3, 0, 1e-6, 0, 0)), dict(pre=(1, 0, -1.0, 0, 0)), dict(pre=(1, 0, NAN, 0, 0)), dict(pre=(1, 0, INF, 0, 0)), dict(pre=(1, 1, 1e-6, A, 0)),
        dict(pre=(0, 0, 0.0, A, 0), h=(0, 0, 0, 0)), dict(residual=(0, 0, 0, 0), block=(0, 0, 0, 0)), dict(block=(0, 0, 0, 0), post=(1, 0, 0.0, 0, 0)),
        dict(block=(0, 0, 0, 0), drop=(1, 0, 0, 0.5)), dict(drop=(1, 0, 0, 1.0)), dict(drop=(1, 0, 0, NAN)), dict(drop=(1, 0, 0, -0.5)),
        dict(gate=mat(A + 16384), every=0), dict(gate=mat(A + 16384), every=-3), dict(y=mat(A + 4096)), dict(h=mat(A + 8192)), dict(h=mat(A)), dict(y=mat(A, 24)),
        dict(residual=(A, 16, A, 1))]),
    ("emtk_residual_norm", seam, emtk.EMTK_ERR_ALIGN, [
        dict(y=mat(A + 8193)), dict(pre=(1, 2, 1e-6, A + 2, 0)), dict(pre=(1, 0, 1e-6, 0, A + 1)), dict(drop=(1, 0, A + 4, 0.5))]),
    ("emtk_residual_norm_backward", seam_grad, emtk.EMTK_ERR_ARG, [
        dict(m=-1), dict(n=16385), dict(type=2), dict(dh=(0, 0, 0, 0)), dict(pre=emtk._NO_NORM), dict(y=(0, 0, 0, 0)), dict(block=(0, 0, 0, 0)),
        dict(pre=emtk._NO_NORM, dh=(0, 0, 0, 0), sums=(A, 0, 0, 0)), dict(post=emtk._NO_NORM, sums=(0, 0, 0, A)), dict(dr=mat(A + 4096)), dict(db=mat(A)),
        dict(db=mat(A + 16384)), dict(dr=mat(A, 20)), dict(every=0, dg=mat(A + 65536)), dict(pre=emtk._NO_NORM, dh=(0, 0, 0, 0), dy=(0, 0, 0, 0))]),
    ("emtk_residual_norm_backward", seam_grad, emtk.EMTK_ERR_ALIGN, [dict(sums=(A + 2, 0, 0, 0)), dict(dg=mat(A + 2)), dict(dr=mat(A + 16385))]),
    ("emtk_logprobs", logprobs, emtk.EMTK_ERR_ARG, [
        dict(m=-1), dict(v=-1), dict(type=3), dict(top=-1, tl=A, ti=A), dict(top=33, v=64, logits=mat(A, 64), tl=A, ti=A), dict(top=17, tl=A, ti=A), dict(top=2), dict(top=2, tl=A),
        dict(tl=A, ti=A), dict(tokens=0), dict(logprob=0), dict(t=0.0), dict(t=-1.0), dict(t=NAN), dict(t=INF), dict(t=1e-45), dict(logits=mat(A, 15)), dict(logits=(0, 16, 0, 0))]),
    ("emtk_logprobs", logprobs, emtk.EMTK_ERR_ALIGN, [dict(type=2, logits=mat(A + 2)), dict(tokens=A + 2), dict(lse=A + 1)]),
    ("emtk_logprobs_backward", logprobs_grad, emtk.EMTK_ERR_ARG, [
        dict(m=-1), dict(type=3), dict(lse=0), dict(tokens=0), dict(entropy=0), dict(t=0.0), dict(dz=mat(A, 20)), dict(dz=(0, 0, 0, 0)), dict(logits=(0, 0, 0, 0))]),
    ("emtk_recurrence", recurrence, emtk.EMTK_ERR_ARG, [
        dict(rows=-1), dict(n=-1), dict(seqs=-1), dict(seqs=3), dict(seqs=0), dict(act=5), dict(act=1), dict(type=2), dict(f=(0, 0, 0, 0)), dict(y=mat(A)), dict(y=mat(A + 4096)),
        dict(x=mat(A, 15))]),
    ("emtk_recurrence", recurrence, emtk.EMTK_ERR_ALIGN, [dict(f=mat(A + 1)), dict(state=A + 2), dict(offsets=A + 1)]),
    ("emtk_recurrence_backward", recurrence_grad, emtk.EMTK_ERR_ARG, [
        dict(states=0), dict(seqs=3), dict(act=2), dict(do=mat(A + 65536)), dict(df=mat(A)), dict(df=mat(A + 4096)), dict(dx=mat(A + 12288)), dict(dy=(0, 0, 0, 0))]),
]


@pytest.mark.parametrize("entry", range(len(REFUSED)))
def test_refusals_without_device(lib, handle, entry):
    name, make, status, changes = REFUSED[entry]
    for change in changes:
        assert getattr(lib, name)(handle, make(**change), None) == status, change
    assert getattr(lib, name)(None, make(), None) == emtk.EMTK_ERR_ARG
    assert getattr(lib, name)(handle, None, None) == emtk.EMTK_ERR_ARG


@pytest.mark.parametrize("t", [2.9e-39, 4e-39, 4.23e-39, 0.0, -1e-3, NAN, INF])
def test_temperatures_too_small_to_scale_by_are_refused(lib, handle, t):
    """log2(e) / T, which logits are scaled by, is beyond fp32 from 4.24e-39 down: 0 times it would be NaN."""
    assert lib.emtk_logprobs(handle, logprobs(t=t), None) == emtk.EMTK_ERR_ARG
    assert lib.emtk_logprobs_backward(handle, logprobs_grad(t=t), None) == emtk.EMTK_ERR_ARG


def test_dropout_refusals_without_device(lib, handle):
    x, y = emtk._PACK_MATRIX.pack(*mat()), emtk._PACK_MATRIX.pack(*mat(A + 4096))
    drop = lambda p=0.5, t=0: emtk._PACK_DROP.pack(1, 2, t, p)  # noqa: E731
    call = lib.emtk_dropout
    for args, status in (((-1, 16, 0, x, y, drop()), emtk.EMTK_ERR_ARG), ((4, 16, 2, x, y, drop()), emtk.EMTK_ERR_ARG), ((4, 17, 0, x, y, drop()), emtk.EMTK_ERR_ARG),
                         ((4, 16, 0, x, y, drop(1.0)), emtk.EMTK_ERR_ARG), ((4, 16, 0, x, y, drop(NAN)), emtk.EMTK_ERR_ARG), ((4, 16, 0, None, y, drop()), emtk.EMTK_ERR_ARG),
                         ((4, 16, 0, x, y, None), emtk.EMTK_ERR_ARG), ((4, 16, 0, x, y, drop(0.5, A + 4)), emtk.EMTK_ERR_ALIGN),
                         ((4, 16, 0, x, emtk._PACK_MATRIX.pack(*mat(A, 20)), drop()), emtk.EMTK_ERR_ARG),
                         ((4, 16, 0, x, emtk._PACK_MATRIX.pack(*mat(A + 1)), drop()), emtk.EMTK_ERR_ALIGN)):
        assert call(handle, *args, None) == status
    assert call(None, 4, 16, 0, x, y, drop(), None) == emtk.EMTK_ERR_ARG


COPY_DRIVER = r"""
#include <cstdio>
#include "nn_internal.h"
int main() {
    using namespace emtk;
    static uint16_t room[256] __attribute__((aligned(16)));
    for (int shift = 0; shift < 8; ++shift)
        for (int ld : {16, 17}) {
            const Copy16 copy = {{room, 16, nullptr, 0}, {room + 128 + shift, ld, nullptr, 0}, 4, 16};
            if (shift == 0 && ld == 16) continue;  // a copy that there is
            const cudaError_t e = launch_copy16(EMTK_TYPE_BF16, &copy, 1, 1, nullptr);
            if (e != cudaErrorInvalidValue) return printf("%d elements off the grid, rows %d apart: %d\n", shift, ld, (int)e), 1;
        }
    return 0;
}
"""


def test_copies_of_16_bits_to_rows_off_the_grid_are_refused(lib, tmp_path):
    """Only a checkpoint is unpacked to rows off the 16-byte grid: that kernel reads the scales, which a 16-bit matrix has not.
    The library's own launcher, in a program without a GPU's memory: it is to refuse before it launches."""
    from paper_2009_04509_gb300 import build
    cuda, obj = os.environ.get("CUDA_HOME", "/usr/local/cuda"), os.path.join(build.BUILD, "nn_pointwise.o")
    if shutil.which("g++") is None or not os.path.exists(os.path.join(cuda, "include", "cuda.h")):
        pytest.skip("no g++ or CUDA headers")
    if not os.path.exists(obj):
        build.build(force=True)
    src, exe = tmp_path / "copy.cpp", tmp_path / "copy"
    src.write_text(COPY_DRIVER)
    subprocess.run(["g++", "-std=c++17", "-w", "-I", build.CSRC, "-I", os.path.join(cuda, "include"), str(src), obj, "-L", os.path.join(cuda, "lib64"),
                    "-lcudart_static", "-ldl", "-lrt", "-lpthread", "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


def test_binding_refuses_tensors_of_another_device(monkeypatch):
    """A tensor of another GPU than the handle's is refused before the library sees its address, each argument alone.
    Stand-ins for the tensors and the library: no GPU is needed."""
    torch = pytest.importorskip("torch")
    calls = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name == "emtk_nn_create":
                    args[-1]._obj.value = 8192 + args[0]
                calls.append(name)
                return 0
            return call

    class Tensor:
        is_cuda = True

        def __init__(self, *shape, dtype=torch.bfloat16, device=1):
            self.shape, self.dtype, self.device_index, self.device = shape, dtype, device, f"cuda:{device}"

        def get_device(self):
            return self.device_index

        def dim(self):
            return len(self.shape)

        def numel(self):
            out = 1
            for s in self.shape:
                out *= s
            return out

        def is_contiguous(self):
            return True

        def stride(self, i=None):
            s = (self.shape[-1], 1) if len(self.shape) == 2 else (1,)
            return s if i is None else s[i]

        def data_ptr(self):
            return 1 << 20

    monkeypatch.setattr(emtk, "load_library", lambda path=None: Library())
    m, n, f32, i32 = 4, 8, torch.float32, torch.int32
    T = Tensor
    nn = emtk.emtk_nn_create(1)
    rows = lambda: T(m, n)  # noqa: E731
    every = [
        (emtk.emtk_dropout, dict(x=rows(), y=rows(), drop=emtk.Drop(0.1, 1, 2, T(1, dtype=torch.int64)))),
        (emtk.emtk_residual_norm, dict(residual=rows(), block=rows(), y=rows(), h=rows(), post=emtk.Norm("rms", T(n), T(n)), pre=emtk.Norm("layer", T(n, dtype=f32), None),
                                       gate=T(2, n), gate_every=2, drop=emtk.Drop(0.1, 1, 2, T(1, dtype=torch.int64)))),
        (emtk.emtk_residual_norm_backward, dict(dy=rows(), dh=rows(), y=rows(), block=rows(), d_residual=rows(), d_block=rows(), post=emtk.Norm("rms", T(n), T(n)),
                                                pre=emtk.Norm("layer", T(n)), gate=T(2, n), gate_every=2, d_gate=T(2, n, dtype=f32), dw_pre=T(n, dtype=f32),
                                                db_pre=T(n, dtype=f32), dw_post=T(n, dtype=f32), db_post=T(n, dtype=f32))),
        (emtk.emtk_logprobs, dict(logits=rows(), tokens=T(m, dtype=i32), logprob=T(m, dtype=f32), entropy=T(m, dtype=f32), lse=T(m, dtype=f32),
                                  top_logprob=T(m, 2, dtype=f32), top_index=T(m, 2, dtype=i32))),
        (emtk.emtk_logprobs_backward, dict(logits=rows(), lse=T(m, dtype=f32), d_logits=rows(), tokens=T(m, dtype=i32), d_logprob=T(m, dtype=f32),
                                           entropy=T(m, dtype=f32), d_entropy=T(m, dtype=f32))),
        (emtk.emtk_recurrence, dict(f=rows(), x=rows(), y=rows(), o=rows(), act="silu", seqs=2, offsets=T(3, dtype=i32), state=T(2, n, dtype=f32), last=T(2, n, dtype=f32),
                                    states=T(2, n, dtype=f32))),
        (emtk.emtk_recurrence_backward, dict(dy=rows(), f=rows(), x=rows(), states=T(2, n, dtype=f32), df=rows(), dx=rows(), o=rows(), act="silu", seqs=2,
                                             offsets=T(3, dtype=i32), d_last=T(2, n, dtype=f32), d_o=rows(), d_state=T(2, n, dtype=f32))),
    ]

    def moved(t):
        """The argument with one of its tensors on another device, each in turn."""
        if isinstance(t, Tensor):
            yield T(*t.shape, dtype=t.dtype, device=0)
        elif isinstance(t, tuple):
            for i, part in enumerate(t):
                for other in moved(part):
                    yield type(t)(*t[:i], other, *t[i + 1:])

    for call, args in every:
        calls.clear()
        call(nn, **args, stream=0)
        assert calls == [call.__name__]
        for name, t in args.items():
            for other in moved(t):
                calls.clear()
                with pytest.raises(ValueError):
                    call(nn, **dict(args, **{name: other}), stream=0)
                assert calls == [], (call.__name__, name)
    emtk.emtk_nn_destroy(nn)
