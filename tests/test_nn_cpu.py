"""Host-side checks of the layers' C ABI that need no GPU: struct layouts, packed argument formats and
refusals before the device is touched."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2009_04509_gb300 import emtk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = ("emtk_matrix", "emtk_dense_args", "emtk_dense_grad_args", "emtk_gated_args", "emtk_gated_grad_args")


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


def test_packed_bytes_fill_the_structs():
    """The binding's packed arguments are the structs: sizes agree and values land in their fields."""
    for packer, name in ((emtk._PACK_MATRIX, "emtk_matrix"), (emtk._PACK_DENSE, "emtk_dense_args"),
                         (emtk._PACK_DENSE_GRAD, "emtk_dense_grad_args"), (emtk._PACK_GATED, "emtk_gated_args"),
                         (emtk._PACK_GATED_GRAD, "emtk_gated_grad_args")):
        st = getattr(emtk, name)
        assert packer.size == ctypes.sizeof(st), name
        n = len(packer.unpack(bytes(packer.size)))
        filled = st.from_buffer_copy(packer.pack(*range(1, n + 1)))
        seen = []
        for f, kind in st._fields_:
            v = getattr(filled, f)
            seen += [getattr(v, g) for g, _ in kind._fields_] if kind is emtk.emtk_matrix else [v]
        assert seen == list(range(1, n + 1)), name


def test_refusals_without_device(lib):
    out = ctypes.c_void_p(1)
    for args in ((-1, 0, 1, 0), (0, -1, 1, 0), (0, 0, 0, 0), (0, 0, 1, 2)):
        assert lib.emtk_nn_create(*args, ctypes.byref(out)) == emtk.EMTK_ERR_ARG
        assert out.value is None
    assert lib.emtk_nn_create(0, 0, 1, 0, None) == emtk.EMTK_ERR_ARG
    assert lib.emtk_nn_destroy(None) == emtk.EMTK_OK
    assert lib.emtk_nn_check(None, None) == emtk.EMTK_ERR_ARG
    for f in (lib.emtk_dense, lib.emtk_dense_backward, lib.emtk_gated, lib.emtk_gated_backward):
        assert f(None, None, None) == emtk.EMTK_ERR_ARG
    for f in (lib.emtk_pack8, lib.emtk_unpack8):
        assert f(None, 0, 0, 0, None, None, None) == emtk.EMTK_ERR_ARG


def test_create_without_gpu_reports_cuda_error(lib):
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(emtk.EmtkError) as e:
        emtk.emtk_nn_create()
    assert e.value.status == emtk.EMTK_ERR_CUDA


def test_binding_checks_shapes_before_the_library():
    torch = pytest.importorskip("torch")
    x, w, y = (torch.zeros(s, dtype=torch.bfloat16) for s in ((4, 8), (6, 8), (4, 6)))
    for change in (dict(w=torch.zeros(6, 9, dtype=torch.bfloat16)), dict(act="tanh"), dict(x=x.float()), {}):
        with pytest.raises(ValueError):  # the last: tensors of the host
            emtk.emtk_dense(1, **dict(dict(x=x, w=w, y=y), **change))


def test_binding_refuses_tensors_of_another_device(monkeypatch):
    """A tensor of another GPU than the handle's is refused before the library sees its address, each argument
    alone; all on the handle's are passed on.  Stand-ins for the tensors and the library: no GPU is needed."""
    torch = pytest.importorskip("torch")
    calls = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name == "emtk_nn_create":
                    args[-1]._obj.value = 4096 + args[0]
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

        def stride(self, i=None):
            s = (self.shape[-1], 1) if len(self.shape) == 2 else (1,)
            return s if i is None else s[i]

        def data_ptr(self):
            return 1 << 20

    monkeypatch.setattr(emtk, "load_library", lambda path=None: Library())
    m, k, n, f32 = 4, 8, 6, torch.float32
    T = Tensor

    def q8(rows, cols, device=1):
        return emtk.Q8(T(rows, cols, dtype=torch.int8, device=device), T(rows, 1, dtype=torch.uint8, device=device))

    nn = emtk.emtk_nn_create(1)
    every = [
        (emtk.emtk_dense, dict(x=T(m, k), w=T(n, k), y=T(m, n), bias=T(n), residual=T(m, n), pre=T(m, n))),
        (emtk.emtk_dense, dict(x=T(m, k), w=T(n, k), y=T(m, n), pre=q8(m, n))),
        (emtk.emtk_dense_backward, dict(dy=T(m, n), x=T(m, k), w=T(n, k), pre=T(m, n), dx=T(m, k), dw=T(n, k), db=T(n, dtype=f32))),
        (emtk.emtk_gated, dict(x=T(m, k), w_gate=T(n, k), w_up=T(n, k), h=T(m, n), bias_gate=T(n), bias_up=T(n), gate=q8(m, n), up=q8(m, n))),
        (emtk.emtk_gated_backward, dict(dh=T(m, n), gate=T(m, n), up=T(m, n), x=q8(m, k), w_gate=T(n, k), w_up=T(n, k), dx=T(m, k),
                                        dw_gate=T(n, k), dw_up=T(n, k), db_gate=T(n, dtype=f32), db_up=T(n, dtype=f32), h=T(m, n))),
        (emtk.emtk_pack8, dict(x=T(m, k), q=q8(m, k))),
        (emtk.emtk_unpack8, dict(q=q8(m, k), x=T(m, k))),
    ]
    for call, args in every:
        calls.clear()
        call(nn, **args, stream=0)
        assert calls == [call.__name__]
        for name, t in args.items():
            parts = [t] if not isinstance(t, emtk.Q8) else list(t)
            for i, part in enumerate(parts):
                other = T(*part.shape, dtype=part.dtype, device=0)
                moved = other if not isinstance(t, emtk.Q8) else emtk.Q8(*(other if j == i else p for j, p in enumerate(parts)))
                calls.clear()
                with pytest.raises(ValueError):
                    call(nn, **dict(args, **{name: moved}), stream=0)
                assert calls == [], (call.__name__, name)
    emtk.emtk_nn_destroy(nn)
