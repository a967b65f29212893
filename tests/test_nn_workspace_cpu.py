"""How large a workspace the layers ask for (host arithmetic of csrc/nn_internal.h, compiled as plain C++)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2009_04509_gb300", "csrc")

DRIVER = r"""
#include <cstdio>
#include "nn_internal.h"
int main() {
    size_t need, left;
    while (scanf("%zu %zu", &need, &left) == 2) printf("%zu\n", emtk::workspace_size(need, left));
    return 0;
}
"""


def test_a_workspace_that_fits_is_not_refused_for_its_reserve(tmp_path):
    """A quarter more than is needed where there is room for it, and what is needed where there is not."""
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    if shutil.which("g++") is None or not os.path.exists(os.path.join(cuda, "include", "cuda.h")):
        pytest.skip("no g++ or CUDA headers")
    src, exe = tmp_path / "size.cpp", tmp_path / "size"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-w", "-I", CSRC, "-I", os.path.join(cuda, "include"), str(src), "-o", str(exe)],
                   check=True)
    gb = 1 << 30
    cases = [(need, left) for need in (1, 256, gb, 40 * gb, 200 * gb) for left in (0, gb, 45 * gb, 54 * gb, 210 * gb, 280 * gb)]
    out = subprocess.run([str(exe)], input="\n".join(f"{n} {f}" for n, f in cases), capture_output=True, text=True, check=True)
    for (need, left), size in zip(cases, map(int, out.stdout.split()), strict=True):
        assert size in (need, need + need // 4)
        if need <= left:
            assert size <= left, (need, left)
        if 2 * need <= left:
            assert size == need + need // 4
