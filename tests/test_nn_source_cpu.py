"""What the layers' kernels must hold to that no run can show, read from their source."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2009_04509_gb300", "csrc")


def test_no_cta_of_a_pair_leaves_before_its_arrivals():
    """A commit of the pair's MMAs arrives at a barrier in each CTA's shared memory, some time after it was
    issued.  Each such barrier must be waited for by code that both CTAs run, after its last commit, and before
    the closing cluster barrier: a CTA that left earlier could have the arrival land in its successor's memory."""
    with open(os.path.join(CSRC, "nn_mm.cu")) as f:
        src = f.read()
    kernel = src[src.index("mm_kernel(const __grid_constant__"):src.index("// Eight columns of a row, of which the first n exist.")]
    cuts = [kernel.rindex(at) for at in ("if (warp == 0) {\n", "} else if (warp == 1 && rank == 0) {",
                                         "} else if (warp >= kFirstEpiWarp) {", "    tc_fence_before();\n    __syncthreads();\n")]
    producer, issuer, epilogue, tail = (kernel[a:b] for a, b in zip(cuts, cuts[1:] + [len(kernel)]))
    tail = tail[:tail.rindex("cluster_sync();")]

    def waited(text):
        return set(re.findall(r"(?:warp_wait_all|warp_wait|mbar_try_wait)\(bar\((kBar[A-Za-z]+)", text))

    committed = set(re.findall(r"mma_commit_pair\(bar\((kBar[A-Za-z]+)", kernel))
    assert committed == set(re.findall(r"mma_commit_pair\(bar\((kBar[A-Za-z]+)", issuer)) != set()
    filled = producer[producer.index("                if (++s == S::kStages) {"):]  # the stages' loop has ended
    assert "rank" not in filled and "rank" not in tail  # both CTAs run these
    # the accumulators' last phases: the epilogue waits for every tile's
    assert committed <= waited(filled) | waited(tail) | (waited(epilogue) & {"kBarAccFull"})


def _sources():
    return {n: open(os.path.join(CSRC, n)).read() for n in sorted(os.listdir(CSRC)) if n.startswith("nn_")}


def test_every_device_function_of_the_layers_is_called():
    text = "\n".join(_sources().values())
    names = set(re.findall(r"__(?:device|global)__[^;{}=]*?\b([a-z]\w*)\s*\(", re.sub(r"__launch_bounds__\([^)]*\)|__cluster_dims__\([^)]*\)", "", text)))
    assert len(names) > 60
    assert [n for n in sorted(names) if len(re.findall(rf"\b{n}\b", text)) < 2] == []


def test_every_field_of_a_kernels_parameters_is_read():
    """A field of a structure that is passed to a kernel by value is read somewhere, not only set."""
    src = _sources()
    for name, struct in (("nn_mm.cu", "MmWork"), ("nn_mm.cu", "MmParams"), ("nn_skinny.cu", "SkinnyParams"),
                         ("nn_rows.cu", "RowsParams"), ("nn_pointwise.cu", "SlopeArgs"), ("nn_pointwise.cu", "PackArgs")):
        text = re.sub(r"//[^\n]*|\bj\.\w+", "", src[name])  # j: the job, whose fields have the same names
        body = re.search(rf"struct {struct} {{(.*?)\n}};", text, re.S).group(1)
        fields = re.findall(r"\*?\b(\w+)(?:\[\w+\])*\s*[,;]", body)
        assert len(fields) > 4, struct
        for f in fields:
            uses = len(re.findall(rf"(?:\.|->){f}\b", text))
            sets = len(re.findall(rf"(?:\.|->){f}(?:\[\w+\])*\s*=[^=]", text))
            assert uses > sets, f"{struct}.{f}"
