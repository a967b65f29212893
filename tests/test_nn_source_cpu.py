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
