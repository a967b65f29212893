"""The products' plan (csrc/nn_plan.cu, host arithmetic) compiled as plain C++: every tile of every job is
dealt out exactly once, every chunk of its contraction to exactly one part, to pairs that exist."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2009_04509_gb300", "csrc")

DRIVER = r"""
#include <cstdio>
#include "nn_plan.cu"
int main() {
    using namespace emtk;
    // divisions: every small divisor and some large ones, at the ends and around multiples
    for (uint32_t d = 1; d < 5000; d += d < 300 ? 1 : 37)
        for (uint64_t q = 0; q * d < (1ull << 31); q = q * 3 + 1)
            for (int e = -1; e <= 1; ++e) {
                const int64_t n = (int64_t)(q * d) + e;
                if (n >= 0 && n < (1ll << 31) && Divisor(d).of((int)n) != (int)(n / d)) return printf("divisor %u of %lld\n", d, (long long)n), 1;
            }
    int n, kind, sms;
    while (scanf("%d %d %d", &n, &kind, &sms) == 3) {
        MmJob jobs[kMaxJobs] = {};
        for (int i = 0; i < n; ++i) {
            jobs[i].kind = (MmKind)kind;
            if (scanf("%d %d %d %d", &jobs[i].M, &jobs[i].N, &jobs[i].K, &jobs[i].terms) != 4) return 1;
        }
        const MmPlan p = plan_mm(jobs, n, sms);
        printf("plan %d %d %zu %d\n", p.tn, p.pairs, p.workspace, p.pieces);
        for (int i = 0; i < p.pieces; ++i) {
            const MmPlan::Piece &c = p.piece[i];
            printf("%d %d %d %d %d %d %d %d %lld\n", c.job, c.tile0, c.tiles, c.parts, c.chunks_per_part, c.units, c.pair_lo,
                   c.pair_count, (long long)c.part_at);
        }
    }
    return 0;
}
"""


def ceil(a, b):
    return -(-a // b)


def test_every_unit_is_dealt_once(tmp_path):
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    if shutil.which("g++") is None or not os.path.exists(os.path.join(cuda, "include", "cuda.h")):
        pytest.skip("no g++ or CUDA headers")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-I", CSRC, "-I", os.path.join(cuda, "include"), str(src), "-o",
                    str(exe)], check=True)
    rng = random.Random(0)
    size = lambda hi: int(round(2 ** rng.uniform(0, hi)))  # noqa: E731
    cases = [(1, 0, 152, [(1, 1, 0, 1)]), (1, 1, 152, [(5, 700, 0, 1)]), (2, 0, 1, [(300, 300, 300, 1), (40, 40, 9000, 1)])]
    for _ in range(1500):
        n, kind = rng.choice((1, 1, 2, 3)), 0
        if n == 1:
            kind = rng.choice((0, 1))
        m, f, k = size(15), size(14), size(14)
        jobs = {1: [(m, f, k, 1)], 2: [(m, k, f, 1), (f, k, m, 1)], 3: [(m, k, f, 2), (f, k, m, 1), (f, k, m, 1)]}[n]
        cases.append((n, kind, rng.choice((152, 148, 20)), jobs))
    text = "\n".join(" ".join(map(str, (n, kind, sms, *[v for j in jobs for v in j]))) for n, kind, sms, jobs in cases)
    out = subprocess.run([str(exe)], input=text, capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    lines = iter(out.stdout.splitlines())
    for n, kind, sms, jobs in cases:
        word, tn, pairs, workspace, pieces = next(lines).split()
        tn, pairs, workspace, pieces = int(tn), int(pairs), int(workspace), int(pieces)
        assert word == "plan" and tn in (128, 256) and 1 <= pairs <= max(1, sms // 2) and 1 <= pieces <= 8
        seen = [[] for _ in jobs]
        ends, busy = [], set()
        for _ in range(pieces):
            job, tile0, tiles, parts, cpp, units, lo, count, at = map(int, next(lines).split())
            m, cols, k, terms = jobs[job]
            total = ceil(k, 64) * terms
            assert tiles > 0 and units == tiles * parts and 0 <= lo and count > 0 and lo + count <= pairs
            assert parts == 1 and total <= cpp or (parts - 1) * cpp < total <= parts * cpp
            busy |= {lo + u % count for u in range(min(units, count))}
            seen[job].append((tile0, tile0 + tiles))
            if parts > 1:
                ends.append((at, at + units * 256 * tn))
        assert 0 in busy and max(busy) < pairs
        for job, (m, cols, k, terms) in enumerate(jobs):
            want = ceil(m, 256) * ceil(cols, tn // 2 if kind else tn)
            at = 0
            for a, b in sorted(seen[job]):
                assert a == at
                at = b
            assert at == want
        at = 0
        for a, b in sorted(ends):
            assert a == at
            at = b
        assert workspace == 4 * at
