"""Residual norms, dropout, log probabilities and the gated recurrence against their definitions in 64 bits.

Tolerances are error bounds, element by element:
  - a value stored in 16 bits is off by u |value| (u = 2^-8 bf16, 2^-11 fp16; fp16 also 2^-25 absolute below its
    normal range);
  - fp32 arithmetic on the way is off by a number of roundings E = 2^-23 times the magnitude of the terms that are
    added, computed beside the result (the fast exponential, reciprocal and square root: 4 of them, an exponential
    of z |z| more).  A sum of n terms in a tree of 256 threads or more takes n / 256 + 16 of them.
"""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "f32": 0.0}
TINY = {"bf16": 0.0, "fp16": 2.0 ** -25, "f32": 0.0}
E = 2.0 ** -23


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_04509_gb300 import build, emtk
    build.build()
    return emtk


@pytest.fixture(scope="module")
def nn(lib):
    h = lib.emtk_nn_create()
    yield h
    assert lib.emtk_nn_check(h) == lib.EMTK_OK
    lib.emtk_nn_destroy(h)


class Buf:
    """A [rows][cols] view of a wider, possibly shifted buffer; what surrounds it is NaN and must stay as it was
    (inputs: must not be read into a result)."""

    def __init__(self, rows, cols, dtype, pad=0, shift=0, values=None):
        self.whole = torch.full((rows * (cols + pad) + shift + 64,), float("nan"), dtype=dtype, device="cuda")
        self.t = self.whole[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        self.args = (rows, cols, pad, shift)
        if values is not None:
            self.t.copy_(values)

    def surroundings_untouched(self):
        rows, cols, pad, shift = self.args
        w = self.whole.clone()
        w[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = float("nan")
        return bool(torch.isnan(w.float()).all())


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def near(got, want, kind, slack, what=""):
    """got within its rounding of want, and slack (a tensor or number, absolute)."""
    bound = U[kind] * want.abs() * (1 + 2.0 ** -8) + TINY[kind] + slack
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, at {bad.nonzero()[0].tolist()}: " \
                          f"{got[bad][0]} for {want[bad][0]}"


# ------------------------------------------------------------------ dropout
def philox(counter, key):
    """Philox4x32-10 in Python's whole numbers."""
    x, k = list(counter), list(key)
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(b >> 32) ^ x[1] ^ k[0], b & 0xffffffff, (a >> 32) ^ x[3] ^ k[1], a & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return x


def factors(m, n, p, seed, offset):
    """Dropout's factors [m][n], 64 bits: numpy's whole numbers of 64 bits, word by word."""
    low = np.uint64(0xffffffff)
    t = int(np.rint(np.float64(np.float32(p)) * 65536))
    if t == 0:
        return torch.ones(m, n, dtype=torch.float64, device="cuda")
    g, r = np.meshgrid(np.arange(-(-n // 8), dtype=np.uint64), np.arange(m, dtype=np.uint64))
    x = [g, r, np.full_like(g, offset & 0xffffffff), np.full_like(g, (offset >> 32) & 0xffffffff)]
    k = [seed & 0xffffffff, (seed >> 32) & 0xffffffff]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    bits = np.stack([w >> np.uint64(s) & np.uint64(0xffff) for w in x for s in (0, 16)], axis=2).reshape(m, -1)[:, :n]
    return torch.from_numpy((bits >= t) * (65536 / (65536 - t))).cuda()


def test_dropout_is_the_generator(lib, nn):
    """Element by element, from the published generator."""
    m, n, seed, offset = 3, 21, 0xa4093822299f31d0, 0x0370734413198a2e
    x, y = torch.ones(m, n, device="cuda", dtype=torch.bfloat16), torch.empty(m, n, device="cuda", dtype=torch.bfloat16)
    lib.emtk_dropout(nn, x, y, lib.Drop(0.5, seed, offset))
    for i in range(m):
        for j in range(n):
            w = philox((j // 8, i, offset & 0xffffffff, offset >> 32), (seed & 0xffffffff, seed >> 32))[j % 8 // 2]
            assert float(y[i, j]) == (2.0 if (w >> (16 * (j % 2))) & 0xffff >= 32768 else 0.0), (i, j)


SIZES = [(1, 1), (1, 8), (2, 5), (1, 4096), (3, 7), (5, 31), (7, 32), (4, 33), (3, 255), (2, 256), (5, 257), (235, 333), (6, 2048),
         (17, 2300), (700, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("i,size", list(enumerate(SIZES)))
def test_dropout(lib, nn, i, size, dtype):
    m, n = size
    for pad, shift, out_pad, out_shift in ((0, 0, 0, 0), (8, 8, 0, 0), (1, 1, 3, 2), (3, 0, 5, 7), (2, 2, 1, 0), (0, 5, 8, 3)):
        p = random.Random(i * 7 + pad).choice([0.1, 0.25, 0.5, 0.999, 1e-6, 0.0])
        x = Buf(m, n, DT[dtype], pad, shift, randn(gen(i), m, n))
        y = Buf(m, n, DT[dtype], out_pad, out_shift)
        lib.emtk_dropout(nn, x.t, y.t, lib.Drop(p, 1234567890123 + i, (i << 32) + 5))
        want = x.t.double() * factors(m, n, p, 1234567890123 + i, (i << 32) + 5)
        near(y.t, want, dtype, want.abs() * 2 * E)
        assert y.surroundings_untouched()
        before = x.t.double()
        lib.emtk_dropout(nn, x.t, x.t, lib.Drop(p, 1234567890123 + i, (i << 32) + 5))  # in place
        assert torch.equal(x.t, y.t) and x.surroundings_untouched(), (pad, shift)
        assert torch.equal(before == 0, x.t.double() == 0) or p > 0


@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 3)])
@pytest.mark.parametrize("m,n", [(30000, 333), (7001, 2048)])
def test_dropout_of_many_pieces(lib, nn, m, n, pad, shift):
    """More pieces than threads: every thread goes round its loop, on the grid and off it, apart and in place."""
    x, y = Buf(m, n, torch.bfloat16, pad, shift, randn(gen(m), m, n)), Buf(m, n, torch.bfloat16, pad, shift)
    x.t[x.t == 0] = 1.0
    drop = lib.Drop(0.3, 5, 1 << 35)
    lib.emtk_dropout(nn, x.t, y.t, drop)
    d = factors(m, n, 0.3, 5, 1 << 35)
    want = x.t.double() * d
    near(y.t, want, "bf16", want.abs() * 2 * E)
    assert torch.equal(y.t == 0, d == 0) and y.surroundings_untouched()
    lib.emtk_dropout(nn, x.t, x.t, drop)
    assert torch.equal(x.t, y.t) and x.surroundings_untouched()


def test_dropped_values_are_zero_whatever_they_were(lib, nn):
    m, n = 40, 300
    x = torch.full((m, n), float("nan"), dtype=torch.float16, device="cuda")
    x[::2] = math.inf
    y = torch.empty_like(x)
    lib.emtk_dropout(nn, x, y, lib.Drop(0.3, 7))
    kept = factors(m, n, 0.3, 7, 0) > 0
    assert torch.equal(y[~kept], torch.zeros_like(y[~kept]))
    assert not torch.isfinite(y[kept]).any()


# ------------------------------------------------------------------ residual norms
def norm64(x, kind, w, b, eps, n):
    if kind is None:
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    x = x / torch.sqrt(x.square().mean(1, keepdim=True) + eps)
    x = x * w if w is not None else x
    return x + b if b is not None else x


def norm_config(i):
    r = random.Random(1000 + i)
    c = dict(size=r.choice([(1, 1), (1, 8), (4, 3), (3, 64), (1, 4096), (5, 257), (33, 515), (2, 2048), (3, 2056), (9, 4097), (2, 8192), (2, 8200),
                            (3, 11000), (2, 16383), (2, 16384), (300, 40), (64, 1024), (1000, 96)]),
             pad=r.choice([0, 0, 1, 3, 8]), shift=r.choice([0, 0, 1, 8]), out_pad=r.choice([0, 0, 1, 8]), out_shift=r.choice([0, 0, 3]),
             post=r.choice([None, "rms", "layer"]), pre=r.choice([None, "rms", "layer", "rms", "layer"]),
             gate=r.choice([None, "vector", "rows"]), every=r.choice([1, 2, 3, 7, 64]), p=r.choice([0.0, 0.0, 0.2]),
             scale=r.choice([1.0, 0.5, 0.0]), params=r.choice(["same", "f32"]), weights=r.choice([(1, 1), (1, 0), (0, 0), (0, 1)]),
             residual=r.random() < 0.85, dy=r.random() < 0.8, eps=r.choice([1e-6, 1e-3]))
    if c["pre"] is None:
        c["dy"] = True
    return c


def seam(lib, c, dtype, i):
    """The tensors of a case, and the arguments that both calls share."""
    (m, n), t = c["size"], DT[dtype]
    g = gen(i)
    par = torch.float32 if c["params"] == "f32" else t
    shift = 1 if c["shift"] == 1 else 0  # parameters off the grid too

    def vector(scale, about):
        v = torch.empty(n + shift, dtype=par, device="cuda")[shift:]
        return v.copy_(randn(g, n) * scale + about)

    norms = {}
    for which in ("post", "pre"):
        if c[which]:
            norms[which] = lib.Norm(c[which], vector(0.3, 1.0) if c["weights"][0] else None, vector(0.3, 0.0) if c["weights"][1] else None,
                                    c["eps"])
    groups = -(-m // c["every"])
    gate = randn(g, n).to(t) if c["gate"] == "vector" else randn(g, groups, n).to(t) if c["gate"] == "rows" else None
    shared = dict(norms, gate=gate, scale=c["scale"], drop=lib.Drop(c["p"], 99 + i, 1 << 40) if c["p"] else None,
                  gate_every=c["every"] if c["gate"] == "rows" else None)

    def matrix(scale=1.0):
        return Buf(m, n, t, c["pad"], c["shift"], randn(g, m, n) * scale)

    return shared, matrix, (lambda: Buf(m, n, t, c["out_pad"], c["out_shift"]))


def parts64(c, shared, i):
    m, n = c["size"]
    d = factors(m, n, c["p"], 99 + i, 1 << 40)
    gate = shared["gate"]
    if gate is None:
        g = torch.ones(1, n, dtype=torch.float64, device="cuda")
    else:
        g = gate.double().view(-1, n)
    p = {w: (None, None) if w not in shared else tuple(None if v is None else v.double() for v in shared[w][1:3]) for w in ("post", "pre")}
    return d, g, p


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("i", range(40))
def test_residual_norm(lib, nn, i, dtype):
    c = norm_config(i)
    m, n = c["size"]
    shared, matrix, out = seam(lib, c, dtype, i)
    b, r = matrix(3.0), matrix() if c["residual"] else None
    y, h = out(), out() if c["pre"] else None
    lib.emtk_residual_norm(nn, None if r is None else r.t, b.t, y.t, None if h is None else h.t, **shared)
    d, g, p = parts64(c, shared, i)
    rows = torch.arange(m, device="cuda") // (c["every"] if c["gate"] == "rows" else max(1, m))
    k = n / 256 + 24
    v = norm64(b.t.double(), c["post"], *p["post"], c["eps"], n)
    size_v = v.abs() if c["post"] is None else v.abs() + norm64(b.t.double(), c["post"], p["post"][0], None, c["eps"], n).abs()
    if c["post"] == "layer":  # centring loses what the mean is larger than the spread
        x = b.t.double()
        w = p["post"][0].abs() if p["post"][0] is not None else 1.0
        size_v = size_v + w * x.mean(1, keepdim=True).abs() / torch.sqrt(x.var(1, correction=0, keepdim=True) + c["eps"])
    want = g[rows] * d * v + (c["scale"] * r.t.double() if r else 0.0)
    err = k * E * ((g[rows] * d).abs() * size_v + (abs(c["scale"]) * r.t.double().abs() if r else 0.0))
    near(y.t, want, dtype, err, "y")
    assert y.surroundings_untouched()
    if h is not None:
        want_h = norm64(want, c["pre"], *p["pre"], c["eps"], n)
        spread = torch.sqrt((want.var(1, correction=0, keepdim=True) if c["pre"] == "layer" else want.square().mean(1, keepdim=True)) + c["eps"])
        w = p["pre"][0].abs() if p["pre"][0] is not None else 1.0
        # an error of y, centred and over its spread; and the spread's own, at most the row's rms of errors over it
        slack = w * (err + err.mean(1, keepdim=True) + k * E * (want.abs() + want.mean(1, keepdim=True).abs())) / spread + \
            (want_h.abs() + w) * (err.square().mean(1, keepdim=True).sqrt() / spread + k * E) + k * E * want_h.abs()
        near(h.t, want_h, dtype, slack, "h")
        assert h.surroundings_untouched()
    if r is not None:  # y may be the residual
        lib.emtk_residual_norm(nn, r.t, b.t, r.t, None if h is None else h.t, **shared)
        assert torch.equal(r.t, y.t) and r.surroundings_untouched()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("i", range(40))
def test_residual_norm_backward(lib, nn, i, dtype):
    """Gradients by differentiation of the definition in 64 bits.  The slack: roundings of the terms that each is a
    sum of; for the sums over rows, of their terms' magnitudes."""
    c = norm_config(i)
    m, n = c["size"]
    t = DT[dtype]
    shared, matrix, out = seam(lib, c, dtype, i)
    y, b, dy, dh = matrix(2.0), matrix(3.0), matrix(0.5) if c["dy"] else None, matrix(0.5) if c["pre"] else None
    dr, db = out(), out()
    sums = {}
    for which in ("pre", "post"):
        if which in shared:
            sums["dw_" + which], sums["db_" + which] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    groups = -(-m // c["every"]) if c["gate"] == "rows" else 1
    dg = Buf(groups, n, torch.float32, 3) if c["gate"] == "rows" else torch.empty(n, device="cuda")
    d_gate = dg.t if c["gate"] == "rows" else dg
    opt = lambda x: None if x is None else x.t  # noqa: E731
    call = lambda: lib.emtk_residual_norm_backward(nn, opt(dy), opt(dh), y.t if c["pre"] else None, b.t, dr.t, db.t, d_gate=d_gate, **sums, **shared)  # noqa: E731
    call()
    d, g, p = parts64(c, shared, i)
    g.requires_grad_()
    leaves = {}
    for which in ("pre", "post"):
        if c[which]:
            w, bias = p[which]
            leaves[which] = (torch.ones(n, dtype=torch.float64, device="cuda") if w is None else w, torch.zeros(n, dtype=torch.float64, device="cuda") if bias is None else bias)
            for v in leaves[which]:
                v.requires_grad_()
    rows = torch.arange(m, device="cuda") // (c["every"] if c["gate"] == "rows" else max(1, m))
    y64, b64 = y.t.double().requires_grad_(), b.t.double().requires_grad_()
    stream = dy.t.double() if dy is not None else torch.zeros(m, n, dtype=torch.float64, device="cuda")
    k = (n / 256 + 40) * E
    rms = lambda v: v.square().mean(1, keepdim=True).sqrt()  # noqa: E731
    size_t = stream.abs()
    if c["pre"]:
        norm64(y64, c["pre"], *leaves["pre"], c["eps"], n).backward(dh.t.double())
        stream = stream + y64.grad
        with torch.no_grad():
            q = (dh.t.double() * leaves["pre"][0]).abs()
            mean = y64.mean(1, keepdim=True) if c["pre"] == "layer" else 0.0
            s = torch.sqrt((y64 - mean).square().mean(1, keepdim=True) + c["eps"])
            hat = (y64 - mean).abs() / s
            off = 1 + (y64.mean(1, keepdim=True).abs() / s if c["pre"] == "layer" else 0.0)  # centring
            size_t = size_t + off * (q + rms(q) * (1 + hat)) / s
    near(dr.t, c["scale"] * stream, dtype, k * abs(c["scale"]) * size_t, "d_residual")
    v = norm64(b64, c["post"], *leaves["post"], c["eps"], n) if c["post"] else b64
    (g[rows] * d * v).backward(stream)
    with torch.no_grad():
        size_v = v.abs() + (leaves["post"][1].abs() if c["post"] else 0.0)
        size_u = (g[rows] * d).abs() * size_t
        size_b = size_u
        if c["post"]:
            mean = b64.mean(1, keepdim=True) if c["post"] == "layer" else 0.0
            s = torch.sqrt((b64 - mean).square().mean(1, keepdim=True) + c["eps"])
            hat = (b64 - mean).abs() / s
            off = 1 + (b64.mean(1, keepdim=True).abs() / s if c["post"] == "layer" else 0.0)
            q = size_u * leaves["post"][0].abs()
            size_b = off * (q + rms(q) * (1 + hat)) / s
            size_v = size_v + off * leaves["post"][0].abs()
        near(db.t, b64.grad, dtype, k * size_b, "d_block")
        by_rows = (m / 16 + 40) * E + k
        gate_slack = torch.zeros_like(g).index_add_(0, rows, size_t * d * size_v) * by_rows
        near(d_gate.view(-1, n), g.grad, "f32", gate_slack, "d_gate")
        if c["pre"]:
            mean = y64.mean(1, keepdim=True) if c["pre"] == "layer" else 0.0
            s = torch.sqrt((y64 - mean).square().mean(1, keepdim=True) + c["eps"])
            hat = (y64.abs() + (mean.abs() if c["pre"] == "layer" else 0.0)) / s
            near(sums["dw_pre"], leaves["pre"][0].grad, "f32", (dh.t.double().abs() * hat).sum(0) * by_rows, "dw_pre")
            near(sums["db_pre"], leaves["pre"][1].grad, "f32", dh.t.double().abs().sum(0) * by_rows, "db_pre")
        if c["post"]:
            mean = b64.mean(1, keepdim=True) if c["post"] == "layer" else 0.0
            s = torch.sqrt((b64 - mean).square().mean(1, keepdim=True) + c["eps"])
            hat = (b64.abs() + (mean.abs() if c["post"] == "layer" else 0.0)) / s
            near(sums["dw_post"], leaves["post"][0].grad, "f32", (size_u * hat).sum(0) * by_rows, "dw_post")
            near(sums["db_post"], leaves["post"][1].grad, "f32", size_u.sum(0) * by_rows, "db_post")
    assert dr.surroundings_untouched() and db.surroundings_untouched()
    if c["gate"] == "rows":
        assert dg.surroundings_untouched()
    first = [dr.t.clone(), db.t.clone(), d_gate.clone()] + [v.clone() for v in sums.values()]
    call()  # the same bits
    assert all(torch.equal(x, z) for x, z in zip(first, [dr.t, db.t, d_gate] + list(sums.values())))
    if dy is not None:  # d_residual may be dy; outputs may be absent
        lib.emtk_residual_norm_backward(nn, dy.t, opt(dh), y.t if c["pre"] else None, None, dy.t, None,
                                        **{k2: v2 for k2, v2 in shared.items() if k2 in ("pre", "scale")})
        assert torch.equal(dy.t, first[0]) and dy.surroundings_untouched()


@pytest.mark.parametrize("post,pre,gate,every", [("layer", "rms", "vector", 1), ("rms", "layer", "rows", 7), (None, "layer", None, 1)])
@pytest.mark.parametrize("m,n,pad,shift", [(2500, 2056, 0, 0), (2500, 2059, 1, 3), (400, 8200, 8, 0), (400, 8197, 0, 1), (333, 16384, 0, 0), (333, 16381, 0, 5)])
def test_residual_norm_backward_of_many_rows(lib, nn, monkeypatch, m, n, pad, shift, post, pre, gate, every):
    """More rows than blocks: a block goes from row to row through its stages, with two rows ahead or one."""
    c = dict(norm_config(0), size=(m, n), pad=pad, shift=shift, out_pad=pad, out_shift=shift, post=post, pre=pre, gate=gate, every=every, p=0.2 if gate else 0.0,
             scale=0.5, params="f32", weights=(1, 1), residual=True, dy=True, eps=1e-3)
    monkeypatch.setitem(globals(), "norm_config", lambda i: c)
    test_residual_norm_backward(lib, nn, 3, "bf16")


@pytest.mark.parametrize("pads", [(0,) * 4, (1,) * 4, (3, 1, 0, 2), (1, 0, 0, 0)])
@pytest.mark.parametrize("n,m,every", [(40, 61, 7), (517, 100, 100), (2312, 33, 1), (8, 1, 1)])
def test_sums_with_d_residual_in_dys_place(lib, nn, n, m, every, pads):
    """The sums past the block's norm are of the dy that was given: every result has the bits that it has apart."""
    g = gen(n + m)
    y, dh, b, dy = (Buf(m, n, torch.bfloat16, p, p, randn(g, m, n)).t for p in pads)
    gate, w = randn(g, -(-m // every), n).to(torch.bfloat16), randn(g, n)
    shared = dict(pre=lib.Norm("rms", w), post=lib.Norm("layer", w, w), gate=gate, gate_every=every, scale=0.5, drop=lib.Drop(0.25, 3, 4))
    results = []
    for place in (torch.empty_like(dy), dy):
        sums = {k: torch.empty(n, device="cuda") for k in ("dw_pre", "db_pre", "dw_post", "db_post")}
        d_block, d_gate = torch.empty(m, n, dtype=torch.bfloat16, device="cuda"), torch.empty(gate.shape, device="cuda")
        lib.emtk_residual_norm_backward(nn, dy, dh, y, b, place, d_block, d_gate=d_gate, **sums, **shared)
        results.append([place.clone(), d_block, d_gate, *sums.values()])
    assert all(torch.equal(x, z) for x, z in zip(*results))


@pytest.mark.parametrize("n,m", [(40, 61), (517, 100), (2311, 40), (1000, 9), (8, 33), (3, 50)])
@pytest.mark.parametrize("gate_rows", [1, 3, 1000])
def test_gradients_do_not_depend_on_where_matrices_lie(lib, nn, m, n, gate_rows):
    """All on the 16-byte grid, all off it alike, each otherwise: sums over the same values in other orders."""
    g = gen(n)
    vals = [(randn(g, m, n) * s).to(torch.bfloat16) for s in (1.0, 1.0, 2.0, 1.0)]
    w1, w2, c2 = randn(g, n), randn(g, n), randn(g, n)
    gate = randn(g, -(-m // gate_rows), n).to(torch.bfloat16)
    results = []
    for pads in ((-n % 8,) * 4, (-n % 8 + 3,) * 4, (0, 1, 2, 5)):
        dy, dh, y, b = (Buf(m, n, torch.bfloat16, p, 0 if p == pads[0] and len(set(pads)) == 1 else i, v).t
                        for i, (p, v) in enumerate(zip(pads, vals)))
        if len(set(pads)) == 1 and pads[0] % 8:
            assert len({t.data_ptr() % 16 for t in (dy, dh, y, b)}) == 1
        dr, db = torch.empty_like(vals[0]), torch.empty_like(vals[0])
        f = [torch.empty(n, device="cuda") for _ in range(4)]
        dg = torch.empty(gate.shape, device="cuda")
        lib.emtk_residual_norm_backward(nn, dy, dh, y, b, dr, db, post=lib.Norm("layer", w1, c2), pre=lib.Norm("rms", w2), gate=gate, gate_every=gate_rows,
                                        drop=lib.Drop(0.2, 5, 6), d_gate=dg, dw_pre=f[0], db_pre=f[1], dw_post=f[2], db_post=f[3])
        results.append([dr, db, dg] + f)
    for other in results[1:]:
        assert torch.equal(other[0], results[0][0]) and torch.equal(other[1], results[0][1])
        for a, z in zip(results[0][2:], other[2:]):
            # m terms each, added in another order: their magnitudes are within the largest times m
            assert (a - z).abs().max() <= (m / 8 + 16) * 2.0 ** -23 * m * 40


def test_residual_norm_gradients_against_differences(lib, nn):
    """The backward call against differences of the definition that the forward call is held to."""
    m, n, eps = 3, 24, 1e-3
    g = gen(5)
    r, b, dy, dh = (randn(g, m, n).to(torch.bfloat16) for _ in range(4))
    w1, w2, gate = (randn(g, n).to(torch.bfloat16) for _ in range(3))
    drop = lib.Drop(0.25, 3, 4)
    y, h = torch.empty_like(r), torch.empty_like(r)
    args = dict(post=lib.Norm("layer", w1, None, eps), pre=lib.Norm("rms", w2, None, eps), gate=gate, scale=0.5, drop=drop)
    lib.emtk_residual_norm(nn, r, b, y, h, **args)
    db, dgate = torch.empty_like(r), torch.empty(n, device="cuda")
    lib.emtk_residual_norm_backward(nn, dy, dh, y, b, None, db, d_gate=dgate, **args)
    keep = factors(m, n, 0.25, 3, 4)

    def value(b64, g64):
        out = 0.5 * r.double() + g64 * keep * norm64(b64, "layer", w1.double(), None, eps, n)
        return (out * dy.double()).sum() + (norm64(out, "rms", w2.double(), None, eps, n) * dh.double()).sum()

    for tensor, grad in ((0, db.double()), (1, dgate.double())):
        base = [b.double(), gate.double()]
        step = randn(gen(9), *base[tensor].shape).double()
        hi, lo = list(base), list(base)
        hi[tensor], lo[tensor] = base[tensor] + 1e-5 * step, base[tensor] - 1e-5 * step
        slope = float((value(*hi) - value(*lo)) / 2e-5)
        # y is given in 16 bits (2^-8 of each), the gradient rounded to them: terms' magnitudes times a few of those
        assert abs(slope - float((grad * step).sum())) <= 6 * 2.0 ** -8 * float((grad * step).abs().sum()) + 1e-3


def test_residual_norm_of_nothing(lib, nn):
    """No rows: the sums are 0.  Rows of zeros: eps alone is under the root."""
    e = lambda *s, t=torch.bfloat16: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    lib.emtk_residual_norm(nn, e(0, 16), e(0, 16), e(0, 16), e(0, 16), pre=lib.Norm("rms"))
    dw, dg = torch.ones(16, device="cuda"), torch.ones(16, device="cuda")
    lib.emtk_residual_norm_backward(nn, None, e(0, 16), e(0, 16), e(0, 16), d_gate=dg, pre=lib.Norm("rms"), dw_pre=dw)
    assert not dw.any() and not dg.any()
    z, h = torch.zeros(5, 100, dtype=torch.float16, device="cuda"), e(5, 100, t=torch.float16)
    for kind in ("rms", "layer"):
        bias = torch.full((100,), 0.5, device="cuda")
        lib.emtk_residual_norm(nn, z, None, None, h, pre=lib.Norm(kind, None, bias))
        assert bool((h == 0.5).all())


def test_large_mean_is_centred_first(lib, nn):
    """A layer norm of rows whose mean is 1000 times their spread, in fp32's reach."""
    n = 2048
    x = (randn(gen(2), 4, n) * 0.5 + 500).to(torch.float16)  # steps of 0.25 to 0.5: the values are what they are
    h = torch.empty_like(x)
    lib.emtk_residual_norm(nn, None, x, None, h, pre=lib.Norm("layer"))
    want = norm64(x.double(), "layer", None, None, 1e-6, n)
    near(h, want, "fp16", 1000 * 4 * (n / 256 + 24) * E)


def test_residual_norm_keeps_rows_apart(lib, nn):
    n = 777
    b, r = randn(gen(1), 9, n).to(torch.bfloat16), randn(gen(2), 9, n).to(torch.bfloat16)
    bad = b.clone()
    bad[4, 5], bad[6, 7] = math.nan, math.inf
    outs = []
    for x in (b, bad):
        y, h = torch.empty_like(b), torch.empty_like(b)
        lib.emtk_residual_norm(nn, r, x, y, h, post=lib.Norm("layer"), pre=lib.Norm("rms"))
        outs.append((y, h))
    clean = [0, 1, 2, 3, 5, 7, 8]
    for a, z in zip(*outs):
        assert torch.equal(a[clean], z[clean]) and torch.isnan(z[4]).all() and not torch.isfinite(z[6]).any()


# ------------------------------------------------------------------ log probabilities
def logprobs64(z, tokens, temperature):
    l = torch.log_softmax(z.double() / temperature, 1)
    p = l.exp()
    entropy = -torch.special.xlogy(p, p).sum(1)
    lse = torch.logsumexp(z.double() / temperature, 1)
    v = z.shape[1]
    has = (tokens >= 0) & (tokens < v)
    lp = torch.where(has, l.gather(1, tokens.long().clamp(0, v - 1)[:, None])[:, 0], 0.0)
    return l, lp, entropy, lse


LOGITS = [(1, 1), (5, 2), (300, 3), (4, 7), (9, 8), (3, 9), (40, 31), (7, 33), (3, 256), (2, 257), (5, 1000), (3, 2047), (2, 2049), (3, 2064), (2, 4100),
          (1, 9000), (2, 50001), (1, 131072), (200, 2500), (1, 40000), (65, 64), (50, 150), (300, 600), (600, 1100), (1200, 2600)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "f32"])
@pytest.mark.parametrize("i,size", list(enumerate(LOGITS)))
def test_logprobs(lib, nn, i, size, dtype):
    m, v = size
    r = random.Random(i)
    for pad, shift, top, temperature, masked in ((0, 0, min(v, 5), 1.0, False), (8, 8, 0, 0.7, True), (1, 1, min(v, 32), 1.3, True),
                                                 (3, 2, min(v, r.choice([1, 2, 17])), 1.0, False)):
        g = gen(100 * i + pad)
        z = Buf(m, v, DT[dtype], pad, shift, randn(g, m, v) * 4)
        if masked and v > 4:
            z.t[torch.rand(m, v, generator=g, device="cuda") < 0.5] = -math.inf
            z.t[:, v // 2] = 1.0
        tokens = torch.randint(-2, v, (m,), generator=g, device="cuda").to(torch.int32)
        out = [torch.full((m,), math.nan, device="cuda") for _ in range(3)]
        tops = dict(top_logprob=torch.empty(m, top, device="cuda"), top_index=torch.empty(m, top, dtype=torch.int32, device="cuda")) if top else {}
        lib.emtk_logprobs(nn, z.t, tokens, *out, **tops, temperature=temperature)
        l, lp, entropy, lse = logprobs64(z.t, tokens, temperature)
        p = l.exp()
        l0 = torch.where(p > 0, l, 0.0)
        # exponents: |z - max| / T; S of v / 256 (or v / 2 lanes') terms a thread
        k = (v / 256 + 24 + (z.t.double().nan_to_num(0, 0, 0).abs().amax(1) / temperature) * 2) * E
        spread = 1 + (p * l0.square()).sum(1)
        assert torch.equal(torch.isinf(lp), torch.isinf(out[0]))
        fine = torch.isfinite(lp)
        near(out[0][fine], lp[fine], "f32", (k * (1 + lp.abs()))[fine], "logprob")
        near(out[1], entropy, "f32", k * 4 * spread, "entropy")
        near(out[2], lse, "f32", k * (1 + lse.abs()), "lse")
        if top:
            order = torch.sort(z.t.float(), dim=1, descending=True, stable=True).indices[:, :top]
            assert torch.equal(tops["top_index"].long(), order)
            want = l.gather(1, order)
            fine = torch.isfinite(want)
            assert torch.equal(fine, torch.isfinite(tops["top_logprob"]))
            near(tops["top_logprob"][fine], want[fine], "f32", (k[:, None] * (1 + want.abs()))[fine], "top_logprob")
        # the gradient
        dl, dh = randn(g, m), randn(g, m)
        for has_l, has_h in ((True, True), (True, False), (False, True)):
            dz = Buf(m, v, DT[dtype], pad, (shift + 1) if pad == 3 else shift)
            lib.emtk_logprobs_backward(nn, z.t, out[2], dz.t, tokens=tokens, d_logprob=dl if has_l else None, entropy=out[1],
                                       d_entropy=dh if has_h else None, temperature=temperature)
            given = (tokens >= 0)
            chosen = torch.zeros_like(l).scatter_(1, tokens.long().clamp(0)[:, None], given.double()[:, None])
            a = (dl.double() * given * has_l)[:, None]
            e = (dh.double() * has_h)[:, None]
            want = (a * (chosen - p) - e * p * (l0 + entropy[:, None])) / temperature
            size = (a.abs() * (chosen + p) + e.abs() * p * (l0.abs() + entropy[:, None] + 1)) / temperature
            near(dz.t, want, dtype, 8 * (k + lse.abs() * E)[:, None] * size + 1e-37, "d_logits")
            assert dz.surroundings_untouched()
        if pad != 3:
            lib.emtk_logprobs_backward(nn, z.t, out[2], z.t, tokens=tokens, entropy=out[1], d_entropy=dh, temperature=temperature)
            assert torch.equal(z.t, dz.t) and z.surroundings_untouched()


@pytest.mark.parametrize("v", [6, 300, 5000, 70000])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "f32"])
def test_logprobs_of_odd_rows(lib, nn, v, dtype):
    """Rows of one finite logit, of none, of the type's least value, of equal values, with NaN, with +infinity; tokens
    that are masked, absent or beyond the row."""
    low = torch.finfo(DT[dtype]).min
    z = torch.zeros(12, v, dtype=DT[dtype], device="cuda")
    z[0] = -math.inf
    z[0, 3] = 2.0
    z[1] = -math.inf
    z[2] = low
    z[3] = 1.5
    z[4, 2] = math.nan
    z[5, v - 1] = math.inf
    z[6] = low
    z[6, 4] = 0.0
    z[7] = -math.inf
    z[7, 1] = math.nan
    z[8] = torch.finfo(DT[dtype]).max
    z[9] = -0.0
    z[9, 1::2] = 0.0
    tokens = torch.tensor([3, 0, 1, v - 1, 0, 0, 4, 0, 2, 1, v, -1], dtype=torch.int32, device="cuda")
    lp, ent, lse = (torch.empty(12, device="cuda") for _ in range(3))
    tl, ti = torch.empty(12, 4, device="cuda"), torch.empty(12, 4, dtype=torch.int32, device="cuda")
    lib.emtk_logprobs(nn, z, tokens, lp, ent, lse, tl, ti)
    uniform = -math.log(v)
    for row, l, h in ((0, 0.0, 0.0), (2, uniform, -uniform), (3, uniform, -uniform), (6, 0.0, 0.0), (8, uniform, -uniform), (9, uniform, -uniform)):
        assert abs(float(lp[row]) - l) <= 64 * E * (1 + abs(l)) and abs(float(ent[row]) - h) <= 64 * E * (1 + h), row
    assert float(lp[1]) == -math.inf and float(ent[1]) == 0 and float(lse[1]) == -math.inf
    for row in (4, 5, 7):
        assert math.isnan(float(lp[row])) and math.isnan(float(ent[row])) and math.isnan(float(lse[row])) and torch.isnan(tl[row]).all()
    assert math.isnan(float(lp[10])) and float(lp[11]) == 0.0
    assert ti[0].tolist() == [3, 0, 1, 2] and tl[0].tolist()[1:] == [-math.inf] * 3 and abs(float(tl[0, 0])) <= 64 * E
    assert ti[1].tolist() == [0, 1, 2, 3] and tl[1].tolist() == [-math.inf] * 4
    for row in (2, 3, 8, 9):
        assert ti[row].tolist() == [0, 1, 2, 3]
    assert ti[4].tolist() == [0, 1, 3, 4] and ti[5].tolist()[0] == v - 1 and ti[7].tolist() == [0, 2, 3, 4]
    dz = torch.empty_like(z)
    one = torch.ones(12, device="cuda")
    lib.emtk_logprobs_backward(nn, z, lse, dz, tokens=tokens, d_logprob=one, entropy=ent, d_entropy=one)
    assert not dz[1].any() and not dz[0].any()  # nothing to move
    assert torch.isnan(dz[4]).all() and torch.isfinite(dz[[2, 3, 6, 8, 9, 10, 11]]).all()
    want = torch.full((v,), -1 / v, dtype=torch.float64, device="cuda")
    want[v - 1] += 1
    near(dz[3], want, dtype, 256 * E * want.abs() + 256 * E / v)
    assert dz[10].abs().max() <= 64 * E and dz[11].abs().max() <= 64 * E  # a uniform row's entropy has no slope


def test_equal_logits_come_in_order(lib, nn):
    """Few values, many of them equal: the lowest index first, whatever the row's length and start."""
    for m, v, shift in ((3, 40, 1), (2, 700, 0), (2, 5003, 3), (1, 100001, 0), (400, 700, 3), (2100, 4001, 1)):
        z = Buf(m, v, torch.bfloat16, 1, shift, torch.randint(-3, 4, (m, v), generator=gen(v), device="cuda").float())
        tl, ti = torch.empty(m, 32, device="cuda"), torch.empty(m, 32, dtype=torch.int32, device="cuda")
        lib.emtk_logprobs(nn, z.t, top_logprob=tl, top_index=ti)
        assert torch.equal(ti.long(), torch.sort(z.t.float(), dim=1, descending=True, stable=True).indices[:, :32])
    rising = torch.arange(60000, device="cuda", dtype=torch.float32)[None].contiguous()  # each is the largest yet
    tl, ti = torch.empty(1, 20, device="cuda"), torch.empty(1, 20, dtype=torch.int32, device="cuda")
    lib.emtk_logprobs(nn, rising, top_logprob=tl, top_index=ti)
    assert ti[0].tolist() == list(range(59999, 59979, -1))


@pytest.mark.parametrize("m,v", [(6, 9), (40, 20), (5, 150), (5, 300), (300, 600), (6, 1100), (5, 20000), (5, 50257)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "f32"])
def test_the_largest_beside_nan(lib, nn, m, v, dtype):
    """Rows of NaN, with fewer logits above it than are asked for, and with NaN alone where a row begins and ends: NaN counts
    as the least logit, and every answer is one of the row's columns."""
    g = gen(v)
    for top in (1, 2, 5, 21, 32):
        if top > v:
            continue
        for pad, shift in ((0, 0), (1, 0), (3, 5)):
            rows = torch.full((5, v), math.nan, device="cuda")
            few = torch.linspace(8, v - 9, top - 1).long().unique() if v > 64 else torch.arange(1, min(v - 1, top))
            rows[1, few.cuda()] = randn(g, len(few))
            rows[2, min(7, v // 3):max(v - 7, v - v // 3)] = -math.inf
            rows[3, v // 2:v // 2 + top - 1] = randn(g, rows[3, v // 2:v // 2 + top - 1].shape[0])
            rows[4, v // 2] = -math.inf
            z = Buf(m, v, DT[dtype], pad, shift, rows[torch.arange(m, device="cuda") % 5])
            tl, ti = torch.zeros(m, top, device="cuda"), torch.full((m, top), -7, dtype=torch.int32, device="cuda")
            lib.emtk_logprobs(nn, z.t, top_logprob=tl, top_index=ti)
            x = z.t.float().cpu().numpy()
            nan = np.isnan(x)
            want = np.stack([np.lexsort((np.arange(v), -np.where(nan[i], 0, x[i]), nan[i]))[:top] for i in range(min(m, 40))])
            assert np.array_equal(ti[:40].cpu().numpy(), want), (top, pad, shift)
            assert torch.equal(ti, ti[torch.arange(m, device="cuda") % 5]), (top, pad, shift)
            assert torch.isnan(tl).all()


def test_the_smallest_temperature(lib, nn):
    """All but the largest logits have probability 0, and nothing is NaN."""
    t = 4.3e-39
    z = torch.tensor([[0.0, -1.0, 0.0, -math.inf], [3.0, 2.0, 1.0, 3.0]], device="cuda")
    tokens = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    lp, ent = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    lib.emtk_logprobs(nn, z, tokens, lp, ent, temperature=t)
    assert (lp + math.log(2)).abs().max() <= 8 * E and (ent - math.log(2)).abs().max() <= 8 * E


@pytest.mark.parametrize("dtype,v", [("f32", 1 << 29), ("f32", (1 << 29) + 3), ("bf16", 1 << 30)])
def test_rows_of_two_gigabytes(lib, nn, dtype, v):
    """One row whose bytes pass 31 bits: its pieces go to all threads, and every element is written."""
    z = torch.zeros(1, v, dtype=DT[dtype], device="cuda")
    z[0, v - 1] = 3.0
    dz = torch.full_like(z, math.nan)
    lse, tl, ti = torch.empty(1, device="cuda"), torch.empty(1, 1, device="cuda"), torch.empty(1, 1, dtype=torch.int32, device="cuda")
    lib.emtk_logprobs(nn, z, lse=lse, top_logprob=tl, top_index=ti)
    total = v - 1 + math.exp(3.0)
    assert ti.item() == v - 1 and abs(lse.item() - math.log(total)) <= 64 * E * math.log(total)
    lib.emtk_logprobs_backward(nn, z, lse, dz, tokens=ti.view(-1), d_logprob=torch.ones(1, device="cuda"))
    assert not torch.isnan(dz).any()
    want = torch.full((3000,), -1 / total, dtype=torch.float64, device="cuda")
    for part in (slice(0, 3000), slice(v // 2, v // 2 + 3000), slice(v - 3001, v - 1)):
        near(dz[0, part], want, dtype, 64 * 21 * E / total)
    near(dz[0, v - 1:], 1 - torch.full((1,), math.exp(3.0) / total, dtype=torch.float64, device="cuda"), dtype, 4 * E)


@pytest.mark.parametrize("temperature", [1.0, 0.8, 0.01])
@pytest.mark.parametrize("m,v", [(7, 5), (40, 33), (70, 500), (300, 600), (9, 2500), (7, 40000), (700, 4100), (3000, 1100)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "f32"])
def test_gradient_of_logits_far_from_zero(lib, nn, m, v, temperature, dtype):
    """Rows far from 0, of the type's least and largest values, and small temperatures: p is held as well as it is by the
    row's own maximum and sum.  With T as fp32 has it, l' = (z - max) / T and l = l' - ln S: l' is off by 1.5 E |l'| <= 1.5 E |l|,
    ln S by the v / 256 + 24 roundings of a sum of exponentials, 3 E for exp and 8 E where lse is used as it is
    (up to 32), so p by (v / 256 + 48 + 4 |l|) E of itself; p = 0 beyond |l| = 104.  The entropy that is handed on is off by
    such parts of its terms p and p l."""
    t = float(np.float32(temperature))
    g = gen(v)
    low, high = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max
    rows = randn(g, 7, v)
    rows[0] = low
    rows[1] = low
    rows[1, v // 2] = -math.inf
    rows[2] += {"bf16": 100.0, "fp16": 1000.0, "f32": 1e5}[dtype]
    rows[3] -= {"bf16": 100.0, "fp16": 1000.0, "f32": 1e5}[dtype]
    rows[4] = high
    rows[5] *= 4
    rows[6, v - 1] = 40.0
    z = Buf(m, v, DT[dtype], 1, 1, rows[torch.arange(m, device="cuda") % 7])
    tokens = torch.randint(-1, v, (m,), generator=g, device="cuda").to(torch.int32)
    dl, dh = randn(g, m), randn(g, m)
    ent, lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    lib.emtk_logprobs(nn, z.t, entropy=ent, lse=lse, temperature=t)
    l = torch.log_softmax(z.t.double() / t, 1)
    p = l.exp()
    l0 = torch.where(p > 0, l, 0.0).clamp_min(-1e4)
    entropy = -(p * l0).sum(1, keepdim=True)
    given = tokens >= 0
    chosen = torch.zeros_like(l).scatter_(1, tokens.long().clamp(0)[:, None], given.double()[:, None])
    a, e = (dl.double() * given)[:, None], dh.double()[:, None]
    want = (a * (chosen - p) - e * p * (l0 + entropy)) / t
    off = (v / 256 + 48 + 4 * l0.abs().clamp_max(104)) * E
    off_h = (v / 256 + 48 + 4 * 104) * E * (1 + (p * l0.square()).sum(1, keepdim=True))
    size = a.abs() * (chosen + p) + e.abs() * p * (l0.abs() + entropy + 1)
    slack = (a.abs() * p * off + e.abs() * p * ((l0.abs() + entropy + 1) * off + off_h) + 4 * E * size) / t + 1e-33
    dz = Buf(m, v, DT[dtype], 1, 1)
    lib.emtk_logprobs_backward(nn, z.t, lse, dz.t, tokens=tokens, d_logprob=dl, entropy=ent, d_entropy=dh, temperature=t)
    near(dz.t, want, dtype, slack, "d_logits")
    assert dz.surroundings_untouched()
    lib.emtk_logprobs_backward(nn, z.t, lse, z.t, tokens=tokens, d_logprob=dl, entropy=ent, d_entropy=dh, temperature=t)
    assert torch.equal(z.t, dz.t) and z.surroundings_untouched()


@pytest.mark.parametrize("m,v", [(1, 300007), (41, 102213), (600, 20000), (300, 2500)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_in_place_has_the_same_bits(lib, nn, m, v, dtype):
    """Rows far from 0 among ordinary ones, cut among blocks or not: the same bits in the logits' place as apart."""
    g = gen(m)
    z = (randn(g, m, v) * 2 - 500.0 * (torch.arange(m, device="cuda") % 3 != 1)[:, None]).to(DT[dtype])
    ent, lse, dl = torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), randn(g, m)
    tokens = torch.randint(0, v, (m,), generator=g, device="cuda").to(torch.int32)
    lib.emtk_logprobs(nn, z, entropy=ent, lse=lse, temperature=0.7)
    assert bool((lse[::3] < -32).all()) and bool((lse[1::3].abs() < 32).all())
    dz = torch.empty_like(z)
    args = dict(tokens=tokens, d_logprob=dl, entropy=ent, d_entropy=dl, temperature=0.7)
    lib.emtk_logprobs_backward(nn, z, lse, dz, **args)
    lib.emtk_logprobs_backward(nn, z, lse, z, **args)
    assert torch.equal(z, dz)


@pytest.mark.parametrize("v", [5, 700, 3000, 40000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logprobs_across_the_types_range(lib, nn, v, dtype):
    """The type's least value beside its largest at a temperature that brings their distance into fp32: l is finite."""
    top, t = torch.finfo(DT[dtype]).max, 20.0
    z = torch.full((2, v), -top, dtype=DT[dtype], device="cuda")
    z[:, 3] = top
    z[1, 4] = top / 2
    tokens = torch.tensor([1, 4], dtype=torch.int32, device="cuda")
    lp, tl, ti = torch.empty(2, device="cuda"), torch.empty(2, 3, device="cuda"), torch.empty(2, 3, dtype=torch.int32, device="cuda")
    lib.emtk_logprobs(nn, z, tokens, lp, top_logprob=tl, top_index=ti, temperature=t)
    want = torch.log_softmax(z.double() / t, 1)
    near(lp, want.gather(1, tokens.long()[:, None])[:, 0], "f32", 8 * E * float(top) / 10)
    assert ti.tolist() == [[3, 0, 1], [3, 4, 0]]
    near(tl, want.gather(1, ti.long()), "f32", 8 * E * want.gather(1, ti.long()).abs())


def test_logprobs_of_empty_sizes(lib, nn):
    lib.emtk_logprobs(nn, torch.empty(0, 5, device="cuda"), entropy=torch.empty(0, device="cuda"))
    lp, ent, lse = (torch.empty(3, device="cuda") for _ in range(3))
    none = torch.empty(3, 0, device="cuda")
    lib.emtk_logprobs(nn, none, torch.tensor([-1, 0, 5], dtype=torch.int32, device="cuda"), lp, ent, lse)
    assert float(lp[0]) == 0 and torch.isnan(lp[1:]).all() and not ent.any() and bool((lse == -math.inf).all())
    lib.emtk_logprobs_backward(nn, none, lse, torch.empty(3, 0, device="cuda"))


# ------------------------------------------------------------------ recurrence
def act64(act, z):
    return {"none": lambda: z, "relu": lambda: torch.relu(z), "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z),
            "sigmoid": lambda: torch.sigmoid(z)}[act]()


def slope64(act, z):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(),
            "gelu": lambda: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
            "silu": lambda: s + z * s * (1 - s), "sigmoid": lambda: s * (1 - s)}[act]()


def recur64(f, x, o, dy, at, h0, dlast, act):
    """Everything of both passes, by the definition, one step of all sequences at a time; and each gradient's
    magnitude (the sums with their terms' magnitudes)."""
    rows, n = f.shape
    seqs = len(at) - 1
    a, b = torch.sigmoid(f), torch.sigmoid(-f)
    h = h0.clone()
    before, states = torch.zeros_like(f), torch.zeros_like(f)
    steps = max([at[i + 1] - at[i] for i in range(seqs)] + [0])
    who = [[i for i in range(seqs) if at[i + 1] - at[i] > t] for t in range(steps)]
    for t in range(steps):
        row = [at[i] + t for i in who[t]]
        before[row] = h[who[t]]
        h[who[t]] = a[row] * h[who[t]] + b[row] * x[row]
        states[row] = h[who[t]]
    gate = act64(act, o) if o is not None else torch.ones_like(f)
    g, mag, err = dlast.clone(), dlast.abs(), torch.zeros_like(dlast)
    out = dict(y=states * gate, last=h, states=states, before=before, dx=torch.zeros_like(f), df=torch.zeros_like(f), mag=torch.zeros_like(f), err=torch.zeros_like(f))
    for t in reversed(range(steps)):
        row = [at[i] + t for i in who[t]]
        g[who[t]] += gate[row] * dy[row]
        mag[who[t]] += (gate[row] * dy[row]).abs()
        out["dx"][row] = b[row] * g[who[t]]
        out["df"][row] = g[who[t]] * (before[row] - x[row]) * a[row] * b[row]
        out["mag"][row] = mag[who[t]]
        out["err"][row] = err[who[t]]
        g[who[t]] *= a[row]
        err[who[t]] = a[row] * err[who[t]] + (8 + 4 * f[row].abs()) * E * b[row] * mag[who[t]]
        mag[who[t]] *= a[row]
    out.update(dstate=g, dstate_mag=mag, dstate_err=err, do=dy * states * slope64(act, o) if o is not None else None)
    return out


def recur_case(i):
    r = random.Random(50 + i)
    lengths = r.choice([[1], [5], [8], [9], [127], [128], [129], [300], [700], [1025], [2600], [1] * 70, [3] * 40, [8] * 9, [64] * 5, [130] * 3, [300] * 20,
                        [5, 0, 131, 1, 260, 0], [0, 0], [2000, 3, 700], [1] * 5 + [0] * 3 + [1200]])
    if i >= 48:  # short ones on average, one of them long; lots of steps that end inside one; runs without steps
        lengths = [[1] * 300 + [1500], [2, 0, 7, 9, 8, 16, 17, 0, 1], [24] * 90, [100] * 60, [1, 40, 17, 16, 130] * 12,
                   [64, 63, 0, 1] * 9 + [129, 2, 0, 65, 63, 5], [16] * 650, [63] * 620, [1] * 64 + [64] + [0] * 5 + [700] + [9] * 70][i - 48]
    uniform = len(set(lengths)) == 1 and lengths[0] > 0
    return dict(lengths=lengths, offsets=not uniform or r.random() < 0.4, lead=r.choice([0, 0, 3]), tail=r.choice([0, 0, 5]),
                n=r.choice([1, 2, 7, 31, 32, 33, 64, 100]), act=r.choice(["none", "relu", "gelu", "silu", "sigmoid"]), gated=r.random() < 0.7,
                state=r.random() < 0.6, pad=r.choice([0, 0, 1, 2, 8]), shift=r.choice([0, 0, 1, 2]), f=r.choice([(1.5, 2.0), (1.0, 6.0), (4.0, 0.0), (0.5, -3.0)]))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("i", range(57))
def test_recurrence(lib, nn, i, dtype):
    """Both passes.  An error of b of a few E (and |f| E, of the exponential) moves the state by so much of max |x - h|;
    the roundings of a step stay for as long as the state does, at most min(T, 1 / b) steps.  A step passes g - b g on,
    off by b's error: (8 + 4 |f|) E b |g|, which later factors shrink as they do g (`err`); where a = 1 - b is small that
    is more than so much of a g."""
    c = recur_case(i)
    lead, tail = (c["lead"], c["tail"]) if c["offsets"] else (0, 0)
    at = np.cumsum([lead] + c["lengths"]).tolist()
    rows, n, seqs = at[-1] + tail, c["n"], len(c["lengths"])
    g, t = gen(i), DT[dtype]
    buf = lambda scale=1.0, about=0.0: Buf(rows, n, t, c["pad"], c["shift"], randn(g, rows, n) * scale + about)  # noqa: E731
    f, x, dy = buf(*c["f"]), buf(), buf(0.5)
    o = buf() if c["gated"] else None
    act = c["act"] if c["gated"] else "none"
    state = randn(g, seqs, n) if c["state"] else None
    dlast = randn(g, seqs, n) if c["state"] else None
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda") if c["offsets"] else None
    y, df, dx, do = (Buf(rows, n, t, c["pad"], c["shift"]) for _ in range(4))
    last, dstate = torch.empty(seqs, n, device="cuda"), torch.empty(seqs, n, device="cuda")
    states = lib.emtk_recurrence_states(rows, n, seqs)
    shared = dict(o=o.t if o else None, act=act, seqs=seqs, offsets=offsets)
    lib.emtk_recurrence(nn, f.t, x.t, y.t, state=state, last=last, states=states, **shared)
    lib.emtk_recurrence_backward(nn, dy.t, f.t, x.t, states, df.t, dx.t, d_last=dlast, d_o=do.t if o else None, d_state=dstate, **shared)
    zero = torch.zeros(seqs, n, dtype=torch.float64, device="cuda")
    want = recur64(f.t.double(), x.t.double(), o.t.double() if o else None, dy.t.double(), at, zero + state.double() if c["state"] else zero,
                   dlast.double() if c["state"] else zero, act)
    f64, x64 = f.t.double(), x.t.double()
    b = torch.sigmoid(-f64)
    fmax = float(f64.abs().max()) if rows else 0.0
    life = min(max(c["lengths"]), 1 / float(b.min()) if rows else 1.0)
    k = (24 + 4 * fmax + life) * E
    top = max(float(x64.abs().max()) if rows else 0.0, float(state.abs().max()) if c["state"] else 0.0)
    inside = slice(at[0], at[-1])
    z = o.t.double() if o else None
    gate = act64(act, z) if o else 1.0
    ka = (8 + 4 * z.abs()) * E if o else 0.0
    near(last, want["last"], "f32", k * top, "last")
    near(y.t[inside], want["y"][inside], dtype, (k * top * (abs(gate) + 1) + ka * want["states"].abs() * (1 + abs(gate)))[inside] if o else k * top, "y")
    kd = k + (ka if o else 0.0)
    mag = want["mag"] + (0 if not o else dy.t.double().abs())  # an activation's own error is of 1 + its value
    near(dx.t[inside], want["dx"][inside], dtype, (2 * kd * mag * b)[inside] + (want["err"] * b)[inside], "dx")
    ab = torch.sigmoid(f64) * b
    size = (want["before"] - x64).abs() * mag * ab
    near(df.t[inside], want["df"][inside], dtype, (4 * kd * size + (2 * k * top * mag + want["err"] * (want["before"] - x64).abs()) * ab)[inside], "df")
    near(dstate, want["dstate"], "f32", 4 * (k + 16 * E) * (want["dstate_mag"] + want["dstate"].abs()) + want["dstate_err"] + (16 * E * 4 if o else 0.0), "d_state")
    if o:
        s = slope64(act, z)
        near(do.t[inside], want["do"][inside], dtype,
             (dy.t.double().abs() * (2 * k * top * (s.abs() + 1) + ka * (1 + s.abs()) * want["states"].abs()))[inside], "d_o")
    for out in (y, df, dx) + ((do,) if o else ()):
        assert out.surroundings_untouched()
        assert torch.isnan(out.t[:at[0]].float()).all() and torch.isnan(out.t[at[-1]:].float()).all()  # of no sequence
    again = torch.empty_like(y.t)
    if c["state"]:  # last may be the state; states may be absent
        kept = state.clone()
        lib.emtk_recurrence(nn, f.t, x.t, y.t, state=kept, last=kept, **shared)
        assert torch.equal(kept, last)
    again.copy_(y.t)
    lib.emtk_recurrence(nn, f.t, x.t, y.t, state=state, **shared)
    assert torch.equal(torch.nan_to_num(again), torch.nan_to_num(y.t))


def test_recurrence_step_by_step_is_the_whole(lib, nn):
    """Served one token at a time with the state in hand, in pieces, or in one call: the same within the roundings."""
    seqs, T, n = 6, 300, 96
    g = gen(3)
    f, x, o = ((randn(g, seqs, T, n) * s + m).to(torch.bfloat16) for s, m in ((1.0, 3.0), (1.0, 0.0), (1.0, 0.0)))
    y, last = torch.empty(seqs * T, n, dtype=torch.bfloat16, device="cuda"), torch.empty(seqs, n, device="cuda")
    flat = lambda v: v.reshape(-1, n).contiguous()  # noqa: E731
    lib.emtk_recurrence(nn, flat(f), flat(x), y, o=flat(o), act="silu", seqs=seqs, last=last)
    for step in (1, 7, 60):
        state = torch.zeros(seqs, n, device="cuda")
        parts = []
        for t in range(0, T, step):
            cut = [flat(v[:, t:t + step]) for v in (f, x, o)]
            out = torch.empty_like(cut[0])
            lib.emtk_recurrence(nn, cut[0], cut[1], out, o=cut[2], act="silu", seqs=seqs, state=state, last=state)
            parts.append(out.view(seqs, -1, n))
        whole = torch.cat(parts, 1).reshape(-1, n)
        top = float(x.float().abs().max())
        assert (state - last).abs().max() <= 2 * (40 + 300) * E * top
        near(whole, y.double(), "bf16", 2.0 ** -8 * y.double().abs() + 4 * 340 * E * top)


@pytest.mark.parametrize("pad", [0, 1, 3])
def test_recurrence_of_many_values(lib, nn, pad):
    """Large enough that inputs off the 16-byte grid are copied first: the same bits as on it, and nothing beside the outputs."""
    lengths = [5000, 0, 17, 4200, 1401]
    at = np.cumsum([0] + lengths).tolist()
    rows, n, seqs = at[-1], 1000, len(lengths)
    g = gen(7)
    vals = [(randn(g, rows, n) + (2.0 if i == 0 else 0.0)).to(torch.bfloat16) for i in range(4)]
    assert rows * n >= 10 << 20
    results = []
    for p in (0, pad):
        f, x, o, dy = (Buf(rows, n, torch.bfloat16, p, 0, v) for v in vals)
        outs = [Buf(rows, n, torch.bfloat16, p, 0) for _ in range(4)]
        for offsets in (torch.tensor(at, dtype=torch.int32, device="cuda"), None):
            k = seqs if offsets is not None else 2
            kept = lib.emtk_recurrence_states(rows, n, k)
            shared = dict(o=o.t, act="gelu", seqs=k, offsets=offsets)
            lib.emtk_recurrence(nn, f.t, x.t, outs[0].t, states=kept, **shared)
            lib.emtk_recurrence_backward(nn, dy.t, f.t, x.t, kept, outs[1].t, outs[2].t, d_o=outs[3].t, **shared)
            results.append([b.t.clone() for b in outs])
            assert all(b.surroundings_untouched() for b in outs)
    for i in range(2):
        assert all(torch.equal(a, z) for a, z in zip(results[i], results[2 + i]))


def test_far_gates(lib, nn):
    """Forget gates that keep all (f = 100, infinity), nothing (f = -100, -infinity), and one state among many: finite,
    exact at the ends; NaN stays in its column from its step on."""
    T, n = 400, 40
    f = torch.full((T, n), 100.0, dtype=torch.float16, device="cuda")
    f[:, 1] = math.inf
    f[:, 2] = -100.0
    f[:, 3] = -math.inf
    f[150, 4] = math.nan
    x = randn(gen(1), T, n).to(torch.float16)
    state = randn(gen(2), 1, n)
    y, last, states = torch.empty_like(x), torch.empty(1, n, device="cuda"), lib.emtk_recurrence_states(T, n, 1)
    lib.emtk_recurrence(nn, f, x, y, state=state, last=last, states=states)
    kept = state.to(torch.float16)[0]
    for c in (0, 1, 5, n - 1):
        assert torch.equal(y[:, c], kept[c].expand(T)) and float(last[0, c]) == float(state[0, c])
    for c in (2, 3):
        assert torch.equal(y[:, c], x[:, c]) and float(last[0, c]) == float(x[-1, c])
    assert torch.equal(y[:150, 4], kept[4].expand(150)) and torch.isnan(y[150:, 4]).all()
    df, dx, dstate = torch.empty_like(x), torch.empty_like(x), torch.empty(1, n, device="cuda")
    dy = torch.ones_like(x)
    lib.emtk_recurrence_backward(nn, dy, f, x, states, df, dx, d_state=dstate)
    assert not df[:, [0, 1, 2, 3, 5]].any() and not dx[:, [0, 1, 5]].any() and bool((dx[:, [2, 3]] == 1).all())
    assert float(dstate[0, 0]) == T and float(dstate[0, 1]) == T and not dstate[0, 2:4].any()


@pytest.mark.parametrize("T,seqs", [(6, 1), (300, 1), (300, 40), (20000, 1)])
def test_slopes_of_gates_that_keep_nearly_all(lib, nn, T, seqs):
    """f from 78 to 87: a (1 - a) = 1 - a to 33 digits, small but in bf16's range.  df = g (h - x) (1 - a) is off by (8 + 4 |f|) E of
    the exponential and a rounding for every step that g comes through."""
    n = 38
    rows = T * seqs
    f = (78 + 0.5 * (torch.arange(n, device="cuda") % 19)).to(torch.bfloat16).expand(rows, n).contiguous()
    x = torch.full((rows, n), -2.0 ** 40, dtype=torch.bfloat16, device="cuda")
    dy = torch.full((rows, n), 2.0 ** 60, dtype=torch.bfloat16, device="cuda")
    state = torch.full((seqs, n), 2.0 ** 40, device="cuda")
    y, df, dx = (torch.empty_like(x) for _ in range(3))
    states = lib.emtk_recurrence_states(rows, n, seqs)
    lib.emtk_recurrence(nn, f, x, y, seqs=seqs, state=state, states=states)
    lib.emtk_recurrence_backward(nn, dy, f, x, states, df, dx, seqs=seqs)
    g = 2.0 ** 60 * (T - torch.arange(T, device="cuda", dtype=torch.float64)).repeat(seqs)[:, None]
    b = torch.sigmoid(-f.double())
    off = (8 + 4 * 87 + T) * E
    near(dx, g * b, "bf16", off * g * b, "dx")
    want = g * 2.0 ** 41 * b * torch.sigmoid(f.double())
    near(df, want, "bf16", off * want, "df")


def test_long_memories_settle_right(lib, nn):
    """f = 12: a state that remembers 160,000 steps moves towards x by 6e-6 a step; what 1 - a loses in fp32 would show."""
    T, n = 20000, 32
    f, x = torch.full((T, n), 12.0, dtype=torch.bfloat16, device="cuda"), torch.ones(T, n, dtype=torch.bfloat16, device="cuda")
    y, last = torch.empty_like(x), torch.empty(1, n, device="cuda")
    lib.emtk_recurrence(nn, f, x, y, last=last)
    b = 1 / (1 + math.exp(12.0))
    want = 1 - (1 - b) ** T
    assert (last.double() - want).abs().max() <= 2e-5 * want  # 12 |f| E of the exponential, and a rounding for every tile


@pytest.mark.parametrize("rows", [150, 300])
def test_unsound_offsets_stay_inside(lib, nn, rows):
    """Offsets that fall, or lie outside the rows, are taken as within them: nothing outside is touched."""
    n = 40
    f, x = (Buf(rows, n, torch.bfloat16, 0, 0, randn(gen(s), rows, n)) for s in (1, 2))
    for offs in ([0, 200, 100, 300], [-5, 50, 400, 1000], [300, 300, 0, 0], [2 ** 31 - 1, -2 ** 31, 7, 290]):
        y, states, last = Buf(rows, n, torch.bfloat16), Buf(rows // 128 + 3, n, torch.float32), Buf(3, n, torch.float32)
        at = torch.tensor(offs, dtype=torch.int32, device="cuda")
        lib.emtk_recurrence(nn, f.t, x.t, y.t, seqs=3, offsets=at, states=states.t, last=last.t)
        torch.cuda.synchronize()
        assert y.surroundings_untouched() and states.surroundings_untouched() and last.surroundings_untouched()


# ------------------------------------------------------------------ together, graphs, streams
def test_calls_in_a_graph_with_new_random_numbers(lib):
    """A training step's calls captured once and replayed: other dropout each time by the offset on the device, other
    inputs, the same results as eager calls."""
    nn = lib.emtk_nn_create()
    m, n = 50, 200
    t = torch.bfloat16
    r, b, dh = (torch.empty(m, n, dtype=t, device="cuda") for _ in range(3))
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    w = torch.ones(n, device="cuda")
    outs = lambda: dict(y=torch.empty(m, n, dtype=t, device="cuda"), h=torch.empty(m, n, dtype=t, device="cuda"),  # noqa: E731
                        db=torch.empty(m, n, dtype=t, device="cuda"), dw=torch.empty(n, device="cuda"), lse=torch.empty(m, device="cuda"),
                        dz=torch.empty(m, n, dtype=t, device="cuda"), s=lib.emtk_recurrence_states(m, n, 2), q=torch.empty(m, n, dtype=t, device="cuda"))

    def work(o):
        drop = lib.Drop(0.3, 11, 1000, step)
        pre = lib.Norm("rms", w)
        lib.emtk_residual_norm(nn, r, b, o["y"], o["h"], pre=pre, drop=drop)
        lib.emtk_recurrence(nn, o["h"], b, o["q"], seqs=2, states=o["s"])
        lib.emtk_logprobs(nn, o["q"], lse=o["lse"])
        lib.emtk_logprobs_backward(nn, o["q"], o["lse"], o["dz"])
        lib.emtk_residual_norm_backward(nn, None, dh, o["y"], b, None, o["db"], pre=pre, drop=drop, dw_pre=o["dw"])

    fixed = outs()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        work(fixed)  # grows the workspace
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(fixed)
    last = None
    for i in range(3):
        g = gen(i)
        for v in (r, b, dh):
            v.copy_(randn(g, m, n))
        step.fill_(i)
        graph.replay()
        got = {k: v.clone() for k, v in fixed.items()}
        eager = outs()
        work(eager)
        torch.cuda.synchronize()
        for k in ("y", "h", "db", "dw", "lse", "dz", "q"):
            assert torch.equal(got[k], eager[k]), k
        dropped = factors(m, n, 0.3, 11, 1000 + i) == 0
        assert torch.equal(got["y"][dropped], r[dropped])
        assert last is None or not torch.equal(last, dropped)
        last = dropped
    assert lib.emtk_nn_check(nn) == lib.EMTK_OK
    del graph
    lib.emtk_nn_destroy(nn)


def test_gradients_of_logits_in_graphs(lib):
    """Captured as a handle's first call, in the logits' place and apart, and replayed in turn over ordinary and far rows: as eager."""
    nn, eager = lib.emtk_nn_create(), lib.emtk_nn_create()
    m, v = 20, 30000
    z, dz = torch.zeros(m, v, device="cuda"), torch.empty(m, v, device="cuda")
    lse, dl, tokens = torch.zeros(m, device="cuda"), torch.ones(m, device="cuda"), torch.arange(m, dtype=torch.int32, device="cuda")
    lib.emtk_logprobs_backward(eager, z, lse, dz, tokens=tokens, d_logprob=dl)  # kernels are loaded before a capture
    lib.emtk_logprobs_backward(eager, z, lse, z, tokens=tokens, d_logprob=dl)
    torch.cuda.synchronize()
    graphs = []
    for to in (dz, z):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            lib.emtk_logprobs_backward(nn, z, lse, to, tokens=tokens, d_logprob=dl)
    for i, about in enumerate((0.0, 300.0, -1e6, 3e38)):
        values = randn(gen(i), m, v) + about * (torch.arange(m, device="cuda") % 2)[:, None]
        z.copy_(values)
        lib.emtk_logprobs(eager, z, lse=lse)
        want = torch.empty_like(z)
        lib.emtk_logprobs_backward(eager, z, lse, want, tokens=tokens, d_logprob=dl)
        for graph, out in zip(graphs, (dz, z)):
            graph.replay()
            assert torch.equal(out, want), (about, out is z)
    torch.cuda.synchronize()
    del graphs, graph
    for h in (nn, eager):
        assert lib.emtk_nn_check(h) == lib.EMTK_OK
        lib.emtk_nn_destroy(h)


def test_on_another_stream(lib):
    """Calls on a side stream, after work there that they must wait for."""
    nn = lib.emtk_nn_create()
    side = torch.cuda.Stream()
    m, n = 3000, 2000
    a = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    h, y = torch.empty_like(a), torch.empty_like(a)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        big = torch.ones(8192, 8192, device="cuda")
        for _ in range(4):
            big = big @ big * 1e-4
        a.fill_(2.0)
        lib.emtk_residual_norm(nn, a, None, y, h, pre=lib.Norm("rms", None, None, 0.0), scale=0.5)
        lib.emtk_dropout(nn, h, y, lib.Drop(0.0, 1))
    side.synchronize()
    assert bool((y == 1).all())
    lib.emtk_nn_destroy(nn)


def test_offsets_past_32_bits(lib, nn):
    """A matrix of more than 2^32 bytes: its last rows."""
    m, n = 70000, 32768
    z = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    z[m - 1, n - 1] = 3.0
    lse, ti, tl = torch.empty(m, device="cuda"), torch.empty(m, 1, dtype=torch.int32, device="cuda"), torch.empty(m, 1, device="cuda")
    lib.emtk_logprobs(nn, z, lse=lse, top_index=ti, top_logprob=tl)
    assert ti[m - 1].item() == n - 1 and abs(float(lse[m - 1]) - math.log(n - 1 + math.exp(3.0))) < 1e-4
    lib.emtk_logprobs_backward(nn, z, lse, z, tokens=ti.view(-1), d_logprob=torch.ones(m, device="cuda"))
    assert abs(float(z[m - 1, n - 1]) - (1 - math.exp(3.0) / (n - 1 + math.exp(3.0)))) < 2.0 ** -8
    z.fill_(1.0)
    lib.emtk_dropout(nn, z, z, lib.Drop(0.5, 5))
    assert torch.equal(z[m - 1].double(), factors_of_row(m - 1, n, 0.5, 5))
    rows = m * n // 4096
    f = z.view(rows, 4096)
    f.zero_()
    x = torch.ones(rows, 4096, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    lib.emtk_recurrence(nn, f, x, y, seqs=rows // 4)
    assert torch.equal(y[-4:, 4095].float().cpu(), torch.tensor([0.5, 0.75, 0.875, 0.9375]))


def factors_of_row(i, n, p, seed):
    low = 0xffffffff
    out = torch.empty(n, dtype=torch.float64, device="cuda")
    t = round(p * 65536)
    bits = []
    for g in range(-(-n // 8)):
        for w in philox((g, i, 0, 0), (seed & low, seed >> 32)):
            bits += [w & 0xffff, w >> 16]
    return out.copy_(torch.tensor([0.0 if v < t else 65536 / (65536 - t) for v in bits[:n]], dtype=torch.float64))


def test_binding_refuses(lib, nn):
    e = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    f32 = torch.float32
    x = e(4, 16)
    bad = [
        lambda: lib.emtk_dropout(nn, x, e(4, 17), lib.Drop(0.1, 1)),
        lambda: lib.emtk_dropout(nn, x, e(4, 16, t=torch.float16), lib.Drop(0.1, 1)),
        lambda: lib.emtk_dropout(nn, x, x, lib.Drop(0.1, 1, 0, e(1, t=torch.int32))),
        lambda: lib.emtk_residual_norm(nn, x, None, e(4, 16), e(4, 16), pre=lib.Norm("batch")),
        lambda: lib.emtk_residual_norm(nn, x, None, e(4, 16), e(4, 16), pre=lib.Norm("rms", e(15))),
        lambda: lib.emtk_residual_norm(nn, x, x, e(4, 16), gate=e(3, 16), gate_every=2),
        lambda: lib.emtk_residual_norm(nn, x, x, e(4, 16), gate=e(2, 16), gate_every=-2),
        lambda: lib.emtk_residual_norm(nn),
        lambda: lib.emtk_residual_norm_backward(nn, x, None, None, x, None, x, d_gate=e(16)),
        lambda: lib.emtk_logprobs(nn, x, e(4, t=torch.int64), e(4, t=f32)),
        lambda: lib.emtk_logprobs(nn, x, e(4, t=torch.int32), e(4)),
        lambda: lib.emtk_logprobs(nn, e(4, 16, t=torch.float64)),
        lambda: lib.emtk_recurrence(nn, x, x, e(4, 16), act="tanh"),
        lambda: lib.emtk_recurrence(nn, x, x, e(4, 16), state=e(2, 16, t=f32)),
        lambda: lib.emtk_recurrence(nn, e(4, 16, t=f32), x, x),
        lambda: lib.emtk_recurrence(nn, x, x, e(4, 16), seqs=2, offsets=e(2, t=torch.int32)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    refused = [
        lambda: lib.emtk_dropout(nn, x, e(4, 16), lib.Drop(1.0, 1)),
        lambda: lib.emtk_dropout(nn, x, e(4, 16), lib.Drop(-0.1, 1)),
        lambda: lib.emtk_dropout(nn, x, e(4, 16), lib.Drop(math.nan, 1)),
        lambda: lib.emtk_residual_norm(nn, x, None, e(4, 16), e(4, 16)),  # h without a norm
        lambda: lib.emtk_residual_norm(nn, x, None, e(4, 16), None, pre=lib.Norm("rms")),
        lambda: lib.emtk_residual_norm(nn, x, None, e(4, 16), None, gate=e(16)),  # a gate without a block
        lambda: lib.emtk_residual_norm(nn, x, x, None, None),
        lambda: lib.emtk_residual_norm(nn, x, None, e(4, 16), e(4, 16), pre=lib.Norm("rms", None, None, -1.0)),
        lambda: lib.emtk_residual_norm(nn, e(4, 16), x, x, None),  # y is the block
        lambda: lib.emtk_residual_norm(nn, e(2, 16400), None, None, e(2, 16400), pre=lib.Norm("rms")),
        lambda: lib.emtk_residual_norm_backward(nn, x, None, None, None, e(4, 16), e(4, 16)),  # d_block without the block
        lambda: lib.emtk_residual_norm_backward(nn, x, x, None, None, e(4, 16), pre=lib.Norm("rms")),  # no y
        lambda: lib.emtk_logprobs(nn, x, e(4, t=torch.int32)),
        lambda: lib.emtk_logprobs(nn, x, top_logprob=e(4, 33, t=f32), top_index=e(4, 33, t=torch.int32)),
        lambda: lib.emtk_logprobs(nn, x, top_logprob=e(4, 17, t=f32), top_index=e(4, 17, t=torch.int32)),
        lambda: lib.emtk_logprobs(nn, x, entropy=e(4, t=f32), temperature=0.0),
        lambda: lib.emtk_logprobs(nn, x, entropy=e(4, t=f32), temperature=math.inf),
        lambda: lib.emtk_logprobs_backward(nn, x, None, e(4, 16)),
        lambda: lib.emtk_logprobs_backward(nn, x, e(4, t=f32), e(4, 16), d_logprob=e(4, t=f32)),
        lambda: lib.emtk_logprobs_backward(nn, x, e(4, t=f32), e(4, 16), d_entropy=e(4, t=f32)),
        lambda: lib.emtk_recurrence(nn, x, x, e(4, 16), seqs=3),  # 4 rows are not 3 equal sequences
        lambda: lib.emtk_recurrence(nn, x, x, x),
        lambda: lib.emtk_recurrence(nn, x, x, e(4, 16), act="silu"),  # an activation of nothing
        lambda: lib.emtk_recurrence_backward(nn, x, x, x, None, e(4, 16)),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(lib.EmtkError) as err:
            call()
            pytest.fail(f"call {i} was taken")
        assert err.value.status == lib.EMTK_ERR_ARG, i
