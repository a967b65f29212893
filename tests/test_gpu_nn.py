"""Dense layers, gated blocks and 8-bit checkpoints against their definitions in
64 bits.

Tolerances are error bounds, element by element, from the rounding model:
  - a sum of K products in fp32, in any order and with truncating additions, is
    off by at most K 2^-23 times the sum of the products' magnitudes;
  - activations and slopes change by at most 1.2 times their input's error and add
    (8 + 4 |z|) 2^-23 times (|value| + 1) of their own (a fast exponential);
  - a value stored in 16 bits is off by u |value| more (u = 2^-8 bf16, 2^-11 fp16;
    fp16 also 2^-25 absolute below its normal range);
  - a backward product takes dz rounded to 16 bits: u times the sum of the
    products' magnitudes.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"bf16": 0.0, "fp16": 2.0 ** -25}
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
    """A [rows][cols] view of a wider, possibly shifted buffer; what surrounds it is NaN and
    must stay as it was (inputs: must not be read into a result)."""

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


def act64(act, z):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "sigmoid":
        return torch.sigmoid(z)
    return z


def slope64(act, z):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if act == "sigmoid":
        s = torch.sigmoid(z)
        return s * (1 - s)
    return torch.ones_like(z)


def act_err(z, v, dz):
    """Error of an activation or slope v at z, whose own error is dz."""
    return 1.2 * dz + (8 + 4 * z.abs()) * E * (v.abs() + 1)


def stored(err, v, dtype):
    return err * (1 + U[dtype]) + U[dtype] * v.abs() + TINY[dtype]


def close(got, want, bound, what):
    got = got.double()
    assert not torch.isnan(got).any(), what
    over = (got - want).abs() - bound
    assert (over <= 0).all(), f"{what}: {int((over > 0).sum())} of {over.numel()} beyond the bound, worst by {over.max()}"


def held8(v):
    """The values an 8-bit checkpoint of v stands for (float64 in and out), by definition.  On the CPU:
    there ldexp is exact, the GPU's powers of two in float64 are not."""
    where, v = v.device, v.cpu()
    m, n = v.shape
    w = torch.zeros((m, -(-n // 32) * 32), dtype=torch.float64, device=v.device)
    w[:, :n] = torch.where(torch.isfinite(v), v, 0.0)
    w = w.view(m, -1, 32)
    _, e = torch.frexp(w.abs().amax(2, keepdim=True).clamp_min(2.0 ** -140))
    best = None
    for d in (-8, -7, -6):  # the least power whose largest quotient rounds to at most 127
        step = torch.ldexp(torch.ones_like(w[:, :, :1]), (e + d).clamp_min(-126))
        q = torch.round(w / step)
        fits = q.abs().amax(2, keepdim=True) <= 127
        best = torch.where(fits, step, torch.full_like(step, float("inf"))) if best is None else \
            torch.where(fits & (step < best), step, best)
    out = (torch.round(w / best) * best).view(m, -1)[:, :n]
    return torch.where(torch.isfinite(v), out, float("nan")).to(where)


def q8_of(lib, rows, cols, pad=0):
    codes = torch.full((rows, cols + pad), 77, dtype=torch.int8, device="cuda")
    nb = (cols + 31) // 32
    scales = torch.full((rows, nb + pad), 99, dtype=torch.uint8, device="cuda")
    return lib.Q8(codes[:, :cols], scales[:, :nb])


def q8_values(q, cols):
    step = ((q.scales.long() - 127 + 1023) << 52).view(torch.float64).repeat_interleave(32, 1)[:, :cols]
    c = q.codes.double()
    return torch.where(c == -128, float("nan"), c * step)


# ------------------------------------------------------------------ forward
SHAPES = [(1, 1, 1), (1, 4096, 72), (2, 7, 5), (3, 777, 130), (5, 64, 512), (8, 2048, 96), (9, 200, 48), (16, 1000, 33),
          (17, 129, 65), (33, 72, 257), (64, 512, 128), (100, 2304, 40), (127, 2305, 131), (128, 128, 128),
          (129, 65, 257), (255, 64, 31), (300, 1000, 333), (513, 40, 1030), (1693, 48, 640), (20, 30011, 24),
          (256, 9292, 128), (24, 600, 1000), (47, 1000, 1200), (70, 2500, 700), (120, 2304, 515), (128, 2112, 4100), (2500, 700, 3000), (5000, 1032, 1100)]


def dense_inputs(m, k, n, dtype, pad, shift, seed, bias, residual):
    g = gen(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = DT[dtype]
    x = Buf(m, k, dt, pad, shift, r(m, k))
    w = Buf(n, k, dt, pad, shift, r(n, k) / math.sqrt(k))
    b = None if not bias else r(n).to(dt if bias == "16" else torch.float32)
    res = Buf(m, n, dt, pad, shift, r(m, n)) if residual else None
    return x, w, b, res


@pytest.mark.parametrize("i,shape", list(enumerate(SHAPES)))
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_dense(lib, nn, i, shape, dtype):
    m, k, n = shape
    for case in range(2):
        act = ("none", "relu", "gelu", "silu", "sigmoid")[(i + 2 * case) % 5]
        bias = (None, "16", "32")[(i + case) % 3]
        residual, saved = (i + case) % 2, (i // 2 + case) % 3
        pad, shift = ((0, 0), (8, 8), (3, 1))[(i + case) % 3]
        x, w, b, res = dense_inputs(m, k, n, dtype, pad, shift, 7 * i + case, bias, residual)
        y = Buf(m, n, DT[dtype], pad, shift)
        pre = None if saved == 0 else Buf(m, n, DT[dtype], pad, shift) if saved == 1 else q8_of(lib, m, n, pad)
        lib.emtk_dense(nn, x.t, w.t, y.t, bias=b, act=act, residual=res.t if res else None,
                       pre=pre.t if saved == 1 else pre)
        z = x.t.double() @ w.t.double().t()
        mag = x.t.double().abs() @ w.t.double().abs().t()
        if b is not None:
            z, mag = z + b.double(), mag + b.double().abs()
        dz = (k + 2) * E * mag
        a = act64(act, z)
        want, err = a, act_err(z, a, dz)
        if res:
            want = want + res.t.double()
            err = err + E * want.abs()
        close(y.t, want, stored(err, want, dtype), f"y of case {case}: {act} {bias} {residual} {pad}")
        assert y.surroundings_untouched()
        if saved == 1:
            close(pre.t, z, stored(dz, z, dtype), "pre")
            assert pre.surroundings_untouched()
        if saved == 2:  # half a step off; the step, at most 2 top / 127.5, may differ where top is at an edge
            top = torch.nn.functional.pad(z.abs() + dz, (0, -n % 32)).view(m, -1, 32).amax(2).repeat_interleave(32, 1)[:, :n]
            close(q8_values(pre, n), z, dz + top / 127.5 + 2.0 ** -126, "pre in 8 bits")
    assert lib.emtk_nn_check(nn) == lib.EMTK_OK


@pytest.mark.parametrize("i,shape", list(enumerate(SHAPES)))
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gated(lib, nn, i, shape, dtype):
    m, k, f = shape
    act = ("silu", "gelu", "relu", "sigmoid", "none")[i % 5]
    pad, shift = ((0, 0), (3, 1), (8, 8))[i % 3]
    x, wg, bg, _ = dense_inputs(m, k, f, dtype, pad, shift, i, (None, "32", "16")[i % 3], False)
    _, wu, bu, _ = dense_inputs(m, k, f, dtype, pad, shift, i + 1000, (None, "32", "16")[i % 3], False)
    saved = (i + (dtype == "bf16")) % 3
    h = Buf(m, f, DT[dtype], pad, shift)
    keep = [None, None] if saved == 0 else [Buf(m, f, DT[dtype], pad, shift) for _ in "gu"] if saved == 1 else \
        [q8_of(lib, m, f, pad) for _ in "gu"]
    lib.emtk_gated(nn, x.t, wg.t, wu.t, h.t, bias_gate=bg, bias_up=bu, act=act,
                   gate=keep[0].t if saved == 1 else keep[0], up=keep[1].t if saved == 1 else keep[1])
    zs, errs = [], []
    for w, b in ((wg, bg), (wu, bu)):
        z, mag = x.t.double() @ w.t.double().t(), x.t.double().abs() @ w.t.double().abs().t()
        if b is not None:
            z, mag = z + b.double(), mag + b.double().abs()
        zs.append(z)
        errs.append((k + 2) * E * mag)
    a = act64(act, zs[0])
    ea = act_err(zs[0], a, errs[0])
    want = a * zs[1]
    err = ea * (zs[1].abs() + errs[1]) + a.abs() * errs[1] + E * want.abs()
    close(h.t, want, stored(err, want, dtype), f"h {act}")
    assert h.surroundings_untouched()
    for z, e, kept in zip(zs, errs, keep):
        if saved == 1:
            close(kept.t, z, stored(e, z, dtype), "kept")
            assert kept.surroundings_untouched()
        if saved == 2:
            top = torch.nn.functional.pad(z.abs() + e, (0, -f % 32)).view(m, -1, 32).amax(2).repeat_interleave(32, 1)[:, :f]
            close(q8_values(kept, f), z, e + top / 127.5 + 2.0 ** -126, "kept in 8 bits")


# ------------------------------------------------------------------ gradients
BACK_SHAPES = [(1, 1, 1), (1, 300, 72), (2, 9, 33), (7, 130, 64), (16, 64, 257), (40, 257, 96), (128, 128, 128),
               (130, 72, 200), (235, 1000, 333), (300, 33, 520), (1000, 517, 130), (3000, 40, 24), (2500, 96, 16),
               (3000, 1104, 2504), (1500, 2503, 700)]


def keep(lib, nn, t, how, pad=0):
    """t as it is, or as an 8-bit checkpoint with the values that it stands for."""
    if how != "q8":
        return t.t, t.t.double()
    q = q8_of(lib, *t.t.shape, pad)
    lib.emtk_pack8(nn, t.t, q)
    return q, q8_values(q, t.t.shape[1])


def product_bound(a, b, terms_err, terms, dtype):
    """|error| of a @ b with a off by terms_err relative, before it is stored."""
    return (a.abs() @ b.abs()) * (terms_err + terms * E)


@pytest.mark.parametrize("i,shape", list(enumerate(BACK_SHAPES)))
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_dense_backward(lib, nn, i, shape, dtype):
    m, k, n = shape
    act = ("gelu", "none", "relu", "silu", "sigmoid")[i % 5]
    pad, shift = ((0, 0), (3, 1), (8, 8))[i % 3]
    held = ("16", "q8")[(i + (dtype == "fp16")) % 2]
    g = gen(i)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = DT[dtype]
    dy, x = Buf(m, n, dt, pad, shift, r(m, n)), Buf(m, k, dt, pad, shift, r(m, k))
    w, z = Buf(n, k, dt, pad, shift, r(n, k)), Buf(m, n, dt, pad, shift, 2 * r(m, n))
    dwt = torch.float32 if i % 2 else dt
    dx, dw = Buf(m, k, dt, pad, shift), Buf(n, k, dwt, pad, shift)
    db = torch.full((n,), float("nan"), dtype=torch.float32, device="cuda")
    xk, x64 = keep(lib, nn, x, held, pad)
    zk, z64 = keep(lib, nn, z, held, pad)
    lib.emtk_dense_backward(nn, dy.t, xk, w.t, act=act, pre=None if act == "none" else zk, dx=dx.t, dw=dw.t, db=db)
    s = slope64(act, z64)
    dz = dy.t.double() * s
    # error of dz in fp32, then its rounding to 16 bits (none without an activation)
    e32 = dy.t.double().abs() * act_err(z64, s, 0 * z64) if act != "none" else 0 * dz
    e16 = e32 + U[dtype] * dz.abs() + TINY[dtype] if act != "none" else 0 * dz
    w64 = w.t.double()
    err = e16 @ w64.abs() + n * E * ((dz.abs() + e16) @ w64.abs())
    want = dz @ w64
    close(dx.t, want, stored(err, want, dtype), "dx")
    err = e16.t() @ x64.abs() + m * E * ((dz.abs() + e16).t() @ x64.abs())
    want = dz.t() @ x64
    close(dw.t, want, stored(err, want, dtype) if dwt is dt else err + E * want.abs(), "dw")
    close(db, dz.sum(0), e32.sum(0) + m * E * (dz.abs() + e32).sum(0), "db")
    assert dx.surroundings_untouched() and dw.surroundings_untouched()
    # each output alone gives the same values
    one = torch.empty_like(dx.t)
    lib.emtk_dense_backward(nn, dy.t, None, w.t, act=act, pre=None if act == "none" else zk, dx=one)
    assert torch.equal(one, dx.t)
    one = torch.empty((n, k), dtype=dwt, device="cuda")
    lib.emtk_dense_backward(nn, dy.t, xk, None, act=act, pre=None if act == "none" else zk, dw=one)
    assert torch.equal(one, dw.t)
    one = torch.empty_like(db)
    lib.emtk_dense_backward(nn, dy.t, None, None, act=act, pre=None if act == "none" else zk, db=one)
    assert torch.equal(one, db)


@pytest.mark.parametrize("i,shape", list(enumerate(BACK_SHAPES)))
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gated_backward(lib, nn, i, shape, dtype):
    m, k, f = shape
    act = ("silu", "gelu", "relu", "sigmoid", "none")[i % 5]
    pad, shift = ((3, 1), (0, 0), (8, 8))[i % 3]
    held = ("q8", "16")[(i + (dtype == "fp16")) % 2]
    g = gen(100 + i)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = DT[dtype]
    dh, x = Buf(m, f, dt, pad, shift, r(m, f)), Buf(m, k, dt, pad, shift, r(m, k))
    wg, wu = Buf(f, k, dt, pad, shift, r(f, k)), Buf(f, k, dt, pad, shift, r(f, k))
    gate, up = Buf(m, f, dt, pad, shift, 2 * r(m, f)), Buf(m, f, dt, pad, shift, r(m, f))
    dwt = dt if i % 2 else torch.float32
    dx, dwg, dwu = Buf(m, k, dt, pad, shift), Buf(f, k, dwt, pad, shift), Buf(f, k, dwt, pad, shift)
    h = Buf(m, f, dt, pad, shift)
    dbg, dbu = (torch.full((f,), float("nan"), dtype=torch.float32, device="cuda") for _ in "gu")
    xk, x64 = keep(lib, nn, x, held, pad)
    gk, g64 = keep(lib, nn, gate, held, pad)
    uk, u64 = keep(lib, nn, up, held, pad)
    lib.emtk_gated_backward(nn, dh.t, gk, uk, xk, wg.t, wu.t, act=act, dx=dx.t, dw_gate=dwg.t, dw_up=dwu.t,
                            db_gate=dbg, db_up=dbu, h=h.t)
    d = dh.t.double()
    a, s = act64(act, g64), slope64(act, g64)
    own = 0 if act == "none" else 1
    ea, es = own * act_err(g64, a, 0 * g64), own * act_err(g64, s, 0 * g64)
    want = a * u64
    close(h.t, want, stored(ea * u64.abs() + E * want.abs(), want, dtype), "h")
    dg, du = d * u64 * s, d * a
    eg, eu = (d * u64).abs() * es + 2 * E * dg.abs(), d.abs() * ea + E * du.abs()
    rg, ru = (e + U[dtype] * v.abs() + TINY[dtype] for e, v in ((eg, dg), (eu, du)))
    wg64, wu64 = wg.t.double(), wu.t.double()
    want = dg @ wg64 + du @ wu64
    mag = (dg.abs() + rg) @ wg64.abs() + (du.abs() + ru) @ wu64.abs()
    close(dx.t, want, stored(rg @ wg64.abs() + ru @ wu64.abs() + (2 * f + 1) * E * mag, want, dtype), "dx")
    for name, got, v, rounded in (("dw_gate", dwg, dg, rg), ("dw_up", dwu, du, ru)):
        want = v.t() @ x64
        err = rounded.t() @ x64.abs() + m * E * ((v.abs() + rounded).t() @ x64.abs())
        close(got.t, want, stored(err, want, dtype) if dwt is dt else err + E * want.abs(), name)
        assert got.surroundings_untouched()
    for name, got, v, e in (("db_gate", dbg, dg, eg), ("db_up", dbu, du, eu)):
        close(got, v.sum(0), e.sum(0) + m * E * (v.abs() + e).sum(0), name)
    assert dx.surroundings_untouched() and h.surroundings_untouched()


def test_gradients_against_differences(lib, nn):
    """Gradients of L = sum(c * block(x)) against central differences of L in 64 bits, along random
    directions: the gradients are rounded sums, so the directional derivative is off by no more than
    the elements' bound (here 2^-6 of the summed magnitudes, three bf16 roundings with room)."""
    g = gen(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    m, k, f = 37, 48, 56
    t = torch.bfloat16
    x, wg, wu, c = r(m, k).to(t), (r(f, k) / 7).to(t), (r(f, k) / 7).to(t), r(m, f).to(t)
    for act in ("silu", "gelu", "sigmoid", "none"):
        h, gate, up = (torch.empty((m, f), dtype=t, device="cuda") for _ in range(3))
        lib.emtk_gated(nn, x, wg, wu, h, act=act, gate=gate, up=up)
        dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
        lib.emtk_gated_backward(nn, c, gate, up, x, wg, wu, act=act, dx=dx, dw_gate=dwg, dw_up=dwu)

        def loss(x_, g_, u_):
            return (c.double() * act64(act, x_ @ g_.t()) * (x_ @ u_.t())).sum()

        at = [v.double() for v in (x, wg, wu)]
        for which, grad in enumerate((dx, dwg, dwu)):
            for _ in range(4):
                v = r(*grad.shape).double()
                eps = 1e-4
                hi, lo = list(at), list(at)
                hi[which], lo[which] = at[which] + eps * v, at[which] - eps * v
                diff = (loss(*hi) - loss(*lo)) / (2 * eps)
                got = (grad.double() * v).sum()
                assert abs(got - diff) <= 2.0 ** -6 * (grad.double() * v).abs().sum(), (act, which)


# ------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("m,k,pad", [(1, 1, 0), (3, 32, 0), (2, 31, 1), (5, 33, 0), (4, 255, 3), (7, 256, 8), (9, 517, 0),
                                     (300, 2304, 0)])
def test_pack8_is_its_definition(lib, nn, dtype, m, k, pad):
    g = gen(m * k)
    x = torch.randn(m, k, generator=g, device="cuda")
    x *= torch.exp(4 * torch.randn(m, k, generator=g, device="cuda")) if m % 2 else 1  # wide range within a block
    x = Buf(m, k, DT[dtype], pad, pad % 2, x.clamp(-60000, 60000))
    q = q8_of(lib, m, k, pad)
    lib.emtk_pack8(nn, x.t, q)
    want = held8(x.t.double())
    assert torch.equal(q8_values(q, k), want)
    back = Buf(m, k, DT[dtype], pad, pad % 2)
    lib.emtk_unpack8(nn, q, back.t)
    assert torch.equal(back.t.double(), want.clamp(-65504, 65504).to(DT[dtype]).double() if dtype == "fp16" else want)
    assert back.surroundings_untouched()
    whole = q.codes._base
    if pad:
        assert bool((whole[:, k:] == 77).all()) and bool((q.scales._base[:, -pad:] == 99).all())


def test_pack8_edges(lib, nn):
    """Zeros, the edge where 127.5 would round to 128, subnormals, the largest values, infinities and NaN."""
    rows = [[0.0] * 32,
            [127.0, 64.0, -1.0, 0.5, 1.5] + [0.0] * 27,         # step 1: ties to even
            [127.5, 1.0] + [0.0] * 30,                          # 127.5 / 1 would round to 128: step 2
            [255.0 / 2 - 0.5, -127.0] + [0.0] * 30,
            [2.0 ** -130, 2.0 ** -126] + [0.0] * 30,
            [3.3e38, -1e38, 1.0] + [0.0] * 29,
            [float("inf"), 2.0, -float("inf"), float("nan")] + [1.0] * 28,
            [float("nan")] * 32]
    x = torch.tensor(rows, device="cuda").to(torch.bfloat16)
    q = q8_of(lib, len(rows), 32)
    lib.emtk_pack8(nn, x, q)
    got, want = q8_values(q, 32), held8(x.double())
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    assert q.codes[2, 0].item() == 64 and q.codes[1, 3].item() == 0 and q.codes[1, 4].item() == 2
    back = torch.empty_like(x)
    lib.emtk_unpack8(nn, q, back)
    assert torch.equal(torch.nan_to_num(back.double()), torch.nan_to_num(want))
    assert torch.equal(torch.isnan(back), torch.isnan(want))


def test_unpack8_saturates_in_fp16(lib, nn):
    x = torch.full((1, 32), 65504.0, dtype=torch.float16, device="cuda")
    q, back = q8_of(lib, 1, 32), torch.empty_like(x)
    lib.emtk_pack8(nn, x, q)
    lib.emtk_unpack8(nn, q, back)
    assert torch.equal(back, x)  # 64 * 2^10 = 65536 is beyond fp16


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("m,k,n", [(1, 128, 72), (64, 64, 64), (65, 96, 40), (300, 256, 130), (130, 400, 600),
                                   (1000, 2304, 128), (5000, 128, 300), (9000, 48, 24), (700, 1040, 1030)])
def test_gradients_from_codes_are_those_from_their_values(lib, nn, dtype, m, k, n):
    """x as an 8-bit checkpoint whose rows TMA can read, against x as the 16-bit matrix it stands for:
    the same products of the same values in the same order, so the same bits (with every block's scale
    different, and zero and NaN blocks)."""
    g = gen(m + k)
    t = DT[dtype]
    x = torch.randn(m, k, generator=g, device="cuda") * torch.exp2(torch.randint(-6, 7, (m, 1), generator=g, device="cuda"))
    x[m // 3] = 0
    x = x.to(t)
    q, values = q8_of(lib, m, k), torch.empty_like(x)
    lib.emtk_pack8(nn, x, q)
    lib.emtk_unpack8(nn, q, values)
    dy, w = (torch.randn(*s, generator=g, device="cuda").to(t) for s in ((m, n), (n, k)))
    a, b = torch.empty((n, k), dtype=t, device="cuda"), torch.zeros((n, k), dtype=t, device="cuda")
    c, d = torch.empty_like(x), torch.empty_like(x)
    lib.emtk_dense_backward(nn, dy, values, w, dx=c, dw=a)
    lib.emtk_dense_backward(nn, dy, q, w, dx=d, dw=b)
    assert torch.equal(a, b) and torch.equal(c, d)
    b.zero_()
    lib.emtk_dense_backward(nn, dy, values, None, dw=a)
    lib.emtk_dense_backward(nn, dy, q, None, dw=b)
    assert torch.equal(a, b)
    gate, up = (torch.randn(m, n, generator=g, device="cuda").to(t) for _ in "gu")
    outs = []
    for xx in (values, q):
        o = [torch.zeros((n, k), dtype=torch.float32, device="cuda") for _ in "gu"] + [torch.empty_like(x)]
        lib.emtk_gated_backward(nn, dy, gate, up, xx, w, w, act="silu", dw_gate=o[0], dw_up=o[1], dx=o[2])
        outs.append(o)
    assert all(torch.equal(p, r) for p, r in zip(*outs))
    x[0, 1] = float("nan")
    lib.emtk_pack8(nn, x, q)
    lib.emtk_dense_backward(nn, dy, q, None, dw=b)
    assert torch.isnan(b[:, 1]).all() and torch.equal(torch.isnan(b).any(0).nonzero().flatten().cpu(), torch.tensor([1]))


# ------------------------------------------------------------------ odd ends
@pytest.mark.parametrize("m,k,n", [(0, 8, 8), (4, 0, 40), (4, 8, 0), (0, 0, 0), (300, 0, 300)])
def test_empty_sizes(lib, nn, m, k, n):
    t = torch.bfloat16
    e = lambda *s: torch.full(s, 3.0, dtype=t, device="cuda")  # noqa: E731
    x, w, y, b, res = e(m, k), e(n, k), e(m, n), torch.linspace(-1, 1, n, device="cuda"), e(m, n)
    lib.emtk_dense(nn, x, w, y, bias=b, act="relu", residual=res)
    assert torch.equal(y, (torch.relu(b) + 3.0).to(t).expand(m, n))
    lib.emtk_gated(nn, x, w, w, y, bias_gate=b, bias_up=b, act="none")
    assert torch.equal(y, (b * b).to(t).expand(m, n))
    dx, dw, dw2 = e(m, k), e(n, k), e(n, k)
    db, db2 = (torch.full((n,), 5.0, device="cuda") for _ in "ab")
    lib.emtk_dense_backward(nn, e(m, n), x, w, act="relu", pre=e(m, n), dx=dx, dw=dw, db=db)
    assert torch.equal(db, torch.full((n,), 3.0 * m, device="cuda"))
    assert torch.equal(dx, torch.full_like(dx, 9.0 * n)) and torch.equal(dw, torch.full_like(dw, 9.0 * m))
    lib.emtk_gated_backward(nn, e(m, n), e(m, n), e(m, n), x, w, w, act="none", dx=dx, dw_gate=dw, dw_up=dw2,
                            db_gate=db, db_up=db2)
    assert torch.equal(db, torch.full((n,), 9.0 * m, device="cuda")) and torch.equal(db, db2)
    q = lib.emtk_q8_empty(m, k)
    lib.emtk_pack8(nn, x, q)
    lib.emtk_unpack8(nn, q, x)
    assert torch.equal(x, torch.full_like(x, 3.0))


def test_residual_may_be_the_output(lib, nn):
    g = gen(1)
    for m, k, n in ((1, 512, 96), (30, 100, 67), (300, 128, 512)):
        x, w, y = (torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16) for s in ((m, k), (n, k), (m, n)))
        apart = torch.empty_like(y)
        lib.emtk_dense(nn, x, w, apart, residual=y)
        lib.emtk_dense(nn, x, w, y, residual=y)
        assert torch.equal(y, apart)


@pytest.mark.parametrize("m", [1, 4, 24, 300])
def test_nan_and_infinity_stay_in_their_rows(lib, nn, m):
    g = gen(m)
    k, n = 200, 150
    x = torch.randn(m, k, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn(n, k, generator=g, device="cuda").to(torch.bfloat16)
    clean, y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda"), torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    for act in ("none", "relu", "silu"):
        lib.emtk_dense(nn, x, w, clean, act=act)
        bad = x.clone()
        bad[m // 2, 3] = float("nan")
        lib.emtk_dense(nn, bad, w, y, act=act)
        assert bool(torch.isnan(y[m // 2]).all())
        rest = torch.arange(m, device="cuda") != m // 2
        assert torch.equal(y[rest], clean[rest])
        bad[m // 2, 3] = float("inf")
        lib.emtk_dense(nn, bad, w, y, act=act)
        assert torch.equal(y[rest], clean[rest])
        if act == "relu":  # inf * w: +inf or 0
            assert torch.equal(y[m // 2] == float("inf"), w[:, 3] > 0)


def test_offsets_past_32_bits(lib, nn):
    """Rows far apart: the last element is more than 2^31 elements from the first."""
    m, k, n = 70000, 24, 40
    whole = torch.empty((m, 32768), dtype=torch.bfloat16, device="cuda")
    x = whole[:, :k]
    x.copy_(torch.randn(m, k, generator=gen(2), device="cuda"))
    w = torch.randn(n, k, generator=gen(3), device="cuda").to(torch.bfloat16)
    near, far = torch.empty((m, n), dtype=torch.bfloat16, device="cuda"), whole[:, 64:64 + n]
    lib.emtk_dense(nn, x.contiguous(), w, near)
    lib.emtk_dense(nn, x, w, far)
    assert torch.equal(near, far)
    dw, dw2 = torch.empty_like(w), torch.empty_like(w)
    lib.emtk_dense_backward(nn, near, x.contiguous(), w, dw=dw)
    lib.emtk_dense_backward(nn, far, x, w, dw=dw2)
    assert torch.equal(dw, dw2)
    q = lib.emtk_q8_empty(m, k)
    lib.emtk_pack8(nn, x, q)
    lib.emtk_unpack8(nn, q, whole[:, 128:128 + k])
    assert torch.equal(whole[:, 128:128 + k].double(), held8(x.double()))


def test_other_stream_and_repeats(lib):
    """On a stream of the caller's, several calls in flight, twice the same bits."""
    h = lib.emtk_nn_create(workspace_bytes=1 << 20)
    s = torch.cuda.Stream()
    g = gen(9)
    m, k, f = 333, 264, 520
    t = torch.bfloat16
    x, dh = torch.randn(m, k, generator=g, device="cuda").to(t), torch.randn(m, f, generator=g, device="cuda").to(t)
    wg, wu = (torch.randn(f, k, generator=g, device="cuda").div_(16).to(t) for _ in "gu")
    outs = []
    torch.cuda.synchronize()
    for _ in range(3):
        o = [torch.empty(sh, dtype=t, device="cuda") for sh in ((m, f), (m, f), (m, f), (m, k), (f, k), (f, k))]
        db = [torch.empty(f, device="cuda") for _ in "gu"]
        torch.cuda.synchronize()
        lib.emtk_gated(h, x, wg, wu, o[0], gate=o[1], up=o[2], stream=s)
        lib.emtk_gated_backward(h, dh, o[1], o[2], x, wg, wu, dx=o[3], dw_gate=o[4], dw_up=o[5], db_gate=db[0],
                                db_up=db[1], stream=s)
        outs.append(o + db)
    s.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
    assert lib.emtk_nn_check(h, s) == lib.EMTK_OK
    lib.emtk_nn_destroy(h)


def test_calls_in_a_graph(lib):
    """With the workspace reserved, a training step is captured once and replayed on new values."""
    h = lib.emtk_nn_create(workspace_bytes=64 << 20)
    m, k, n = 200, 96, 72
    t = torch.float16
    x, w, dy = (torch.zeros(s, dtype=t, device="cuda") for s in ((m, k), (n, k), (m, n)))
    y, z, dx, dw = (torch.empty(s, dtype=t, device="cuda") for s in ((m, n), (m, n), (m, k), (n, k)))

    def step():
        lib.emtk_dense(h, x, w, y, act="silu", pre=z)
        lib.emtk_dense_backward(h, dy, x, w, act="silu", pre=z, dx=dx, dw=dw)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = gen(4)
    for v in (x, w, dy):
        v.copy_(torch.randn(*v.shape, generator=g, device="cuda"))
    graph.replay()
    got = [v.clone() for v in (y, dx, dw)]
    step()
    assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw)))
    torch.cuda.synchronize()
    lib.emtk_nn_destroy(h)


@pytest.mark.parametrize("m,n", [(300, 200), (20, 200)])
def test_a_wait_that_runs_out_is_reported(lib, m, n):
    """A handle whose kernels wait for a barrier nothing arrives at: the wait ends at its limit, the
    check says so once, and the device goes on working."""
    h = lib.emtk_nn_create(wait_timeout_ns=50_000_000, debug_stall=True)
    t = torch.bfloat16
    x, w, y = (torch.ones(s, dtype=t, device="cuda") for s in ((m, 256), (n, 256), (m, n)))
    lib.emtk_dense(h, x, w, y)
    assert lib.emtk_nn_check(h) == lib.EMTK_ERR_TIMEOUT
    assert lib.emtk_nn_check(h) == lib.EMTK_OK
    lib.emtk_nn_destroy(h)
    h = lib.emtk_nn_create()
    lib.emtk_dense(h, x, w, y)
    assert lib.emtk_nn_check(h) == lib.EMTK_OK and bool((y == 256).all())
    lib.emtk_nn_destroy(h)


# ------------------------------------------------------------------ refusals
def test_binding_refuses(lib, nn):
    t = torch.bfloat16
    e = lambda *s, d=t: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
    x, w, y = e(4, 8), e(6, 8), e(4, 6)
    bad = [dict(x=x.float()), dict(w=w.half()), dict(y=e(4, 7)), dict(w=e(6, 9)), dict(x=x.t().contiguous().t()),
           dict(bias=e(5)), dict(bias=e(6, d=torch.float64)), dict(act="tanh"), dict(residual=e(3, 6)),
           dict(y=e(4, 6, d=torch.float32)), dict(y=torch.zeros(4, 6, dtype=t)), dict(x=e(8).expand(4, 8)),
           dict(pre=lib.Q8(e(4, 6, d=torch.int8), e(4, 2, d=torch.uint8))), dict(bias=e(6, d=torch.float16))]
    for change in bad:
        args = dict(dict(x=x, w=w, y=y), **change)
        with pytest.raises((ValueError, lib.EmtkError)):
            lib.emtk_dense(nn, **args)
    with pytest.raises(lib.EmtkError) as err:  # an activation's gradient needs its input
        lib.emtk_dense_backward(nn, y, x, w, act="relu", dx=e(4, 8))
    assert err.value.status == lib.EMTK_ERR_ARG
    with pytest.raises(lib.EmtkError):
        lib.emtk_gated(nn, x, w, w, y, bias_gate=e(6))
    with pytest.raises(lib.EmtkError):
        lib.emtk_gated(nn, x, w, w, y, gate=e(4, 6))
    with pytest.raises(lib.EmtkError):
        lib.emtk_gated_backward(nn, y, y, y, x, w, w, dw_gate=e(6, 8))
    with pytest.raises((ValueError, lib.EmtkError)):
        lib.emtk_pack8(nn, x.float(), lib.emtk_q8_empty(4, 8))
    assert lib.emtk_nn_check(nn) == lib.EMTK_OK


def test_exhausted_memory_is_reported_and_survived(lib):
    """A workspace that cannot grow: EMTK_ERR_OOM, nothing leaked, and the next call works."""
    before = lib.emtk_debug_alloc_counts()
    h = lib.emtk_nn_create()
    t = torch.bfloat16
    dy, x, w, z = (torch.ones(s, dtype=t, device="cuda") for s in ((64, 32), (64, 16), (32, 16), (64, 32)))
    dw = torch.zeros((32, 16), dtype=t, device="cuda")
    lib.emtk_debug_fail_alloc(0)
    with pytest.raises(lib.EmtkError) as err:
        lib.emtk_dense_backward(h, dy, x, w, act="relu", pre=z, dw=dw)
    assert err.value.status == lib.EMTK_ERR_OOM
    lib.emtk_dense_backward(h, dy, x, w, act="relu", pre=z, dw=dw)
    assert bool((dw == 64).all())
    lib.emtk_nn_destroy(h)
    assert lib.emtk_debug_alloc_counts() == before
    lib.emtk_debug_fail_alloc(0)
    with pytest.raises(lib.EmtkError) as err:
        lib.emtk_nn_create()
    assert err.value.status == lib.EMTK_ERR_OOM
    assert lib.emtk_debug_alloc_counts() == before


def test_numpy_definition_of_the_scale_byte(lib, nn):
    """The stored scale is the least power, for every bf16 magnitude as a block's largest."""
    bits = np.arange(1, 0x7F80, dtype=np.uint16)
    x = torch.zeros((bits.size, 32), dtype=torch.bfloat16, device="cuda")
    x[:, 5] = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    q = q8_of(lib, bits.size, 32)
    lib.emtk_pack8(nn, x, q)
    v = x[:, 5].double().cpu().numpy()
    s = q.scales[:, 0].cpu().numpy().astype(np.int64)
    assert (np.rint(v / 2.0 ** (s - 127)) <= 127).all()
    lower = s - 1
    assert ((np.rint(v / 2.0 ** (lower - 127)) > 127) | (s == 1)).all()


# ------------------------------------------------- row distances of what is written
# (m, k, n): tiles of 256 rows, last rows and columns partial; a contraction that is split.
@pytest.mark.parametrize("m,k,n", [(300, 96, 152), (257, 200, 340), (700, 64, 95), (256, 9292, 72), (260, 5000, 131)])
@pytest.mark.parametrize("pad", [0, 2, 4, 7])
def test_row_distances(lib, nn, m, k, n, pad):
    """y, a residual, z and g, u kept in 16 and in 8 bits with rows on 16, 8, 4, 2 bytes and (codes) on any
    byte: the values, and that nothing between the rows is touched.  A call's sums are in the same order
    whatever the distance, so its results are compared with the same call's on aligned rows bit by bit; those
    are tested against 64 bits above."""
    dt = torch.bfloat16
    g = gen(m + n + pad)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    x, w, w2, b, c = r(m, k), r(n, k) / 8, r(n, k) / 8, r(n), r(m, n)
    wide = -(-n // 16) * 16 + 16 - n  # aligned rows

    def run(pad, kept):
        y, h = (Buf(m, n, dt, pad) for _ in "yh")
        res = Buf(m, n, dt, pad, 0, c)
        new = (lambda: q8_of(lib, m, n, pad)) if kept == 8 else (lambda: Buf(m, n, dt, pad))
        z, gate, up = new(), new(), new()
        t = (lambda q: q) if kept == 8 else (lambda q: q.t)
        lib.emtk_dense(nn, x, w, y.t, bias=b, act="gelu", residual=res.t, pre=t(z))
        alone = Buf(m, n, dt, pad), Buf(m, n, dt, pad)
        lib.emtk_dense(nn, x, w, alone[0].t, bias=b, act="gelu", residual=res.t)
        lib.emtk_gated(nn, x, w, w2, h.t, act="silu", gate=t(gate), up=t(up))
        lib.emtk_gated(nn, x, w, w2, alone[1].t, act="silu")
        assert all(v.surroundings_untouched() for v in (y, h, *alone))
        for q in (z, gate, up):
            if kept == 8:
                assert bool((q.codes._base[:, n:] == 77).all()) and bool((q.scales._base[:, (n + 31) // 32:] == 99).all())
            else:
                assert q.surroundings_untouched()
        return [v.t for v in (y, h, *alone)] + [v for q in (z, gate, up) for v in ((q.codes, q.scales) if kept == 8 else (q.t,))]

    for kept in (16, 8):
        for got, want in zip(run(pad, kept), run(wide, kept)):
            assert torch.equal(got, want)


@pytest.mark.parametrize("m,k", [(1, 40), (33, 24), (50, 70), (40, 100), (21, 200), (600, 85), (1500, 264), (300, 1000),
                                 (70, 2305), (5000, 33)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (1, 1), (6, 2), (3, 5)])
def test_pack8_and_back_at_any_distance(lib, nn, m, k, pad, shift):
    """Rows of values and of codes at every alignment, narrow rows that share a warp included."""
    g = gen(m * k + pad)
    x = torch.randn(m, k, generator=g, device="cuda") * torch.exp(2 * torch.randn(m, k, generator=g, device="cuda"))
    x = Buf(m, k, torch.bfloat16, pad, shift, x)
    nb = (k + 31) // 32
    whole = torch.full((m * (k + pad) + shift + 16,), 77, dtype=torch.int8, device="cuda")
    codes = whole[shift:shift + m * (k + pad)].view(m, k + pad)
    q = lib.Q8(codes[:, :k], torch.full((m, nb), 99, dtype=torch.uint8, device="cuda"))
    lib.emtk_pack8(nn, x.t, q)
    want = held8(x.t.double())
    assert torch.equal(q8_values(q, k), want)
    assert bool((codes[:, k:] == 77).all()) and bool((whole[:shift] == 77).all()) and bool((whole[-16:] == 77).all())
    for p, s in ((pad, shift), (0, 0), (1, 3)):
        back = Buf(m, k, torch.bfloat16, p, s)
        lib.emtk_unpack8(nn, q, back.t)
        assert torch.equal(back.t.double(), want) and back.surroundings_untouched()


@pytest.mark.parametrize("eight", ["gate", "up"])
@pytest.mark.parametrize("m,k,f", [(256, 9292, 128), (256, 9292, 72), (64, 16384, 64), (40, 100, 72), (8, 512, 40), (300, 96, 152)])
def test_gate_and_up_kept_in_unlike_kinds(lib, nn, m, k, f, eight):
    """One of g and u kept in 16 bits, the other in 8, where the contraction is split over many parts (the
    first three) and where it is not: each within the bounds of its own kind."""
    dt = torch.bfloat16
    g = gen(m + f)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    x, wg, wu = r(m, k), r(f, k) / 16, r(f, k) / 16
    h, kept16, kept8 = torch.empty((m, f), dtype=dt, device="cuda"), torch.empty((m, f), dtype=dt, device="cuda"), q8_of(lib, m, f)
    gate, up = (kept8, kept16) if eight == "gate" else (kept16, kept8)
    lib.emtk_gated(nn, x, wg, wu, h, act="silu", gate=gate, up=up)
    for w, kept in ((wg, gate), (wu, up)):
        z, e = x.double() @ w.double().t(), (k + 2) * E * (x.double().abs() @ w.double().abs().t())
        if kept is kept16:
            close(kept, z, stored(e, z, "bf16"), "kept in 16 bits")
        else:
            top = torch.nn.functional.pad(z.abs() + e, (0, -f % 32)).view(m, -1, 32).amax(2).repeat_interleave(32, 1)[:, :f]
            close(q8_values(kept, f), z, e + top / 127.5 + 2.0 ** -126, "kept in 8 bits")


def test_a_graph_outlives_a_larger_call(lib):
    """A call captured into a graph, then a larger one that the workspace has to grow for: the workspace that
    the graph holds is kept (seen in the library's count of allocations before the graph runs again), the
    graph gives its results, and all of it goes with the handle."""
    before = lib.emtk_debug_alloc_counts()
    h = lib.emtk_nn_create()
    t = torch.bfloat16
    g = gen(8)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(t)  # noqa: E731
    dy, x, w, z = r(200, 72), r(200, 96), r(72, 96), r(200, 72)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    step = lambda: lib.emtk_dense_backward(h, dy, x, w, act="gelu", pre=z, dx=dx, dw=dw)  # noqa: E731
    large = [r(*s) for s in ((3000, 520), (3000, 264), (520, 264), (3000, 520))]
    out = [torch.empty_like(large[1]), torch.empty_like(large[2])]
    grow = lambda: lib.emtk_dense_backward(h, *large[:3], act="gelu", pre=large[3], dx=out[0], dw=out[1])  # noqa: E731
    step()
    want = dx.clone(), dw.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        with pytest.raises(lib.EmtkError):  # too large for the workspace, and it cannot grow now
            grow()
    held = lib.emtk_debug_alloc_counts()[0]
    grow()
    assert lib.emtk_debug_alloc_counts()[0] == held + 1
    grown = [v.clone() for v in out]
    for _ in range(3):
        dx.zero_(), dw.zero_()
        graph.replay()
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
        grow()
        assert all(torch.equal(a, b) for a, b in zip(out, grown))
    assert lib.emtk_nn_check(h) == lib.EMTK_OK
    torch.cuda.synchronize()
    del graph
    lib.emtk_nn_destroy(h)
    assert lib.emtk_debug_alloc_counts() == before


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gelu_in_its_tail(lib, nn, dtype):
    """z Phi(z) and its slope for z in [-12, 0], relative to the value (the slope: to the sum of its two terms):
    the exponent z^2 / 2, up to 72 and on to 104 in powers of two, is rounded twice (2^-23 of it: 1.2e-5 of the
    value), the rest of the arithmetic is some ten fp32 roundings: together below 2^-16, and the one to 16 bits.
    z itself is exact: one product, with 1, few rows and many columns, and the reverse."""
    dt = DT[dtype]
    z = torch.linspace(-12, 0, 4803, dtype=torch.float64, device="cuda").to(dt).unique()
    n = z.numel()
    z64 = z.double()
    phi, e = torch.special.erfc(-z64 * math.sqrt(0.5)) / 2, torch.exp(-z64 * z64 / 2) / math.sqrt(2 * math.pi)
    bound = lambda v, mag: 2.0 ** -16 * mag + U[dtype] * v.abs() + max(TINY[dtype], 2.0 ** -133)  # noqa: E731
    want = z64 * phi
    one = torch.ones((1, 1), dtype=dt, device="cuda")
    for rows in (1, 3, 40, 200):
        y, ones = torch.empty((rows, n), dtype=dt, device="cuda"), torch.ones((rows, 1), dtype=dt, device="cuda")
        lib.emtk_dense(nn, ones, z.view(n, 1), y, act="gelu")
        close(y, want.expand(rows, n), bound(want, want.abs()), f"{rows} rows")
        lib.emtk_gated(nn, ones, z.view(n, 1), torch.ones((n, 1), dtype=dt, device="cuda"), y, act="gelu")
        close(y, want.expand(rows, n), bound(want, want.abs()), f"{rows} rows, gated")
    y = torch.empty((n, 1), dtype=dt, device="cuda")
    lib.emtk_dense(nn, z.view(n, 1), one, y, act="gelu")
    close(y[:, 0], want, bound(want, want.abs()), "a column")
    want = phi + z64 * e
    lib.emtk_dense_backward(nn, torch.ones((n, 1), dtype=dt, device="cuda"), None, one, act="gelu", pre=z.view(n, 1), dx=y)
    close(y[:, 0], want, bound(want, phi + z64.abs() * e), "slope")


# --------------------------------------------- slopes beyond fp16's range
def stored_slopes(v, err, peak):
    """Error of dz, dg or du as the products take them in fp16: 2^-11 of the value and 2^-19 of the call's largest."""
    return err + U["fp16"] * (v.abs() + err) + 2.0 ** -19 * peak


@pytest.mark.parametrize("shape", [(33, 40, 72), (300, 264, 520), (257, 129, 65), (3000, 40, 24), (600, 85, 701)])
@pytest.mark.parametrize("size", [2.0 ** -23, 2.0 ** -12, 1.0, 2.0 ** 8, 2.0 ** 13])
def test_fp16_gated_slopes_of_any_size(lib, nn, shape, size):
    """dg = dh u act'(g) and du = dh act(g) where fp16 would lose them, below its least or beyond its largest
    number, and the gradients are ordinary ones: dh and u of `size` / 2 .. `size`, x and the weights so that
    dx and the fp32 dw fit.  The call before and the call after are not affected."""
    m, k, f = shape
    g = gen(m + k)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = torch.float16
    signs = lambda *s: torch.sign(r(*s)) * (0.5 + 0.5 * torch.rand(*s, generator=g, device="cuda"))  # noqa: E731
    small = min(1.0, 2.0 ** -6 / size)  # of x and the weights
    dh, up, gate = (signs(m, f) * size).to(dt), (signs(m, f) * size).to(dt), r(m, f).to(dt)
    x, wg, wu = (r(*s).mul_(small).to(dt) for s in ((m, k), (f, k), (f, k)))
    new = lambda: [torch.empty((m, k), dtype=dt, device="cuda")] + \
        [torch.empty(s, device="cuda") for s in ((f, k), (f, k), (f,), (f,))]  # noqa: E731
    call = lambda d, u, o: lib.emtk_gated_backward(nn, d, gate, u, x, wg, wu, act="silu", dx=o[0], dw_gate=o[1], dw_up=o[2],
                                                   db_gate=o[3], db_up=o[4])  # noqa: E731
    plain = r(m, f).to(dt), r(m, f).to(dt)
    before, out, after = new(), new(), new()
    call(*plain, before)
    call(dh, up, out)
    call(*plain, after)
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    d, u64, g64 = dh.double(), up.double(), gate.double()
    a, s = act64("silu", g64), slope64("silu", g64)
    ea, es = act_err(g64, a, 0 * g64), act_err(g64, s, 0 * g64)
    dg, du = d * u64 * s, d * a
    eg, eu = (d * u64).abs() * es + 2 * E * dg.abs(), d.abs() * ea + E * du.abs()
    peak = torch.maximum(dg.abs().max(), du.abs().max())
    rg, ru = stored_slopes(dg, eg, peak), stored_slopes(du, eu, peak)
    wg64, wu64, x64 = wg.double(), wu.double(), x.double()
    want = dg @ wg64 + du @ wu64
    mag = (dg.abs() + rg) @ wg64.abs() + (du.abs() + ru) @ wu64.abs()
    close(out[0], want, stored(rg @ wg64.abs() + ru @ wu64.abs() + (2 * f + 1) * E * mag, want, "fp16"), "dx")
    for name, got, v, e, rounded, db in (("gate", out[1], dg, eg, rg, out[3]), ("up", out[2], du, eu, ru, out[4])):
        want = v.t() @ x64
        err = rounded.t() @ x64.abs() + (m + 1) * E * ((v.abs() + rounded).t() @ x64.abs())
        close(got, want, err + E * want.abs(), "dw_" + name)
        close(db, v.sum(0), e.sum(0) + m * E * (v.abs() + e).sum(0), "db_" + name)


@pytest.mark.parametrize("shape", [(33, 40, 72), (300, 264, 520), (257, 129, 65), (3000, 40, 24), (5000, 33, 8)])
@pytest.mark.parametrize("size", [2.0 ** -22, 2.0 ** -14, 2.0 ** -6, 60000.0])
@pytest.mark.parametrize("act", ["gelu", "sigmoid"])
def test_fp16_dense_slopes_of_any_size(lib, nn, shape, size, act):
    """dz = dy act'(z) likewise: gelu's slope, 1.13 at its largest, takes 60000 beyond fp16."""
    m, k, n = shape
    g = gen(m + k)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = torch.float16
    dy = (torch.sign(r(m, n)) * (0.9 + 0.1 * torch.rand(m, n, generator=g, device="cuda")) * size).to(dt)
    z = (1.4 + 0.2 * r(m, n)).to(dt)
    small = min(1.0, 2.0 ** -6 / size)
    x, w = r(m, k).mul_(small).to(dt), r(n, k).mul_(small).to(dt)
    dx, dw = torch.empty((m, k), dtype=dt, device="cuda"), torch.empty((n, k), device="cuda")
    lib.emtk_dense_backward(nn, dy, x, w, act=act, pre=z, dx=dx, dw=dw)
    s, d = slope64(act, z.double()), dy.double()
    dz, e = d * s, d.abs() * act_err(z.double(), s, 0 * s)
    rounded = stored_slopes(dz, e, dz.abs().max())
    x64, w64 = x.double(), w.double()
    want = dz @ w64
    err = rounded @ w64.abs() + (n + 1) * E * ((dz.abs() + rounded) @ w64.abs())
    close(dx, want, stored(err, want, "fp16"), "dx")
    want = dz.t() @ x64
    close(dw, want, rounded.t() @ x64.abs() + (m + 1) * E * ((dz.abs() + rounded).t() @ x64.abs()) + E * want.abs(), "dw")


def test_fp16_slopes_from_checkpoints_in_a_graph(lib):
    """Sizes that only the device knows: a captured call on ordinary values is replayed with u in 8 bits near
    10^10, with dh near the least number, with an infinity in one row, and on the ordinary values again."""
    h = lib.emtk_nn_create(workspace_bytes=64 << 20)
    m, k, f = 200, 96, 72
    dt = torch.float16
    g = gen(6)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dh, gate, x, w = r(m, f).to(dt), r(m, f), r(m, k).to(dt), (r(f, k) / 8).to(dt)
    gq, uq = lib.emtk_q8_empty(m, f), lib.emtk_q8_empty(m, f)
    u = r(m, f)
    lib.emtk_pack8(h, gate.to(dt), gq)
    lib.emtk_pack8(h, u.to(dt), uq)
    dx, dwg, dwu = torch.empty((m, k), dtype=dt, device="cuda"), torch.empty((f, k), device="cuda"), torch.empty((f, k), device="cuda")
    step = lambda: lib.emtk_gated_backward(h, dh, gq, uq, x, w, w, act="silu", dx=dx, dw_gate=dwg, dw_up=dwu)  # noqa: E731
    step()
    ordinary = [v.clone() for v in (dx, dwg, dwu)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()

    def check():
        g64, u64, d = q8_values(gq, f), q8_values(uq, f), dh.double()
        a, s = act64("silu", g64), slope64("silu", g64)
        dg, du = d * u64 * s, d * a
        eg, eu = (d * u64).abs() * act_err(g64, s, 0 * s) + 2 * E * dg.abs(), d.abs() * act_err(g64, a, 0 * a) + E * du.abs()
        peak = torch.maximum(dg.abs().max(), du.abs().max())
        x64 = x.double()
        for got, v, e in ((dwg, dg, eg), (dwu, du, eu)):
            rounded = stored_slopes(v, e, peak)
            want = v.t() @ x64
            close(got, want, rounded.t() @ x64.abs() + (m + 2) * E * ((v.abs() + rounded).t() @ x64.abs()), "dw")

    kept = dh.clone()
    lib.emtk_pack8(h, (u * 1e10).to(torch.bfloat16), uq)
    graph.replay()
    check()
    lib.emtk_pack8(h, u.to(dt), uq)
    dh.copy_(kept * 2.0 ** -17)
    graph.replay()
    check()
    dh.copy_(kept)
    dh[17, 3] = float("inf")
    graph.replay()
    rest = torch.arange(m, device="cuda") != 17
    assert not bool(torch.isfinite(dx[17]).all()) and torch.equal(dx[rest], ordinary[0][rest])
    dh.copy_(kept)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip((dx, dwg, dwu), ordinary))
    assert lib.emtk_nn_check(h) == lib.EMTK_OK
    torch.cuda.synchronize()
    del graph
    lib.emtk_nn_destroy(h)
