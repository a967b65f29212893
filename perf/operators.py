"""The library's dense, gated and 8-bit checkpoint operators: cases, plain forms and 64-bit definitions.

Shapes: ``m`` rows (hits or tokens), ``k`` inputs, ``n`` outputs (``f`` for the gated block).  Weights are
[out][in].  Every matrix is row-major; ``pad`` widens its rows in memory by that many elements.

    dense        y = act(x w^T + b) + r
    dense_bwd    dz = dy act'(z);  dx = dz w,  dw = dz^T x,  db = sum over rows of dz
    gated        h = act(g) u  with  g = x wg^T + bg,  u = x wu^T + bu
    gated_bwd    dg = dh u act'(g),  du = dh act(g);  dx = dg wg + du wu,  dwg = dg^T x,  dwu = du^T x,  dbg, dbu
    gated_step   gated, keeping g and u as checkpoints, and gated_bwd from them
    ckpt         x and z kept as 8-bit checkpoints, read back, and dense_bwd from them

An 8-bit checkpoint holds blocks of 32 columns of a row as whole numbers of -127 .. 127 times a power of two,
the least for which the block's largest magnitude rounds to at most 127.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "silu", "sigmoid")
BLOCK = 32


# ------------------------------------------------------------------ cases
def _case(op, m, k, n, dtype, act, bias, residual=False, pad=0, saved="", **more):
    return dict(op=op, m=m, k=k, n=n, dtype=dtype, act=act, bias=bias, residual=residual, pad=pad, saved=saved, **more)


def listed():
    return [
        # one hit or token through a square layer of a served network: latency, bound by the weights' bytes
        _case("dense", 1, 4096, 4096, "bf16", "none", True, True, name="dense single row"),
        # the CNN's dense-1 (92,928 -> 128) on the 256 hits of one plane: few outputs, a very long sum
        _case("dense", 256, 92928, 128, "bf16", "relu", True, name="dense long sum"),
        # a patch and one more feature into an odd width, batch of 1693 hits, rows that no 16-byte load fits
        _case("dense", 1693, 2305, 515, "fp16", "gelu", True, True, 3, name="dense ragged"),
        # a training or prompt batch through a wide layer with its residual
        _case("dense", 16384, 4096, 4096, "bf16", "none", True, True, name="dense large"),
        # gradients of the first layer of a student on the 20,000 patches of one APA
        _case("dense_bwd", 20000, 2304, 512, "bf16", "gelu", True, name="dense gradients patches"),
        # gradients of a small odd layer on a batch of 235 hits
        _case("dense_bwd", 235, 1000, 333, "fp16", "relu", True, name="dense gradients small"),
        # one token through a gated block's projections
        _case("gated", 1, 4096, 10240, "bf16", "silu", False, name="gated single row"),
        # a ragged batch through a block whose width is no multiple of a tile
        _case("gated", 777, 1000, 2730, "fp16", "gelu", True, name="gated ragged"),
        # gradients of a block of odd width, g and u kept in 16 bits
        _case("gated_bwd", 2048, 2048, 5461, "bf16", "silu", True, name="gated gradients odd"),
        # a training step of a large block that keeps g and u in 8 bits
        _case("gated_step", 8192, 4096, 10240, "bf16", "silu", False, saved="q8", name="gated step large"),
        # 20,000 patches kept in 8 bits for the gradients of a 2304 -> 128 layer
        _case("ckpt", 20000, 2304, 128, "bf16", "relu", True, name="checkpoint patches"),
        # a small odd layer on checkpoints whose last block is not full
        _case("ckpt", 333, 517, 130, "fp16", "silu", True, name="checkpoint small"),
    ]


def _size(rng, low, high):
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < 0.5:  # widths are round numbers as often as not
        v = v // 8 * 8
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(("dense", "dense", "dense_bwd", "gated", "gated", "gated_bwd", "gated_step", "ckpt"))
    m = _size(rng, 1, 16384)
    k = _size(rng, 64, 8192)
    n = _size(rng, 32, 10240)
    # products of m k n that a pass takes; no more than the largest listed case
    products = {"dense": 1, "dense_bwd": 2, "gated": 2, "gated_bwd": 4, "gated_step": 6, "ckpt": 2}[op]
    most = 6 * 8192 * 4096 * 10240
    m = max(1, min(m, most // (products * k * n)))
    return _case(op, m, k, n, rng.choice(("bf16", "fp16")), rng.choice(ACTS if "gated" not in op else ACTS[1:]),
                 rng.random() < 0.5 and op != "gated_step", op == "dense" and rng.random() < 0.5,
                 rng.choice((0, 0, 0, 1, 3, 8)), rng.choice(("q8", "16")) if op == "gated_step" else "")


# ------------------------------------------------------------------ inputs
def _matrix(g, rows, cols, case, scale, zero_rows=False):
    """[rows][cols] normal values in the case's type, rows case["pad"] elements apart from each other; a few
    rows of activations are zero, as padding rows of a batch are."""
    full = torch.empty((rows, cols + case["pad"]), dtype=DTYPES[case["dtype"]], device="cuda")
    v = full[:, :cols]
    for r in range(0, rows, 4096):  # in pieces: the fp32 draws of a large matrix stay small
        part = v[r:r + 4096]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(scale))
    if zero_rows and rows > 64:
        v[torch.randint(0, rows, (rows // 64,), generator=g, device="cuda")] = 0
    return v


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, m, k, n = case["op"], case["m"], case["k"], case["n"]
    dtype = DTYPES[case["dtype"]]
    s = dict(case=case)

    def rows(cols, scale=1.0, zero=False):
        return _matrix(g, m, cols, case, scale, zero)

    def weight():
        return _matrix(g, n, k, case, 1.0 / math.sqrt(k))

    def like(rows_, cols):  # an output with the case's row distance
        return torch.empty((rows_, cols + case["pad"]), dtype=dtype, device="cuda")[:, :cols]

    def bias():
        return torch.randn(n, generator=g, device="cuda").mul_(0.1).to(dtype) if case["bias"] else None

    s["x"] = rows(k, 1.0, True)
    gated = op.startswith("gated")
    for name in (("wg", "wu") if gated else ("w",)):
        s[name] = weight()
    if op in ("dense", "gated", "gated_step"):
        s["y"] = like(m, n)
    if op == "dense":
        s["b"] = bias()
        s["r"] = rows(n) if case["residual"] else None
    elif op == "gated":
        s["bg"], s["bu"] = bias(), bias()
    if op in ("dense_bwd", "ckpt"):
        s["dy"] = rows(n, 0.1, True)
        s["z"] = rows(n) if case["act"] != "none" else None
        s["db"] = torch.empty(n, dtype=torch.float32, device="cuda") if case["bias"] else None
        s["dx"], s["dw"] = like(m, k), like(n, k)
    if op in ("gated_bwd", "gated_step"):
        s["dh"] = rows(n, 0.1, True)
        s["dx"], s["dwg"], s["dwu"] = like(m, k), like(n, k), like(n, k)
        for name in ("dbg", "dbu"):
            s[name] = torch.empty(n, dtype=torch.float32, device="cuda") if case["bias"] else None
    if op == "gated_bwd":
        s["g"], s["u"] = rows(n), rows(n)
    if op == "gated_step" and case["saved"] == "16":
        s["g"], s["u"] = like(m, n), like(m, n)
    if op == "ckpt":
        s["values"] = like(m, k)
    blocks = lambda cols: -(-cols // BLOCK)  # noqa: E731
    eight = lambda cols: (torch.empty((m, cols), dtype=torch.int8, device="cuda"),  # noqa: E731
                          torch.empty((m, blocks(cols)), dtype=torch.uint8, device="cuda"))
    if op == "ckpt":
        s["x8"] = eight(k)
        s["z8"] = eight(n) if case["act"] != "none" else None
    if op == "gated_step" and case["saved"] == "q8":
        s["g8"], s["u8"] = eight(n), eight(n)
    return s


# ------------------------------------------------------------------ plain forms, 32 bits
def _act(act, z):
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    return z


def _slope(act, z):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if act == "sigmoid":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 - p)
    return torch.ones_like(z)


def _eight(v):
    """The values that an 8-bit checkpoint of v (fp32) stands for."""
    m, n = v.shape
    blocks = -(-n // BLOCK)
    w = torch.zeros((m, blocks * BLOCK), dtype=v.dtype, device=v.device)
    w[:, :n] = v
    w = w.view(m, blocks, BLOCK)
    mant, e = torch.frexp(w.abs().amax(2, keepdim=True))  # amax = mant 2^e, mant in [0.5, 1)
    e = torch.clamp_min(torch.where(mant >= 127.5 / 128, e + 1, e) - 7, -126)
    step = ((e + 127) << 23).view(torch.float32)  # 2^e from its bits: powers computed on the GPU need not be exact
    return (torch.round(w / step) * step).view(m, -1)[:, :n]  # to even at a tie, as everywhere


def _dense_grads(s, x, z):
    c = s["case"]
    dz = s["dy"].float()
    if z is not None:
        dz = dz * _slope(c["act"], z)
    t = DTYPES[c["dtype"]]
    return {"dx": (dz @ s["w"].float()).to(t), "dw": (dz.t() @ x).to(t), **({"db": dz.sum(0)} if c["bias"] else {})}


def _gated_grads(s, x, g, u):
    c = s["case"]
    t = DTYPES[c["dtype"]]
    dh = s["dh"].float()
    dg, du = dh * u * _slope(c["act"], g), dh * _act(c["act"], g)
    out = {"dx": (dg @ s["wg"].float() + du @ s["wu"].float()).to(t), "dwg": (dg.t() @ x).to(t), "dwu": (du.t() @ x).to(t)}
    if c["bias"]:
        out.update(dbg=dg.sum(0), dbu=du.sum(0))
    return out


def _plain(s):
    c = s["case"]
    t, op, act = DTYPES[c["dtype"]], c["op"], c["act"]
    x = s["x"].float()
    if op == "dense":
        z = x @ s["w"].float().t()
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _act(act, z)
        return {"y": (y + s["r"].float() if s["r"] is not None else y).to(t)}
    if op == "dense_bwd":
        return _dense_grads(s, x, s["z"].float() if s["z"] is not None else None)
    if op == "ckpt":
        x = _eight(x)
        z = _eight(s["z"].float()) if s["z"] is not None else None
        return {"values": x.to(t), **_dense_grads(s, x, z)}
    if op == "gated_bwd":
        return _gated_grads(s, x, s["g"].float(), s["u"].float())
    g, u = x @ s["wg"].float().t(), x @ s["wu"].float().t()
    if op == "gated" and s["bg"] is not None:
        g, u = g + s["bg"].float(), u + s["bu"].float()
    h = (_act(act, g) * u).to(t)
    if op == "gated":
        return {"h": h}
    # what is kept for the gradients is held in 8 or 16 bits
    g, u = (_eight(g), _eight(u)) if c["saved"] == "q8" else (g.to(t).float(), u.to(t).float())
    return {"h": h, **_gated_grads(s, x, g, u)}


# ------------------------------------------------------------------ the library's operators
_nn = None


def _library():
    global _nn
    from paper_2009_04509_gb300 import emtk
    if _nn is None:
        _nn = emtk.emtk_nn_create()
    return emtk, _nn


def _own(s):
    emtk, nn = _library()
    c = s["case"]
    op, act = c["op"], c["act"]
    if op == "dense":
        emtk.emtk_dense(nn, s["x"], s["w"], s["y"], bias=s["b"], act=act, residual=s["r"])
        return {"y": s["y"]}
    if op == "gated":
        emtk.emtk_gated(nn, s["x"], s["wg"], s["wu"], s["y"], bias_gate=s["bg"], bias_up=s["bu"], act=act)
        return {"h": s["y"]}
    if op in ("dense_bwd", "ckpt"):
        x, z, out = s["x"], s["z"], {}
        if op == "ckpt":
            x = emtk.Q8(*s["x8"])
            emtk.emtk_pack8(nn, s["x"], x)
            emtk.emtk_unpack8(nn, x, s["values"])
            out["values"] = s["values"]
            if z is not None:
                z = emtk.Q8(*s["z8"])
                emtk.emtk_pack8(nn, s["z"], z)
        emtk.emtk_dense_backward(nn, s["dy"], x, s["w"], act=act, pre=z, dx=s["dx"], dw=s["dw"], db=s["db"])
        return {**out, "dx": s["dx"], "dw": s["dw"], **({"db": s["db"]} if c["bias"] else {})}
    out = {}
    if op == "gated_step":
        g, u = (emtk.Q8(*s["g8"]), emtk.Q8(*s["u8"])) if c["saved"] == "q8" else (s["g"], s["u"])
        emtk.emtk_gated(nn, s["x"], s["wg"], s["wu"], s["y"], act=act, gate=g, up=u)
        out["h"] = s["y"]
    else:
        g, u = s["g"], s["u"]
    emtk.emtk_gated_backward(nn, s["dh"], g, u, s["x"], s["wg"], s["wu"], act=act, dx=s["dx"], dw_gate=s["dwg"],
                             dw_up=s["dwu"], db_gate=s["dbg"], db_up=s["dbu"])
    return {**out, **{name: s[name] for name in ("dx", "dwg", "dwu") + (("dbg", "dbu") if c["bias"] else ())}}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, m, k, n = case["op"], case["m"], case["k"], case["n"]
    xs, ws, ys = m * k, n * k, m * n
    z = ys if case["act"] != "none" else 0
    b = n if case["bias"] else 0
    q = 33 / 32  # bytes of a value in 8 bits
    if op == "dense":
        return {"bytes": 2 * (xs + ws + ys + b + (ys if case["residual"] else 0)), "flops": 2 * m * k * n}
    if op == "gated":
        return {"bytes": 2 * (xs + 2 * ws + ys + 2 * b), "flops": 4 * m * k * n}
    if op == "dense_bwd":
        return {"bytes": 2 * (2 * xs + 2 * ws + ys + z) + 4 * b, "flops": 4 * m * k * n}
    if op == "ckpt":  # and each checkpoint written
        return {"bytes": 2 * (3 * xs + 2 * ws + ys + z) + q * (xs + z) + 4 * b, "flops": 4 * m * k * n}
    if op == "gated_bwd":
        return {"bytes": 2 * (2 * xs + 4 * ws + 3 * ys) + 8 * b, "flops": 8 * m * k * n}
    return {"bytes": 2 * (2 * xs + 4 * ws + 2 * ys) + 2 * (q if case["saved"] == "q8" else 2) * ys, "flops": 12 * m * k * n}


# ------------------------------------------------------------------ the definition in 64 bits
def _phi(z):  # the normal distribution function
    return torch.special.ndtr(z)


_F64 = {
    "none": (lambda z: z, lambda z: torch.ones_like(z)),
    "relu": (torch.relu, lambda z: torch.where(z > 0, 1.0, 0.0).double()),
    "gelu": (lambda z: z * _phi(z), lambda z: _phi(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)),
    "silu": (lambda z: z * torch.sigmoid(z), lambda z: torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)),
    "sigmoid": (torch.sigmoid, lambda z: torch.sigmoid(z) * torch.sigmoid(-z)),
}


def _held8(v):
    n = v.shape[1]
    w = torch.nn.functional.pad(v, (0, -n % BLOCK)).unflatten(1, (-1, BLOCK))
    top = w.abs().amax(2, keepdim=True)
    power = lambda e: ((e + 1023) << 52).view(torch.float64)  # noqa: E731  2^e exactly
    e = torch.floor(torch.log2(torch.clamp_min(top, 2.0 ** -200))).long() - 6
    e = torch.where(torch.round(top / power(e)) > 127, e + 1, e)
    e = torch.where(torch.round(top / power(e - 1)) <= 127, e - 1, e)  # log2 may be one off at a power of two
    step = power(torch.clamp_min(e, -126))
    return (torch.round(w / step) * step).flatten(1)[:, :n]


def exact(case, seed):
    s = prepare(case, seed)
    d = {name: v.double() for name, v in s.items() if isinstance(v, torch.Tensor)}
    f, df = _F64[case["act"]]
    op = case["op"]
    if op == "dense":
        y = f(torch.einsum("mk,nk->mn", d["x"], d["w"]) + d.get("b", 0.0)) + d.get("r", 0.0)
        return {"y": y}
    if op in ("dense_bwd", "ckpt"):
        x, z, out = d["x"], d.get("z"), {}
        if op == "ckpt":
            x = out["values"] = _held8(x)
            z = None if z is None else _held8(z)
        dz = d["dy"] if z is None else d["dy"] * df(z)
        out.update(dx=torch.einsum("mn,nk->mk", dz, d["w"]), dw=torch.einsum("mn,mk->nk", dz, x))
        if case["bias"]:
            out["db"] = torch.einsum("mn->n", dz)
        return out
    out = {}
    if op == "gated_bwd":
        g, u = d["g"], d["u"]
    else:
        g = torch.einsum("mk,nk->mn", d["x"], d["wg"]) + d.get("bg", 0.0)
        u = torch.einsum("mk,nk->mn", d["x"], d["wu"]) + d.get("bu", 0.0)
        out["h"] = f(g) * u
        if op == "gated":
            return out
        held = _held8 if case["saved"] == "q8" else (lambda v: v.to(DTYPES[case["dtype"]]).double())
        g, u = held(g), held(u)
    dg, du = d["dh"] * u * df(g), d["dh"] * f(g)
    out.update(dx=torch.einsum("mn,nk->mk", dg, d["wg"]) + torch.einsum("mn,nk->mk", du, d["wu"]),
               dwg=torch.einsum("mn,mk->nk", dg, d["x"]), dwu=torch.einsum("mn,mk->nk", du, d["x"]))
    if case["bias"]:
        out.update(dbg=torch.einsum("mn->n", dg), dbu=torch.einsum("mn->n", du))
    return out
