"""The library's operators around a network's products: cases, plain forms and 64-bit definitions.

``m`` rows (tokens, hits, steps of sequences), ``n`` columns.  Every matrix is row-major; ``pad`` widens its rows
in memory by that many elements.

    norm        y = s r + g D Npost(b),  h = Npre(y)      norms around a block's output b, gate g, dropout D
    norm_bwd    gradients of r, b, g and both norms' parameters from dy and dh
    dropout     y = x or 0, by Philox4x32-10 numbers of (column / 8, row, offset) under the seed
    logprob     log probability of a token of every row, the row's entropy and its largest log probabilities
    logprob_step    the same, and the gradient of the logits
    recur       h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(f),  y_t = act(o_t) h_t, along each sequence
    recur_step  the same, and the gradients of f, x, o and the first states
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------ cases
def _norm(op, m, n, dtype, pre, post, gate, every=0, p=0.0, scale=1.0, pad=0, params="same", **more):
    return dict(op=op, m=m, n=n, dtype=dtype, pre=pre, post=post, gate=gate, every=every or m, p=p, scale=scale, pad=pad,
                params=params, **more)


def _logprob(op, m, n, dtype, top=0, temperature=1.0, masked=False, pad=0, **more):
    return dict(op=op, m=m, n=n, dtype=dtype, top=top, temperature=temperature, masked=masked, pad=pad, **more)


def _recur(op, m, n, dtype, seqs, ragged, act, state, pad=0, **more):
    return dict(op=op, m=m, n=n, dtype=dtype, seqs=seqs, ragged=ragged, act=act, state=state, pad=pad, **more)


def listed():
    return [
        # one token between two blocks of a served network: latency
        _norm("norm", 1, 4096, "bf16", "rms", "rms", "vector", name="norm single row"),
        # a batch of 1693 hits of odd width in training, one gate row for every 7 hits, rows that no 16-byte load fits
        _norm("norm", 1693, 515, "fp16", "layer", "layer", "rows", 7, 0.1, 0.5, 3, name="norm ragged"),
        # a prompt or a training batch between two blocks
        _norm("norm", 16384, 4096, "bf16", "rms", "rms", "vector", name="norm large"),
        # gradients of a training step with dropout at an odd width, parameters in fp32
        _norm("norm_bwd", 8192, 5461, "bf16", "layer", "rms", "vector", p=0.1, params="f32", name="norm gradients odd"),
        # a small odd batch
        dict(op="dropout", m=235, n=333, dtype="fp16", p=0.1, pad=0, name="dropout small"),
        # the inner width of a large block
        dict(op="dropout", m=16384, n=10240, dtype="bf16", p=0.2, pad=0, name="dropout large"),
        # what a served network answers for one token: the sampled token's log probability and 8 alternatives
        _logprob("logprob", 1, 131072, "bf16", 8, 0.8, name="logprob single row"),
        # the student's three classes on the 20,000 hits of one APA, beside a fourth column: loss and gradient
        _logprob("logprob_step", 20000, 3, "bf16", pad=1, name="logprob classes"),
        # loss, entropy and gradient of a training batch over a large vocabulary
        _logprob("logprob_step", 8192, 65536, "bf16", masked=True, name="logprob step large"),
        # one token for each of 64 sequences, their states in hand
        _recur("recur", 64, 4096, "bf16", 64, False, "silu", True, name="recurrence tokens"),
        # 800 wires of 1000 time intervals each, 64 features: a training step
        _recur("recur_step", 800000, 64, "bf16", 800, False, "silu", False, name="recurrence wires"),
        # four long sequences of unlike lengths in one batch: a training step
        _recur("recur_step", 20011, 2048, "fp16", 4, True, "sigmoid", True, name="recurrence long"),
    ]


def _size(rng, low, high):
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < 0.5:  # widths are round numbers as often as not
        v = v // 8 * 8
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(("norm", "norm", "norm_bwd", "norm_bwd", "dropout", "logprob", "logprob_step", "recur", "recur_step"))
    pad, dtype = rng.choice((0, 0, 0, 1, 3, 8)), rng.choice(("bf16", "fp16"))
    most = 1 << 26  # values of a matrix
    if op.startswith("norm"):
        n = _size(rng, 32, 16384)
        m = min(_size(rng, 1, 32768), max(1, most // n))
        gate = rng.choice(("none", "vector", "rows"))
        post = rng.choice(("none", "rms", "layer"))
        return _norm(op, m, n, dtype, rng.choice(("rms", "layer")), post, gate,
                     max(1, m // rng.choice((1, 3, 16))) if gate == "rows" else 0, rng.choice((0.0, 0.0, 0.1, 0.5)),
                     rng.choice((1.0, 0.5)), pad, rng.choice(("same", "f32")))
    if op == "dropout":
        n = _size(rng, 32, 16384)
        return dict(op=op, m=min(_size(rng, 1, 32768), max(1, most // n)), n=n, dtype=dtype, p=rng.choice((0.1, 0.25, 0.5)), pad=pad)
    if op.startswith("logprob"):
        n = _size(rng, 3, 200000)
        m = min(_size(rng, 1, 32768), max(1, most // n))
        top = min(n, rng.choice((0, 1, 5, 8, 20))) if op == "logprob" else 0
        return _logprob(op, m, n, rng.choice(("bf16", "fp16", "f32")), top, rng.choice((1.0, 0.7, 1.3)), rng.random() < 0.5, pad)
    n = _size(rng, 16, 4096)
    length = _size(rng, 1, 32768)
    seqs = max(1, min(_size(rng, 1, 512), most // (n * length)))
    length = max(1, min(length, most // n))
    return _recur(op, length * seqs, n, dtype, seqs, rng.random() < 0.5, rng.choice(("none", "silu", "sigmoid", "gelu")),
                  rng.random() < 0.5, pad)


# ------------------------------------------------------------------ inputs
def _empty(rows, cols, dtype, pad):
    return torch.empty((rows, cols + pad), dtype=dtype, device="cuda")[:, :cols]


def _matrix(g, rows, cols, dtype, pad, scale=1.0, shift=0.0):
    """[rows][cols] normal values, rows ``pad`` elements apart from each other."""
    v = _empty(rows, cols, dtype, pad)
    step = max(1, (1 << 24) // max(1, cols))
    for r in range(0, rows, step):  # in pieces: the fp32 draws of a large matrix stay small
        part = v[r:r + step]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(scale).add_(shift))
    return v


def _offsets(case, g):
    """Where each sequence starts, and the end of the last: cuts at random places."""
    m, seqs = case["m"], case["seqs"]
    cuts = torch.randint(0, m + 1, (seqs - 1,), generator=g, device="cuda").sort().values
    edge = torch.tensor([0, m], device="cuda")
    return torch.cat([edge[:1], cuts, edge[1:]]).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, m, n, pad, dtype = case["op"], case["m"], case["n"], case["pad"], DTYPES[case["dtype"]]
    s = dict(case=case)

    def rows(scale=1.0, shift=0.0):
        return _matrix(g, m, n, dtype, pad, scale, shift)

    def like():
        return _empty(m, n, dtype, pad)

    def vector(scale=1.0, shift=0.0, count=m):
        return torch.randn(count, generator=g, device="cuda").mul_(scale).add_(shift)

    if op in ("norm", "norm_bwd", "dropout"):
        s["seed"], s["offset"] = seed * 7919 + 12345678901, seed + (1 << 33)
    if op == "dropout":
        s["x"], s["y"] = rows(), like()
    elif op.startswith("norm"):
        params = torch.float32 if case["params"] == "f32" else dtype
        for which in ("pre", "post"):
            kind = case[which]
            s[which + "_w"] = vector(0.2, 1.0, n).to(params) if kind != "none" else None
            s[which + "_b"] = vector(0.2, 0.0, n).to(params) if kind == "layer" else None
        groups = -(-m // case["every"])
        s["gate"] = _matrix(g, groups, n, dtype, 0, 0.3, 0.5) if case["gate"] != "none" else None
        s["block"] = rows(2.0, 0.1)
        if op == "norm":
            s["residual"], s["y"], s["h"] = rows(), like(), like()
        else:
            s["y"], s["dy"], s["dh"] = rows(), rows(0.1), rows(0.1)
            s["dr"], s["db"] = like(), like()
            s["d_gate"] = torch.empty((groups, n), dtype=torch.float32, device="cuda") if case["gate"] != "none" else None
            for which in ("pre", "post"):
                for name in ("w", "b"):
                    s[f"d{name}_{which}"] = torch.empty(n, dtype=torch.float32, device="cuda") if s[f"{which}_{name}"] is not None else None
    elif op.startswith("logprob"):
        s["z"] = rows(3.0)
        columns = torch.randperm(n, generator=g, device="cuda")
        if case["masked"]:  # a third of the columns may not be answered
            s["z"][:, columns[:n // 3]] = -math.inf
            columns = columns[n // 3:]
        tokens = columns[torch.randint(0, len(columns), (m,), generator=g, device="cuda")]
        if m > 16:
            tokens[torch.randint(0, m, (m // 16,), generator=g, device="cuda")] = -1  # padding: no token
        s["tokens"] = tokens.to(torch.int32)
        for name in ("logprob", "entropy", "lse"):
            s[name] = torch.empty(m, dtype=torch.float32, device="cuda")
        if case["top"]:
            s["top_logprob"] = torch.empty((m, case["top"]), dtype=torch.float32, device="cuda")
            s["top_index"] = torch.empty((m, case["top"]), dtype=torch.int32, device="cuda")
        if op == "logprob_step":
            s["dlogprob"], s["dentropy"], s["dz"] = vector(1.0, -1.0), vector(0.1), like()
    else:
        seqs, gated = case["seqs"], case["act"] != "none"
        s["f"], s["x"], s["y"] = rows(1.5, 2.0), rows(), like()
        s["o"] = rows() if gated else None
        s["offsets"] = _offsets(case, g) if case["ragged"] else None
        s["state"] = _matrix(g, seqs, n, torch.float32, 0) if case["state"] else None
        s["last"] = torch.empty((seqs, n), dtype=torch.float32, device="cuda")
        if op == "recur_step":
            s["dy"] = rows(0.1)
            s["dlast"] = _matrix(g, seqs, n, torch.float32, 0, 0.1) if case["state"] else None
            s["df"], s["dx"], s["do"] = like(), like(), like() if gated else None
            s["dstate"] = torch.empty((seqs, n), dtype=torch.float32, device="cuda")
            s["states"] = torch.empty((m // 128 + seqs, n), dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms, 32 bits
def _act(act, z):
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    return z


def _slope(act, z):
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    p = 1 / (1 + torch.exp(-z))
    return p * (1 + z * (1 - p)) if act == "silu" else p * (1 - p)


def _kept(s):
    """Dropout's factors [m][n]: 0, or 1 over the share that stays."""
    c = s["case"]
    drop = round(c["p"] * 65536)
    if not drop:
        return None
    low = 0xffffffff
    c0 = torch.arange(-(-c["n"] // 8), device="cuda")[None, :].expand(c["m"], -1)
    c1 = torch.arange(c["m"], device="cuda")[:, None].expand_as(c0)
    c2, c3 = torch.full_like(c0, s["offset"] & low), torch.full_like(c0, s["offset"] >> 32)
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # the products' 64 bits; the shifts below drop the sign
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 2)
    halves = torch.stack([words & 0xffff, words >> 16], 3).flatten(1)[:, :c["n"]]
    return (halves >= drop).float() * (65536 / (65536 - drop))


def _normed(x, kind):
    """The normalised rows and 1 / their spread."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    r = 1 / torch.sqrt(x.square().mean(1, keepdim=True) + EPS)
    return x * r, r


def _norm_forward(s):
    c = s["case"]
    t = DTYPES[c["dtype"]]

    def norm(x, which):
        if c[which] == "none":
            return x
        v = _normed(x, c[which])[0] * s[which + "_w"].float()
        return v + s[which + "_b"].float() if c[which] == "layer" else v

    v = norm(s["block"].float(), "post")
    kept = _kept(s)
    v = v if kept is None else v * kept
    if s["gate"] is not None:
        v = v * s["gate"].float().repeat_interleave(c["every"], 0)[:c["m"]]
    y = s["residual"].float() * c["scale"] + v
    return {"y": y.to(t), "h": norm(y, "pre").to(t)}


def _norm_gradients(s):
    c = s["case"]
    t = DTYPES[c["dtype"]]

    def back(d, x, which):
        """The gradient of a norm's input, of its weight and of its bias."""
        if c[which] == "none":
            return d, {}
        xhat, r = _normed(x, c[which])
        out = {f"dw_{which}": (d * xhat).sum(0), **({f"db_{which}": d.sum(0)} if c[which] == "layer" else {})}
        d = d * s[which + "_w"].float()
        mean = d.mean(1, keepdim=True) if c[which] == "layer" else 0
        return r * (d - mean - xhat * (d * xhat).mean(1, keepdim=True)), out

    dx, out = back(s["dh"].float(), s["y"].float(), "pre")
    stream = dx + s["dy"].float()
    out["dr"] = (stream * c["scale"]).to(t)
    b = s["block"].float()
    kept = _kept(s)
    dv = stream if kept is None else stream * kept
    if s["gate"] is not None:
        v = b if c["post"] == "none" else _normed(b, c["post"])[0] * s["post_w"].float()
        v = v + s["post_b"].float() if c["post"] == "layer" else v
        groups = s["gate"].shape[0]
        each = torch.nn.functional.pad(dv * v, (0, 0, 0, groups * c["every"] - c["m"]))
        out["d_gate"] = each.view(groups, c["every"], -1).sum(1)
        dv = dv * s["gate"].float().repeat_interleave(c["every"], 0)[:c["m"]]
    db, more = back(dv, b, "post")
    return {**out, **more, "db": db.to(t)}


def _logprobs(s):
    c = s["case"]
    z = s["z"].float() + 0.0  # no -0 beside 0
    d = (z - z.amax(1, keepdim=True)) * (1 / c["temperature"])
    e = torch.exp(d)
    total = e.sum(1)
    entropy = torch.log(total) - torch.where(e > 0, e * d, 0).sum(1) / total
    logp = d - torch.log(total)[:, None]
    given = s["tokens"].long()
    out = {"logprob": torch.where(given >= 0, logp.gather(1, given.clamp_min(0)[:, None])[:, 0], 0.0), "entropy": entropy}
    if c["top"]:
        bits = z.view(torch.int32).long()
        order = torch.where(bits < 0, bits ^ 0x7fffffff, bits)  # ordered as the values are
        key = (order << 32) - torch.arange(c["n"], device="cuda")  # the lowest index first among equals
        index = (-torch.topk(key, c["top"], dim=1).values) & 0xffffffff
        out.update(top_logprob=logp.gather(1, index), top_index=index.int())
    if c["op"] == "logprob_step":
        p = e / total[:, None]
        dlogp = torch.where(given >= 0, s["dlogprob"], 0.0)[:, None]
        dz = torch.where(p > 0, -p * (dlogp + s["dentropy"][:, None] * (logp + entropy[:, None])), 0)
        dz.scatter_add_(1, given.clamp_min(0)[:, None], dlogp)
        out["dz"] = (dz * (1 / c["temperature"])).to(DTYPES[c["dtype"]])
    return out


def _starts(s):
    """Each row's sequence, its first row and its last."""
    c = s["case"]
    m, seqs = c["m"], c["seqs"]
    at = s["offsets"].long() if s["offsets"] is not None else torch.arange(seqs + 1, device="cuda") * (m // seqs)
    seq = torch.searchsorted(at, torch.arange(m, device="cuda"), right=True) - 1
    return at, seq, at[seq], at[seq + 1] - 1


def _scan(b, v, first, longest):
    """Runs of steps joined pairwise, doubling: (1 - product of (1 - b), state from 0 of h = (1 - b) h + v)."""
    step, at = 1, torch.arange(b.shape[0], device="cuda")
    while step < longest:
        joined = (at - step >= first)[step:, None]
        pb, pv = b[:-step], v[:-step]
        v = torch.cat([v[:step], torch.where(joined, v[step:] + (pv - b[step:] * pv), v[step:])])
        b = torch.cat([b[:step], torch.where(joined, b[step:] + (pb - b[step:] * pb), b[step:])])
        step *= 2
    return b, v


def _recurrence(s):
    c = s["case"]
    t, act = DTYPES[c["dtype"]], c["act"]
    at, seq, first, final = _starts(s)
    f, x = s["f"].float(), s["x"].float()
    b = 1 / (1 + torch.exp(f))
    zero = torch.zeros_like(s["last"])
    h0 = s["state"] if s["state"] is not None else zero
    longest = c["m"] if c["ragged"] else c["m"] // c["seqs"]
    through, h = _scan(b, b * x, first, longest)
    h = h + (h0[seq] - through * h0[seq])
    some = (at[1:] > at[:-1])[:, None]
    out = {"last": torch.where(some, h[(at[1:] - 1).clamp_min(0)], h0)}
    o = s["o"].float() if s["o"] is not None else None
    out["y"] = (h if o is None else h * _act(act, o)).to(t)
    if c["op"] == "recur":
        return out
    dy = s["dy"].float()
    row = torch.arange(c["m"], device="cuda")
    before = torch.where((row > first)[:, None], torch.cat([h0[:1], h[:-1]]), h0[seq])
    u = dy if o is None else dy * _act(act, o)
    dlast = s["dlast"] if s["dlast"] is not None else zero
    u = torch.where((row == final)[:, None], u + dlast[seq], u)
    # backwards in time: g_t = u_t + (1 - b_{t+1}) g_{t+1}
    after = torch.where((row < final)[:, None], torch.cat([b[1:], b[:1]]), 1.0).flip(0)
    _, g = _scan(after, u.flip(0), (c["m"] - 1 - final).flip(0), longest)
    g = g.flip(0)
    a = 1 / (1 + torch.exp(-f))
    out.update(dx=(b * g).to(t), df=(g * (before - x) * a * b).to(t))
    if o is not None:
        out["do"] = (dy * h * _slope(act, o)).to(t)
    top = at[:-1].clamp_max(c["m"] - 1)
    out["dstate"] = torch.where(some, g[top] - b[top] * g[top], dlast)
    return out


def _plain(s):
    op = s["case"]["op"]
    if op == "dropout":
        return {"y": (s["x"].float() * _kept(s)).to(s["x"].dtype)}
    if op.startswith("norm"):
        return _norm_forward(s) if op == "norm" else _norm_gradients(s)
    return _logprobs(s) if op.startswith("logprob") else _recurrence(s)


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
    op = c["op"]
    if op in ("norm", "norm_bwd", "dropout"):
        drop = emtk.Drop(c["p"], s["seed"], s["offset"]) if c["p"] else None
    if op == "dropout":
        emtk.emtk_dropout(nn, s["x"], s["y"], drop)
        return {"y": s["y"]}
    if op.startswith("norm"):
        pre, post = (emtk.Norm(c[w], s[w + "_w"], s[w + "_b"], EPS) if c[w] != "none" else None for w in ("pre", "post"))
        if op == "norm":
            emtk.emtk_residual_norm(nn, s["residual"], s["block"], s["y"], s["h"], post=post, pre=pre, gate=s["gate"],
                                    gate_every=c["every"], scale=c["scale"], drop=drop)
            return {"y": s["y"], "h": s["h"]}
        grads = {name: s[name] for name in ("dw_pre", "db_pre", "dw_post", "db_post", "d_gate")}
        emtk.emtk_residual_norm_backward(nn, s["dy"], s["dh"], s["y"], s["block"], s["dr"], s["db"], post=post, pre=pre,
                                         gate=s["gate"], gate_every=c["every"], scale=c["scale"], drop=drop, **grads)
        return {"dr": s["dr"], "db": s["db"], **{k: v for k, v in grads.items() if v is not None}}
    if op.startswith("logprob"):
        top = {name: s[name] for name in ("top_logprob", "top_index")} if c["top"] else {}
        step = op == "logprob_step"
        emtk.emtk_logprobs(nn, s["z"], s["tokens"], s["logprob"], s["entropy"], s["lse"] if step else None, **top,
                           temperature=c["temperature"])
        out = {"logprob": s["logprob"], "entropy": s["entropy"], **top}
        if step:
            emtk.emtk_logprobs_backward(nn, s["z"], s["lse"], s["dz"], tokens=s["tokens"], d_logprob=s["dlogprob"],
                                        entropy=s["entropy"], d_entropy=s["dentropy"], temperature=c["temperature"])
            out["dz"] = s["dz"]
        return out
    step = op == "recur_step"
    emtk.emtk_recurrence(nn, s["f"], s["x"], s["y"], o=s["o"], act=c["act"], seqs=c["seqs"], offsets=s["offsets"],
                         state=s["state"], last=s["last"], states=s["states"] if step else None)
    out = {"y": s["y"], "last": s["last"]}
    if step:
        emtk.emtk_recurrence_backward(nn, s["dy"], s["f"], s["x"], s["states"], s["df"], s["dx"], o=s["o"], act=c["act"],
                                      seqs=c["seqs"], offsets=s["offsets"], d_last=s["dlast"], d_o=s["do"], d_state=s["dstate"])
        out.update(df=s["df"], dx=s["dx"], dstate=s["dstate"], **({"do": s["do"]} if s["do"] is not None else {}))
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, m, n = case["op"], case["m"], case["n"]
    e = 4 if case["dtype"] == "f32" else 2
    one = e * m * n
    if op == "dropout":
        return {"bytes": 2 * one, "flops": 8 * m * n}
    if op.startswith("norm"):
        params = n * (4 if case["params"] == "f32" else 2) * sum({"none": 0, "rms": 1, "layer": 2}[case[w]] for w in ("pre", "post"))
        gate = 2 * n * -(-m // case["every"]) if case["gate"] != "none" else 0
        if op == "norm":
            return {"bytes": 4 * one + params + gate, "flops": 16 * m * n}
        return {"bytes": 6 * one + 3 * params + 3 * gate, "flops": 32 * m * n}
    if op.startswith("logprob"):
        return {"bytes": (2 if op == "logprob_step" else 1) * one + m * (20 + 8 * case["top"]), "flops": 8 * m * n}
    gated = case["act"] != "none"
    states = 4 * n * case["seqs"] * (2 if case["state"] else 1)
    if op == "recur":
        return {"bytes": (4 if gated else 3) * one + states, "flops": 16 * m * n}
    return {"bytes": (8 if gated else 6) * one + 2 * states, "flops": 48 * m * n}


# ------------------------------------------------------------------ the definition in 64 bits
def _philox(case, s):
    """Which elements dropout keeps, by 16-bit limbs: no product here has more than 48 bits."""
    m, n = case["m"], case["n"]
    word = 2 ** 32

    def product(x, k):  # (upper, lower) word of x k
        lo, hi = x * (k % 65536), x * (k // 65536)
        t = (lo // 65536) + hi
        return t // 65536, (t % 65536) * 65536 + lo % 65536

    col, row = torch.meshgrid(torch.arange((n + 7) // 8, device="cuda"), torch.arange(m, device="cuda"), indexing="xy")
    x = [col, row, torch.full_like(col, s["offset"] % word), torch.full_like(col, s["offset"] // word)]
    key = [s["seed"] % word, s["seed"] // word]
    for r in range(10):
        h0, l0 = product(x[0], 0xD2511F53)
        h1, l1 = product(x[2], 0xCD9E8D57)
        x = [h1.bitwise_xor(x[1]).bitwise_xor((key[0] + r * 0x9E3779B9) % word), l1,
             h0.bitwise_xor(x[3]).bitwise_xor((key[1] + r * 0xBB67AE85) % word), l0]
    numbers = torch.empty((m, (n + 7) // 8, 8), dtype=torch.int64, device="cuda")
    for i in range(8):
        numbers[:, :, i] = x[i // 2] // (65536 if i % 2 else 1) % 65536
    return numbers.view(m, -1)[:, :n] / 65536


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    op, m, n = case["op"], case["m"], case["n"]
    if op in ("dropout", "norm", "norm_bwd"):
        p = round(case["p"] * 65536) / 65536
        factor = (_philox(case, s) >= p).double() / (1 - p) if p else torch.ones((), device="cuda", dtype=torch.float64)
    if op == "dropout":
        return {"y": d["x"] * factor}
    if op.startswith("norm"):
        gate = d["gate"][torch.arange(m, device="cuda") // case["every"]] if s["gate"] is not None else 1.0

        def norm(x, which, w, b):
            if case[which] == "none":
                return x
            if case[which] == "layer":
                return (x - x.mean(1, True)) / torch.sqrt(x.var(1, correction=0, keepdim=True) + EPS) * w + b
            return x / torch.sqrt((x * x).sum(1, keepdim=True) / n + EPS) * w

        w = {k: d.get(k) for k in ("pre_w", "pre_b", "post_w", "post_b")}
        if op == "norm":
            y = case["scale"] * d["residual"] + gate * factor * norm(d["block"], "post", w["post_w"], w["post_b"])
            return {"y": y, "h": norm(y, "pre", w["pre_w"], w["pre_b"])}
        # by differentiation: h of the y that is given, and y of its parts
        w = {k: v.requires_grad_() if v is not None else None for k, v in w.items()}
        y, b, r = d["y"].requires_grad_(), d["block"].requires_grad_(), torch.zeros(m, n, device="cuda", dtype=torch.float64, requires_grad=True)
        g = d["gate"].requires_grad_() if s["gate"] is not None else None
        norm(y, "pre", w["pre_w"], w["pre_b"]).backward(d["dh"])
        rows = g[torch.arange(m, device="cuda") // case["every"]] if g is not None else 1.0
        (case["scale"] * r + rows * factor * norm(b, "post", w["post_w"], w["post_b"])).backward(y.grad + d["dy"])
        out = {"dr": r.grad, "db": b.grad, **{f"d{k[-1]}_{k[:-2]}": v.grad for k, v in w.items() if v is not None}}
        return {**out, "d_gate": g.grad} if g is not None else out
    if op.startswith("logprob"):
        z = d["z"] / case["temperature"]
        given = s["tokens"].long()
        has = given >= 0
        logp = torch.log_softmax(z, 1)
        p = torch.exp(logp)
        entropy = -torch.special.xlogy(p, p).sum(1)
        out = {"logprob": torch.where(has, logp[torch.arange(m, device="cuda"), given * has], 0.0), "entropy": entropy}
        if case["top"]:
            order = torch.sort(d["z"], dim=1, descending=True, stable=True).indices[:, :case["top"]]
            out.update(top_logprob=torch.take_along_dim(logp, order, 1), top_index=order.int())
        if op == "logprob_step":
            chosen = torch.zeros_like(z)
            chosen[torch.arange(m, device="cuda")[has], given[has]] = 1.0
            dz = (chosen - p) * (d["dlogprob"] * has)[:, None]
            dz -= d["dentropy"][:, None] * (torch.special.xlogy(p, p) + p * entropy[:, None])
            out["dz"] = dz / case["temperature"]
        return out
    # one step of every sequence after another
    seqs = case["seqs"]
    at = s["offsets"].long().tolist() if s["offsets"] is not None else [i * (m // seqs) for i in range(seqs + 1)]
    longest = max(b - a for a, b in zip(at, at[1:]))
    if longest > 40000:
        return None
    lengths = torch.tensor([b - a for a, b in zip(at, at[1:])], device="cuda")
    begin = torch.tensor(at[:-1], device="cuda")
    order = torch.argsort(lengths, descending=True, stable=True)  # so that the sequences still running are the first
    running = (lengths[None, :] > torch.arange(longest, device="cuda")[:, None]).sum(1).tolist()
    a, h = torch.sigmoid(d["f"]), d["state"].clone() if s["state"] is not None else torch.zeros(seqs, n, device="cuda", dtype=torch.float64)
    first = h.clone()
    states = torch.empty(m, n, device="cuda", dtype=torch.float64)
    for t in range(longest):
        who = order[:running[t]]
        row = begin[who] + t
        h[who] = a[row] * h[who] + torch.sigmoid(-d["f"][row]) * d["x"][row]
        states[row] = h[who]
    o = d.get("o")
    act, slope = {
        "silu": (lambda v: v * torch.sigmoid(v), lambda v: torch.sigmoid(v) + v * torch.sigmoid(v) * torch.sigmoid(-v)),
        "sigmoid": (torch.sigmoid, lambda v: torch.sigmoid(v) * torch.sigmoid(-v)),
        "gelu": (lambda v: v * torch.special.ndtr(v), lambda v: torch.special.ndtr(v) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)),
        "none": (None, None)}[case["act"]]
    out = {"y": states if o is None else states * act(o), "last": h}
    if op == "recur":
        return out
    g = d["dlast"].clone() if s["dlast"] is not None else torch.zeros_like(h)
    u = d["dy"] if o is None else d["dy"] * act(o)
    dx, df = torch.empty_like(states), torch.empty_like(states)
    for t in reversed(range(longest)):
        who = order[:running[t]]
        row = begin[who] + t
        total = g[who] + u[row]
        dx[row] = torch.sigmoid(-d["f"][row]) * total
        previous = states[row - 1] if t else first[who]
        df[row] = total * (previous - d["x"][row]) * a[row] * torch.sigmoid(-d["f"][row])
        g[who] = a[row] * total
    out.update(df=df, dx=dx, dstate=g)
    if o is not None:
        out["do"] = d["dy"] * states * slope(o)
    return out
