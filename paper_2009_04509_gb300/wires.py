"""Learns the waveforms of wires, interval by interval, and continues them, with the library's operators.

    python -m paper_2009_04509_gb300.wires --wires 480 --steps 300

A wire of a synthetic plane is a sequence: its charge in each time interval (6 ticks, the
patch cut's) as one of a few levels.  The network reads a wire from its start and gives, at each
interval, the log probabilities of the next one's level:

    s = embedding[level]                                          rows: the intervals of all wires
    a block, twice over the stream s:
      f, x, o = n w_in^T + b_in,   n = rms(s)                     emtk_residual_norm, emtk_dense
      r = silu(o) h,  h_t = a h_(t-1) + (1 - a) x                 emtk_recurrence along each wire
      s = s + gate dropout(r w_mix^T),  n = rms(s)                emtk_dense, emtk_residual_norm
      s = s + gate dropout((silu(n w_gate^T) n w_up^T) w_down^T)  emtk_gated, emtk_dense, emtk_residual_norm
    log probabilities of n w_head^T                               emtk_dense, emtk_logprobs

A training step keeps what the backward pass needs and draws dropout anew from a counter; weights are
held in fp32 (Adam) and copied to bf16.  Served, a step takes one level of each wire with
the recurrences' states in hand.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2009_04509_gb300 import emtk, synth  # noqa: E402

LEVELS = 16
TICKS = 6  # of an interval


class WireModel:
    def __init__(self, width: int = 128, hidden: int = 256, blocks: int = 2, levels: int = LEVELS, dropout: float = 0.0,
                 seed: int = 0, device="cuda:0"):
        import torch
        self.torch, self.device = torch, torch.device(device)
        self.nn = emtk.emtk_nn_create(self.device.index or 0)
        self.width, self.hidden, self.blocks, self.levels, self.dropout = width, hidden, blocks, levels, dropout
        g = torch.Generator(device=self.device)
        g.manual_seed(seed)

        def normal(out, inp):
            return torch.randn(out, inp, generator=g, device=self.device) / math.sqrt(inp)

        ones, p = lambda n: torch.ones(n, device=self.device), {}  # noqa: E731
        p["embedding"] = torch.randn(levels, width, generator=g, device=self.device)
        for b in range(blocks):
            p[f"n1_{b}"], p[f"n2_{b}"] = ones(width), ones(width)
            p[f"in_{b}"] = normal(3 * width, width)
            p[f"b_in_{b}"] = torch.cat([torch.full((width,), 2.0, device=self.device), torch.zeros(2 * width, device=self.device)])
            p[f"mix_{b}"], p[f"gate1_{b}"], p[f"gate2_{b}"] = normal(width, width), ones(width), ones(width)
            p[f"wg_{b}"], p[f"wu_{b}"], p[f"down_{b}"] = normal(hidden, width), normal(hidden, width), normal(width, hidden)
        p["n_out"], p["head"] = ones(width), normal(levels, width)
        self.master = p
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in p.items()}
        self.steps = 0
        self._refresh()

    def close(self) -> None:
        if self.nn is not None:
            emtk.emtk_nn_destroy(self.nn)
            self.nn = None

    def _refresh(self) -> None:
        """What the operators read: matrices and gates in bf16, norms' weights and biases as they are."""
        t = self.torch.bfloat16
        self.w = {k: v.to(t) if v.dim() == 2 or k.startswith("gate") else v for k, v in self.master.items()}

    def _new(self, rows: int, cols: int):
        return self.torch.empty((rows, cols), dtype=self.torch.bfloat16, device=self.device)

    def _norm(self, b: int) -> emtk.Norm:
        """The norm before block b (after the last: before the head)."""
        return emtk.Norm("rms", self.w[f"n1_{b}" if b < self.blocks else "n_out"])

    def _drop(self, b: int, which: int, train: bool):
        return emtk.Drop(self.dropout, 0x5eed, (self.steps * self.blocks + b) * 2 + which) if train and self.dropout else None

    def logits(self, levels, seqs: int = 1, offsets=None, states=None, keep: dict | None = None):
        """levels [rows] (the sequences one after another) -> logits [rows][levels] of the next level.  states: a list of
        each block's [seqs][width] fp32 states, taken on; keep: receives what the backward pass needs."""
        nn, w, d, m = self.nn, self.w, self.width, levels.shape[0]
        train = keep is not None
        s = w["embedding"][levels.long()]
        n = self._new(m, d)
        emtk.emtk_residual_norm(nn, s, None, None, n, pre=self._norm(0))
        kept = [dict(s=s)]
        for b in range(self.blocks):
            k = dict(n1=n, p=self._new(m, 3 * d), r=self._new(m, d), m=self._new(m, d), s1=self._new(m, d), n2=self._new(m, d),
                     h=self._new(m, self.hidden), u=self._new(m, d), s=self._new(m, d))
            emtk.emtk_dense(nn, n, w[f"in_{b}"], k["p"], bias=w[f"b_in_{b}"])
            f, x, o = k["p"].split(d, 1)
            k["states"] = emtk.emtk_recurrence_states(m, d, seqs, self.device) if train else None
            state = states[b] if states is not None else None
            emtk.emtk_recurrence(nn, f, x, k["r"], o=o, act="silu", seqs=seqs, offsets=offsets, state=state, last=state, states=k["states"])
            emtk.emtk_dense(nn, k["r"], w[f"mix_{b}"], k["m"])
            emtk.emtk_residual_norm(nn, s, k["m"], k["s1"], k["n2"], pre=emtk.Norm("rms", w[f"n2_{b}"]), gate=w[f"gate1_{b}"],
                                    drop=self._drop(b, 0, train))
            if train:
                k["g"], k["v"] = self._new(m, self.hidden), self._new(m, self.hidden)
            emtk.emtk_gated(nn, k["n2"], w[f"wg_{b}"], w[f"wu_{b}"], k["h"], gate=k.get("g"), up=k.get("v"))
            emtk.emtk_dense(nn, k["h"], w[f"down_{b}"], k["u"])
            n = self._new(m, d)
            emtk.emtk_residual_norm(nn, k["s1"], k["u"], k["s"], n, pre=self._norm(b + 1), gate=w[f"gate2_{b}"], drop=self._drop(b, 1, train))
            s = k["s"]
            kept.append(k)
        out = self._new(m, self.levels)
        emtk.emtk_dense(nn, n, w["head"], out)
        if train:
            keep.update(levels=levels, blocks=kept, n=n, seqs=seqs, offsets=offsets)
        return out

    def gradients(self, dlogits, keep: dict) -> dict:
        """Gradients (fp32) of every weight from dlogits and what logits() kept."""
        t, w, nn, d = self.torch, self.w, self.nn, self.width
        m, seqs, offsets = dlogits.shape[0], keep["seqs"], keep["offsets"]
        grad = {k: t.empty_like(v) for k, v in self.master.items()}
        dn, ds = self._new(m, d), None
        emtk.emtk_dense_backward(nn, dlogits, keep["n"], w["head"], dx=dn, dw=grad["head"])
        for b in reversed(range(self.blocks)):
            k = keep["blocks"][b + 1]
            ds1, du, dh, dn2 = self._new(m, d), self._new(m, d), self._new(m, self.hidden), self._new(m, d)
            emtk.emtk_residual_norm_backward(nn, ds, dn, k["s"], k["u"], ds1, du, pre=self._norm(b + 1), gate=w[f"gate2_{b}"],
                                             drop=self._drop(b, 1, True), d_gate=grad[f"gate2_{b}"],
                                             dw_pre=grad[f"n1_{b + 1}" if b + 1 < self.blocks else "n_out"])
            emtk.emtk_dense_backward(nn, du, k["h"], w[f"down_{b}"], dx=dh, dw=grad[f"down_{b}"])
            emtk.emtk_gated_backward(nn, dh, k["g"], k["v"], k["n2"], w[f"wg_{b}"], w[f"wu_{b}"], dx=dn2, dw_gate=grad[f"wg_{b}"],
                                     dw_up=grad[f"wu_{b}"])
            ds, dm, dr, dp = self._new(m, d), self._new(m, d), self._new(m, d), self._new(m, 3 * d)
            emtk.emtk_residual_norm_backward(nn, ds1, dn2, k["s1"], k["m"], ds, dm, pre=emtk.Norm("rms", w[f"n2_{b}"]), gate=w[f"gate1_{b}"],
                                             drop=self._drop(b, 0, True), d_gate=grad[f"gate1_{b}"], dw_pre=grad[f"n2_{b}"])
            emtk.emtk_dense_backward(nn, dm, k["r"], w[f"mix_{b}"], dx=dr, dw=grad[f"mix_{b}"])
            (f, x, o), (df, dx, do) = k["p"].split(d, 1), dp.split(d, 1)
            emtk.emtk_recurrence_backward(nn, dr, f, x, k["states"], df, dx, o=o, act="silu", seqs=seqs, offsets=offsets, d_o=do)
            dn = self._new(m, d)
            emtk.emtk_dense_backward(nn, dp, k["n1"], w[f"in_{b}"], dx=dn, dw=grad[f"in_{b}"], db=grad[f"b_in_{b}"])
        ds0 = self._new(m, d)
        emtk.emtk_residual_norm_backward(nn, ds, dn, keep["blocks"][0]["s"], None, ds0, pre=self._norm(0), dw_pre=grad["n1_0"])
        grad["embedding"].zero_().index_add_(0, keep["levels"].long(), ds0.float())
        return grad

    def logprobs(self, logits, targets, keep: dict | None = None):
        """Log probability of each row's target (0 where it is negative); keep: for dlogits()."""
        t, m = self.torch, logits.shape[0]
        out, lse = t.empty(m, device=self.device), t.empty(m, device=self.device)
        emtk.emtk_logprobs(self.nn, logits, targets, out, lse=lse)
        if keep is not None:
            keep.update(logits=logits, lse=lse, targets=targets)
        return out

    def dlogits(self, d_logprob, keep: dict):
        d = self.torch.empty_like(keep["logits"])
        emtk.emtk_logprobs_backward(self.nn, keep["logits"], keep["lse"], d, tokens=keep["targets"], d_logprob=d_logprob)
        return d

    def step(self, levels, targets, seqs: int = 1, offsets=None, lr: float = 2e-3):
        """One Adam step on the mean log probability of the targets that are given; returns it (not read back)."""
        keep, t = {}, self.torch
        logprob = self.logprobs(self.logits(levels, seqs, offsets, keep=keep), targets, keep)
        given = (targets >= 0).sum().clamp_min(1)
        grads = self.gradients(self.dlogits((t.full_like(logprob, -1.0) / given), keep), keep)
        self.steps += 1
        c1, c2 = 1 - 0.9 ** self.steps, 1 - 0.999 ** self.steps
        for k, v in self.master.items():
            m1, m2 = self.moments[k]
            m1.mul_(0.9).add_(grads[k], alpha=0.1)
            m2.mul_(0.999).addcmul_(grads[k], grads[k], value=0.001)
            v.addcdiv_(m1 / c1, (m2 / c2).sqrt_().add_(1e-8), value=-lr)
        self._refresh()
        return logprob.sum() / given

    def states(self, seqs: int) -> list:
        return [self.torch.zeros(seqs, self.width, device=self.device) for _ in range(self.blocks)]

    def likeliest(self, levels, states, count: int):
        """Continues each sequence by `count` levels, each the likeliest; levels [seqs]: the ones before."""
        t, seqs = self.torch, levels.shape[0]
        out, logprob = t.empty((count, seqs), dtype=t.int32, device=self.device), t.empty((seqs, 1), device=self.device)
        for i in range(count):
            emtk.emtk_logprobs(self.nn, self.logits(levels, seqs, states=states), top_logprob=logprob, top_index=out[i].view(seqs, 1))
            levels = out[i]
        return out


def wire_levels(wires: int, seed: int = 0, device="cuda:0", nticks: int = 6000):
    """Levels [wires][nticks / 6] (int32) of a synthetic plane's intervals: equal steps of the square root of the charge."""
    import torch
    plane = synth.single_plane(seed=seed, nwires=wires, nhits=8 * wires, n_tracks=max(5, wires // 4), nticks=nticks)
    adc = torch.from_numpy(plane.adc).to(device)[:, :plane.nticks // TICKS * TICKS]
    charge = adc.reshape(wires, -1, TICKS).mean(2).clamp_min(0).sqrt()
    return (charge * (LEVELS / float(charge.max()))).to(torch.int32).clamp_max(LEVELS - 1)


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--wires", type=int, default=480)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--lr", type=float, default=2e-3)
    args = ap.parse_args()
    import torch

    levels = wire_levels(args.wires)
    held = max(1, args.wires // 10)  # the last tenth is not trained on
    train, length = args.wires - held, levels.shape[1]
    net = WireModel(dropout=args.dropout)
    try:
        g = torch.Generator(device=levels.device)
        g.manual_seed(1)

        def rows(pick):
            """Inputs and targets of some wires: a wire's last interval has none."""
            v = levels[pick]
            return v.reshape(-1), torch.cat([v[:, 1:], torch.full_like(v[:, :1], -1)], 1).reshape(-1).contiguous()

        def quality():
            x, y = rows(torch.arange(train, args.wires, device=levels.device))
            return float(net.logprobs(net.logits(x, held), y).sum() / (y >= 0).sum())

        before = quality()
        batch = min(args.batch, train)
        for i in range(args.steps):
            if i == min(20, args.steps // 2):  # the first steps load kernels and grow the workspace
                torch.cuda.synchronize()
                t0, timed = time.perf_counter(), args.steps - i
            net.step(*rows(torch.randint(0, train, (batch,), generator=g, device=levels.device)), seqs=batch, lr=args.lr)
        torch.cuda.synchronize()
        per_step = (time.perf_counter() - t0) / timed if args.steps else 0.0
        after = quality()
        states = net.states(held)
        net.likeliest(levels[train:, 0].contiguous(), states, 20)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        net.likeliest(levels[train:, 0].contiguous(), states, 200)
        torch.cuda.synchronize()
        single = (time.perf_counter() - t0) / 200
        rc = emtk.emtk_nn_check(net.nn)
    finally:
        net.close()
    print(f"{args.steps} steps of {batch} wires x {length} intervals, {1e6 * per_step:.0f} us each; held-out log probability of an interval "
          f"{before:.4f} -> {after:.4f}; one more interval of {held} wires {1e6 * single:.0f} us")
    return 0 if rc == emtk.EMTK_OK else 1


if __name__ == "__main__":
    sys.exit(main())
