"""Trains and serves a student of the CNN on cut patches, with the library's layers.

    python -m paper_2009_04509_gb300.student --hits 20000 --steps 300

The student is a small residual network on a hit's 48 x 48 patch (2304 values):

    a = gelu(x w_in^T + b_in)                          emtk_dense
    h = silu(a w_gate^T) * (a w_up^T)                  emtk_gated
    r = h w_down^T + b_down + a                        emtk_dense with a residual
    logits = r w_out^T + b_out  (track, em, none, Michel)

It learns the CNN's scores (emtk_infer_patches) on patches that emtk_extract_patches
cuts from a synthetic plane: softmax cross entropy on the first three, binary cross
entropy on the fourth.  Between its two passes a step keeps x, the first layer's z and
the block's g and u as 8-bit checkpoints and recomputes h in the backward pass; weights
are held in fp32 (Adam) and copied to bf16 for the products.  Served, the same calls
take any number of rows, one hit included.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2009_04509_gb300 import emtk, synth  # noqa: E402

PATCH = 48 * 48
INPUT_SCALE = 2.0 ** -5  # raw ADC counts to about 1; exact in bf16


class Student:
    def __init__(self, width: int = 128, hidden: int = 512, seed: int = 0, device="cuda:0"):
        import torch
        self.torch, self.device = torch, torch.device(device)
        self.nn = emtk.emtk_nn_create(self.device.index or 0)
        g = torch.Generator(device=self.device)
        g.manual_seed(seed)

        def normal(out, inp):
            return torch.randn(out, inp, generator=g, device=self.device) / math.sqrt(inp)

        zeros = lambda n: torch.zeros(n, device=self.device)  # noqa: E731
        self.master = dict(w_in=normal(width, PATCH), b_in=zeros(width), w_gate=normal(hidden, width),
                           w_up=normal(hidden, width), w_down=normal(width, hidden), b_down=zeros(width),
                           w_out=normal(4, width), b_out=zeros(4))
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in self.master.items()}
        self.steps = 0
        self._refresh()

    def close(self) -> None:
        if self.nn is not None:
            emtk.emtk_nn_destroy(self.nn)
            self.nn = None

    def _refresh(self) -> None:
        """The products' copies: weights in bf16, biases as they are."""
        self.w = {k: v.to(self.torch.bfloat16) if v.dim() == 2 else v for k, v in self.master.items()}

    def _new(self, rows: int, cols: int):
        return self.torch.empty((rows, cols), dtype=self.torch.bfloat16, device=self.device)

    def logits(self, x, keep: dict | None = None):
        """x [n][2304] bf16 -> [n][4]; with keep, what the backward pass needs goes there."""
        w, m = self.w, x.shape[0]
        width, hidden = w["w_in"].shape[0], w["w_gate"].shape[0]
        a, h, r, out = self._new(m, width), self._new(m, hidden), self._new(m, width), self._new(m, 4)
        z = g = u = None
        if keep is not None:
            z, g, u = (emtk.emtk_q8_empty(m, n, self.device) for n in (width, hidden, hidden))
            x8 = emtk.emtk_q8_empty(m, PATCH, self.device)
            emtk.emtk_pack8(self.nn, x, x8)
            keep.update(x=x8, z=z, a=a, g=g, u=u, r=r)
        emtk.emtk_dense(self.nn, x, w["w_in"], a, bias=w["b_in"], act="gelu", pre=z)
        emtk.emtk_gated(self.nn, a, w["w_gate"], w["w_up"], h, act="silu", gate=g, up=u)
        emtk.emtk_dense(self.nn, h, w["w_down"], r, bias=w["b_down"], residual=a)
        emtk.emtk_dense(self.nn, r, w["w_out"], out, bias=w["b_out"])
        return out

    def gradients(self, dlogits, keep: dict) -> dict:
        """Gradients (fp32) of every weight from dlogits [n][4] and what logits() kept."""
        t, w, nn = self.torch, self.w, self.nn
        m = dlogits.shape[0]
        d = {k: t.empty_like(v) for k, v in self.master.items()}
        dr, da, dh, h = self._new(m, w["w_out"].shape[1]), self._new(m, w["w_gate"].shape[1]), \
            self._new(m, w["w_down"].shape[1]), self._new(m, w["w_down"].shape[1])
        emtk.emtk_dense_backward(nn, dlogits, keep["r"], w["w_out"], dx=dr, dw=d["w_out"], db=d["b_out"])
        emtk.emtk_dense_backward(nn, dr, None, w["w_down"], dx=dh)
        emtk.emtk_gated_backward(nn, dh, keep["g"], keep["u"], keep["a"], w["w_gate"], w["w_up"], act="silu", dx=da,
                                 dw_gate=d["w_gate"], dw_up=d["w_up"], h=h)
        emtk.emtk_dense_backward(nn, dr, h, None, dw=d["w_down"], db=d["b_down"])
        da += dr  # the residual's gradient
        emtk.emtk_dense_backward(nn, da, keep["x"], None, act="gelu", pre=keep["z"], dw=d["w_in"], db=d["b_in"])
        return d

    def loss(self, logits, scores):
        """(loss, dlogits in bf16) of the distillation against the CNN's scores [n][4]."""
        t = self.torch
        z = logits.float()
        p, q = t.softmax(z[:, :3], 1), t.sigmoid(z[:, 3])
        eps = 1e-6
        loss = -(scores[:, :3] * t.log(p + eps)).sum(1) - scores[:, 3] * t.log(q + eps) - \
            (1 - scores[:, 3]) * t.log(1 - q + eps)
        d = t.cat([p * scores[:, :3].sum(1, keepdim=True) - scores[:, :3], (q - scores[:, 3])[:, None]], 1) / z.shape[0]
        return loss.mean(), d.to(t.bfloat16)

    def step(self, x, scores, lr: float = 1e-3):
        """One Adam step; returns the loss (a tensor, not read back)."""
        keep = {}
        loss, d = self.loss(self.logits(x, keep), scores)
        grads = self.gradients(d, keep)
        self.steps += 1
        c1, c2 = 1 - 0.9 ** self.steps, 1 - 0.999 ** self.steps
        for k, v in self.master.items():
            m1, m2 = self.moments[k]
            m1.mul_(0.9).add_(grads[k], alpha=0.1)
            m2.mul_(0.999).addcmul_(grads[k], grads[k], value=0.001)
            v.addcdiv_(m1 / c1, (m2 / c2).sqrt_().add_(1e-8), value=-lr)
        self._refresh()
        return loss


def patches_and_scores(hits: int, seed: int = 0, device="cuda:0"):
    """Patches of a synthetic plane's hits, bf16 [n][2304] scaled, and the CNN's scores [n][4]."""
    import torch
    dev = torch.device(device)
    plane = synth.single_plane(seed=seed, nwires=800, nhits=hits, n_tracks=max(5, hits // 50))
    adc, at = torch.from_numpy(plane.adc).to(dev), torch.from_numpy(plane.hits).to(dev)
    ctx = emtk.emtk_create(synth.he_normal_weights(0), precision="bf16", device=dev.index or 0)
    try:
        patches = torch.empty((plane.nhits, 48, 48), dtype=torch.float32, device=dev)
        scores = torch.empty((plane.nhits, 4), dtype=torch.float32, device=dev)
        emtk.emtk_extract_patches(ctx, adc, plane.nticks, at, patches, "f32")
        emtk.emtk_infer_patches(ctx, patches, scores)
        rc = emtk.emtk_check(ctx)
    finally:
        emtk.emtk_destroy(ctx)
    if rc != emtk.EMTK_OK:
        raise emtk.EmtkError(rc, "emtk_infer_patches")
    return (patches.view(plane.nhits, PATCH) * INPUT_SCALE).to(torch.bfloat16), scores


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--hits", type=int, default=20000)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--lr", type=float, default=1e-3)
    args = ap.parse_args()
    import torch

    x, scores = patches_and_scores(args.hits)
    held = max(1, x.shape[0] // 10)  # the last tenth is not trained on
    train = x.shape[0] - held
    net = Student(args.width, args.hidden)
    try:
        g = torch.Generator(device=x.device)
        g.manual_seed(1)

        def quality():
            z = net.logits(x[train:])
            loss, _ = net.loss(z, scores[train:])
            same = (z[:, :3].float().argmax(1) == scores[train:, :3].argmax(1)).float().mean()
            return float(loss), float(same)

        before = quality()
        for i in range(args.steps):
            if i == min(20, args.steps // 2):  # the first steps load kernels and grow the workspace
                torch.cuda.synchronize()
                t0, timed = time.perf_counter(), args.steps - i
            pick = torch.randint(0, train, (min(args.batch, train),), generator=g, device=x.device)
            net.step(x[pick], scores[pick], args.lr)
        torch.cuda.synchronize()
        per_step = (time.perf_counter() - t0) / timed if args.steps else 0.0
        after = quality()
        one = x[:1].contiguous()
        for _ in range(20):
            net.logits(one)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        for _ in range(200):
            net.logits(one)
        torch.cuda.synchronize()
        single = (time.perf_counter() - t0) / 200
        rc = emtk.emtk_nn_check(net.nn)
    finally:
        net.close()
    print(f"{args.steps} steps of {min(args.batch, train)} hits, {1e6 * per_step:.0f} us each; held-out loss {before[0]:.4f} -> "
          f"{after[0]:.4f}, same class as the CNN {before[1]:.3f} -> {after[1]:.3f}; one hit {1e6 * single:.1f} us")
    return 0 if rc == emtk.EMTK_OK else 1


if __name__ == "__main__":
    sys.exit(main())
