"""The wires' network: norms, dropout, dense layers, recurrences, gated blocks and log probabilities run together as a
user runs them, against the same network in torch's autograd in 64 bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wires():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_04509_gb300 import build, wires as m
    build.build()
    return m


def reference(net, levels, targets, at, weights, masks):
    """Log probabilities and the gradients of their sum times `weights`, from the bf16 weights in 64 bits."""
    p = {k: v.double().requires_grad_() for k, v in net.w.items()}
    d = net.width

    def rms(x, w):
        return x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-6) * w

    s = p["embedding"][levels.long()]
    for b in range(net.blocks):
        n = rms(s, p[f"n1_{b}"])
        f, x, o = (n @ p[f"in_{b}"].t() + p[f"b_in_{b}"]).split(d, 1)
        states = []
        for i, j in zip(at, at[1:]):
            h = torch.zeros(d, dtype=torch.float64, device="cuda")
            for t in range(i, j):
                a = torch.sigmoid(f[t])
                h = a * h + (1 - a) * x[t]
                states.append(h)
        r = torch.stack(states) * torch.nn.functional.silu(o)
        s = s + p[f"gate1_{b}"] * masks[2 * b] * (r @ p[f"mix_{b}"].t())
        n = rms(s, p[f"n2_{b}"])
        h = torch.nn.functional.silu(n @ p[f"wg_{b}"].t()) * (n @ p[f"wu_{b}"].t())
        s = s + p[f"gate2_{b}"] * masks[2 * b + 1] * (h @ p[f"down_{b}"].t())
    logp = torch.log_softmax(rms(s, p["n_out"]) @ p["head"].t(), 1)
    given = targets >= 0
    out = torch.where(given, logp.gather(1, targets.long().clamp_min(0)[:, None])[:, 0], 0.0)
    (out * weights.double()).sum().backward()
    return out.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("dropout", [0.0, 0.2])
def test_gradients_against_autograd(wires, dropout):
    """One pass over sequences of unlike lengths and its gradients.  Each of the chain's tensors is rounded to bf16 (2^-8 of
    its values, 2^-9 in rms over sqrt 3); some twenty of them in a row, independent, add in squares to below 2^-5 of the norms."""
    from tests.test_gpu_around import factors
    net = wires.WireModel(width=72, hidden=136, blocks=2, dropout=dropout, seed=3)
    try:
        lengths = [40, 0, 1, 150, 9]
        at = torch.tensor([0] + lengths).cumsum(0).tolist()
        m, seqs = at[-1], len(lengths)
        g = torch.Generator(device="cuda")
        g.manual_seed(0)
        levels = torch.randint(0, net.levels, (m,), generator=g, device="cuda").int()
        targets = torch.randint(-2, net.levels, (m,), generator=g, device="cuda").int()
        offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
        keep = {}
        out = net.logprobs(net.logits(levels, seqs, offsets, keep=keep), targets, keep)
        weights = torch.randn(m, generator=g, device="cuda")
        grads = net.gradients(net.dlogits(weights, keep), keep)
        masks = [factors(m, net.width, dropout, 0x5eed, i) for i in range(2 * net.blocks)]
        want_out, want = reference(net, levels, targets, at, weights, masks)
        assert (out.double() - want_out).norm() <= 2.0 ** -5 * want_out.norm()
        assert set(want) == set(grads)
        for k, v in want.items():
            assert (grads[k].double() - v).norm() <= 2.0 ** -5 * v.norm(), k
    finally:
        net.close()


def test_served_step_by_step_gives_the_whole(wires):
    """A sequence read one level at a time, states in hand, has the log probabilities of the whole read at once (rounded to
    bf16 at the same places; the products of few rows add in another order, so that those roundings may fall otherwise: as above)."""
    net = wires.WireModel(width=64, hidden=128, seed=1)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(2)
        seqs, T = 5, 33
        levels = torch.randint(0, net.levels, (seqs, T), generator=g, device="cuda").int()
        whole = net.logits(levels.reshape(-1), seqs).view(seqs, T, -1).double()
        states = net.states(seqs)
        for t in range(T):
            part = net.logits(levels[:, t].contiguous(), seqs, states=states)
            assert (part.double() - whole[:, t]).norm() <= 2.0 ** -5 * whole[:, t].norm(), t
        more = net.likeliest(levels[:, -1].contiguous(), states, 3)
        assert more.shape == (3, seqs) and bool(((more >= 0) & (more < net.levels)).all())
    finally:
        net.close()


def test_a_training_run_holds_together(wires):
    from paper_2009_04509_gb300 import emtk
    levels = wires.wire_levels(24, nticks=1200)
    net = wires.WireModel(width=64, hidden=64, dropout=0.1)
    try:
        v = levels[:16]
        x, y = v.reshape(-1), torch.cat([v[:, 1:], torch.full_like(v[:, :1], -1)], 1).reshape(-1).contiguous()
        values = [float(net.step(x, y, seqs=16)) for _ in range(5)]
        assert all(u == u and u <= 0 for u in values)
        assert all(bool(torch.isfinite(p).all()) for p in net.master.values())
        assert emtk.emtk_nn_check(net.nn) == emtk.EMTK_OK
    finally:
        net.close()
