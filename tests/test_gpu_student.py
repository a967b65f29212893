"""The student network: the library's layers run together as a user runs them, against the same
network in torch's autograd on fp32 weights."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def student():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_04509_gb300 import build, student as m
    build.build()
    return m


def reference(net, x, dlogits):
    """Gradients of sum(logits * dlogits) by autograd, from the bf16 weights as fp64."""
    p = {k: v.double().requires_grad_() for k, v in net.w.items()}
    z = x.double() @ p["w_in"].t() + p["b_in"]
    a = torch.nn.functional.gelu(z)
    h = torch.nn.functional.silu(a @ p["w_gate"].t()) * (a @ p["w_up"].t())
    r = h @ p["w_down"].t() + p["b_down"] + a
    out = r @ p["w_out"].t() + p["b_out"]
    (out * dlogits.double()).sum().backward()
    return out.detach(), {k: v.grad for k, v in p.items()}


def test_step_against_autograd(student):
    """One pass and its gradients.  Each of the chain's tensors is rounded to bf16 (2^-8 of its values) and
    the checkpoints to 8 bits (at most 1/127 of their block's largest value, 2 sqrt 3 times that smaller in
    rms: about 2^-7 of the values' rms); half a dozen of them in a row, independent, add in squares to below
    2^-5 of the norms."""
    net = student.Student(width=96, hidden=200, seed=3)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(0)
        x = (torch.randn(700, 2304, generator=g, device="cuda") * 0.5).to(torch.bfloat16)
        dlogits = torch.randn(700, 4, generator=g, device="cuda").to(torch.bfloat16)
        keep = {}
        out = net.logits(x, keep)
        grads = net.gradients(dlogits, keep)
        want_out, want = reference(net, x, dlogits)
        assert (out.double() - want_out).norm() <= 2.0 ** -5 * want_out.norm()
        for k, v in want.items():
            assert (grads[k].double() - v).norm() <= 2.0 ** -5 * v.norm(), k
        # served: any number of rows gives the batch's rows
        for rows in (1, 3, 40, 300):
            one = net.logits(x[:rows].contiguous())
            assert (one.double() - want_out[:rows]).norm() <= 2.0 ** -5 * want_out[:rows].norm(), rows
    finally:
        net.close()


def test_training_learns_the_scores(student):
    x, scores = student.patches_and_scores(2000, seed=1)
    net = student.Student(seed=2)
    try:
        first = float(net.step(x, scores))
        for _ in range(60):
            last = net.step(x, scores)
        assert float(last) < first - 0.05 and float(last) == float(last)
        from paper_2009_04509_gb300 import emtk
        assert emtk.emtk_nn_check(net.nn) == emtk.EMTK_OK
    finally:
        net.close()
