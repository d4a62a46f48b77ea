"""The block operators as a model uses them: the example's residual steps and loss run, and their gradients
are those of the same model in PyTorch operations."""
import pytest
import torch

from test_gpu_window_example import example

pytestmark = pytest.mark.gpu


def test_example_runs_with_dropout():
    first, last, right, far = example().main(steps=3, quiet=True, dropout=0.1)
    assert all(torch.isfinite(torch.tensor(v)) for v in (first, last, right, far))


def test_gradients_are_those_of_plain_operations():
    """Loss of two residual steps around a linear map: the example's functions against float64 autograd.
    h and the head's product are rounded to bf16 (2^-8 relative each) before they meet the loss, the gradients
    twice more: within 4 x 2^-8 of their norms."""
    ex = example()
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    B, T, d, V, bf = 2, 40, 256, 100, torch.bfloat16
    x, y, gate, a, b = r(B, T, d), r(B, T, d).to(bf), r(d).to(bf), (1 + 0.1 * r(d)).to(bf), (1 + 0.1 * r(d)).to(bf)
    E = (r(d, V) * d ** -0.5).to(bf)
    t = torch.randint(-1, V, (B, T), generator=g, device="cuda")
    leaves = [v.clone().requires_grad_() for v in (x, y, gate, a, b, E)]
    x1, h = ex.ResidualStep.apply(*leaves[:5], True, (0.0, None, 0))
    x2, h2 = ex.ResidualStep.apply(x1, h, None, None, leaves[4], False, (0.0, None, 1))
    loss = ex.TokenLoss.apply(h2 @ leaves[5], t)
    got = torch.autograd.grad(loss, leaves)
    want_leaves = [v.double().requires_grad_() for v in (x, y, gate, a, b, E)]
    X, Y, G, A, Bp, Ed = want_leaves
    norm = lambda v, w: v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w   # noqa: E731
    z1 = X + G * norm(Y, A)
    z2 = z1 + norm(z1, Bp)
    lp = torch.log_softmax(norm(z2, Bp) @ Ed, -1).gather(-1, t.clamp(min=0)[..., None])[..., 0]
    want_loss = -torch.where(t >= 0, lp, 0.0).sum() / (t >= 0).sum()
    want = torch.autograd.grad(want_loss, want_leaves)
    loss, want_loss = loss.item(), want_loss.item()
    assert abs(loss - want_loss) < 2 ** -6 * want_loss
    for n, u, v in zip(("x", "y", "gate", "gamma_post", "gamma_pre", "E"), got, want):
        assert float((u.double() - v).norm() / v.norm()) < 2 ** -6, n
