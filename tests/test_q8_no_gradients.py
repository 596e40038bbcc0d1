"""The 8-bit operators give no gradients, and say so instead of losing them: a tensor that requires them is refused while autograd
records."""
import pytest
import torch

from paper_2507_17301_b200 import build

build.build()
from paper_2507_17301_b200 import nm  # noqa: E402


def test_refused_while_autograd_records():
    """(No GPU: the refusal comes before that of a host tensor.)"""
    x, g = torch.zeros(4, 64), torch.zeros(4, 64, requires_grad=True)
    for call in (lambda: nm.nm_q8_rows(g), lambda: nm.nm_q8_silu_mul(g, x), lambda: nm.nm_q8_rmsnorm(g, x[0])):
        with pytest.raises(TypeError, match="requires gradients"):
            call()
        for off in (torch.no_grad(), torch.inference_mode()):
            with off, pytest.raises(TypeError, match="two-dimensional"):
                call()
    with pytest.raises(TypeError, match="two-dimensional"):
        nm.nm_q8_rows(g.detach())


@pytest.mark.gpu
def test_every_argument_that_can_require_them():
    x, w, r = torch.randn(4, 64).cuda(), torch.ones(64).cuda(), torch.randn(4, 64).cuda()
    h = nm.nm_q8_prune(torch.randn(32, 64).cuda().requires_grad_(), 2, 4, 8)        # (a parameter can be pruned: the handle is a constant)
    q, s = nm.nm_q8_rows(x)
    b = torch.zeros(32).cuda()
    y = nm.nm_q8_linear(h, q, s, bias=b)
    calls = [(lambda t: nm.nm_q8_rows(t), x), (lambda t: nm.nm_q8_silu_mul(t, r), x), (lambda t: nm.nm_q8_silu_mul(r, t), x),
             (lambda t: nm.nm_q8_rmsnorm(t, w), x), (lambda t: nm.nm_q8_rmsnorm(x, t), w), (lambda t: nm.nm_q8_rmsnorm(x, w, residual=t), r),
             (lambda t: nm.nm_q8_linear(h, q, t), s), (lambda t: (nm.nm_q8_linear(h, q, s, bias=t),), b)]
    for call, t in calls:
        leaf = t.clone().requires_grad_()
        want = call(t)
        with pytest.raises(TypeError, match="requires gradients"):
            call(leaf)
        with torch.no_grad():
            got = call(leaf)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        got = call(leaf.detach())
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    with torch.no_grad():
        assert torch.equal(nm.nm_q8_linear(h, q, s, bias=torch.nn.Parameter(b)), y)
