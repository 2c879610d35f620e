"""The autograd functions have first derivatives only: a second one (a gradient penalty, say) raises and is not silently taken for zero."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def outputs(which, x):
    from paper_2508_15706_b200 import inner
    if which == "norm":
        return inner.block_norm(x, torch.ones(16, device="cuda"))[1].pow(3).sum()
    if which == "residual":
        return inner.block_norm(x, torch.ones(16, device="cuda"), branch=2 * x, gate=x, branch_weight=torch.ones(16, device="cuda"))[0].pow(3).sum()
    if which == "rotary":
        q = x.view(1, 6, 1, 16)
        return sum(t.pow(3).sum() for t in inner.rotary(inner.Rotary(16), q, q))
    return inner.next_token_loss(x, torch.arange(6, device="cuda")).pow(2)


@pytest.mark.parametrize("which", ["norm", "residual", "rotary", "loss"])
def test_second_derivative_raises(which):
    x = torch.randn(6, 16, device="cuda", requires_grad=True)
    plain, = torch.autograd.grad(outputs(which, x), x)
    g, = torch.autograd.grad(outputs(which, x), x, create_graph=True)
    assert torch.equal(g, plain)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (g.square().sum() + x.square().sum()).backward()
