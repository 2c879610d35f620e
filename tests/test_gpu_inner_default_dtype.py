"""What is allocated within a call does not depend on torch's default type (a program that builds its model under
torch.set_default_dtype(torch.bfloat16) calls the same operators)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
def test_operators_under_another_default_type(default):
    from paper_2508_15706_b200 import inner
    before = torch.get_default_dtype()
    x = torch.randn(6, 64, device="cuda").bfloat16()
    w, t = torch.ones(64, device="cuda"), torch.arange(6, device="cuda")

    def all_of_them():
        leaf = x.detach().clone().requires_grad_()
        y, h = inner.block_norm(leaf, w, branch=2 * leaf)
        q, _ = inner.rotary(inner.Rotary(64), h.view(1, 6, 1, 64))
        loss = inner.next_token_loss(q.view(6, 64) + y, t)
        loss.backward()
        opt = inner.AdamW([(6, 64)], grad_dtype=torch.bfloat16, param_dtype=torch.bfloat16)
        theta, state = x.clone().view(-1), opt.new_state()
        opt.step(theta, leaf.grad.view(-1), *state, step=1, lr=1e-2)
        return [loss.detach(), leaf.grad, theta, *inner.token_loss(x, t), *inner.norm_forward(x, w)[1:3]]

    want = all_of_them()
    torch.set_default_dtype(default)
    try:
        got = all_of_them()
    finally:
        torch.set_default_dtype(before)
    assert all(a.dtype is b.dtype and torch.equal(a, b) for a, b in zip(got, want))
