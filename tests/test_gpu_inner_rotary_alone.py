"""Queries without keys through the autograd function (cross attention, a head that is turned alone): the same as with keys."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
def test_queries_alone(act):
    from paper_2508_15706_b200 import inner
    rope = inner.Rotary(32, layout="interleaved")
    q = torch.randn(2, 9, 3, 48, device="cuda").to(act).requires_grad_()
    k = torch.randn(2, 9, 1, 48, device="cuda").to(act)
    pos = torch.randint(0, 500, (2, 9), device="cuda")
    w = torch.randn(2, 9, 3, 48, device="cuda").to(act)
    both, _ = inner.rotary(rope, q, k, pos)
    want, = torch.autograd.grad((both * w).sum(), q)
    for alone in (inner.rotary(rope, q, None, pos), inner.rotary(rope, q, positions=pos)):
        assert alone[1] is None and torch.equal(alone[0], both)
        got, = torch.autograd.grad((alone[0] * w).sum(), q)
        assert torch.equal(got, want)
