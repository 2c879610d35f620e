"""Calls of attention and of the rows' combine that are refused with the library's own error."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_scale_that_fp32_cannot_hold():
    from paper_2508_15706_b200 import inner
    from paper_2508_15706_b200.binding import SlError
    q = torch.randn(9, 1, 8, device="cuda")
    out, lse = inner.attention_forward(q, q, q)
    for scale in (1e39, -1e39, 1e300, float("inf"), float("-inf"), float("nan"), 0.0, 1e-60, -1.0):
        with pytest.raises(SlError):
            inner.attention_forward(q, q, q, scale=scale)
        with pytest.raises(SlError):
            inner.attention_backward(q, q, q, q, out, lse, scale=scale)
        with pytest.raises(SlError):
            inner.attention(q, q, q, scale=scale)


def test_tensors_of_other_dimensions_under_autograd():
    from paper_2508_15706_b200 import inner
    from paper_2508_15706_b200.binding import SlError
    good = torch.randn(6, 1, 8, device="cuda")
    for bad in (torch.randn((), device="cuda"), torch.randn(1, device="cuda"), torch.randn(16, device="cuda"), torch.randn(32, device="cuda")[::2], torch.randn(6, 8, device="cuda"), torch.randn(8, 6, device="cuda").t(),
                torch.randn(2, 2, 6, 1, 8, device="cuda")):
        for q, k, v in ((bad, bad, bad), (bad, good, good), (good, bad, bad), (good, good, bad)):
            with pytest.raises(SlError):
                inner.attention(q, k, v)


def test_rows_of_other_dimensions_under_autograd():
    from paper_2508_15706_b200 import inner
    from paper_2508_15706_b200.binding import SlError
    r = inner.route(torch.randn(4, 8, device="cuda"), 2)
    for bad in (torch.randn((), device="cuda"), torch.randn(8, device="cuda"), torch.randn(8, 1, 16, device="cuda")):
        with pytest.raises(SlError):
            inner.combine(bad, r)
