"""Outputs that cannot be allocated."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_memory_that_is_not_there():
    """Outputs that cannot be allocated raise what torch raises, and the next call works."""
    from paper_2508_15706_b200 import inner
    with pytest.raises(torch.OutOfMemoryError):
        inner._empties(0, torch.float32, 1 << 20, 1 << 20)
    x = torch.randn(5, 1, 8, device="cuda")
    assert torch.all(torch.isfinite(inner.attention_forward(x, x, x)[0]))
