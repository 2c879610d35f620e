"""NaN in a gradient that arrives reaches the gradients of every key that its query sees, whatever the weight."""
import pytest
import torch

from test_gpu_inner_attention import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [32, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_nan_gradient_reaches_weights_that_vanish(act, d, causal):
    """Scores 200 apart: all weights but one are 0 in fp32.  A NaN in the gradient of token 60 still makes the gradients of every key it sees
    NaN, as p (dp - delta) does, and leaves the others finite."""
    from paper_2508_15706_b200 import inner
    n = 150
    q, k, v, dout = make([n], 0, 1, 1, d, act, 23, "apart")
    q.zero_(), k.zero_()
    q[:, 0, 0], k[:, 0, 0] = 200.0, torch.arange(n, device="cuda").to(act)
    out, lse = inner.attention_forward(q, k, v, causal=causal, scale=1.0)
    dout[60, 0, 2] = float("nan")
    dq, dk, dv = inner.attention_backward(dout, q, k, v, out, lse, causal=causal, scale=1.0)
    seen = torch.arange(n, device="cuda") <= 60 if causal else torch.ones(n, dtype=torch.bool, device="cuda")
    assert torch.all(torch.isnan(dq[60])) and torch.all(torch.isfinite(dq[:60])) and torch.all(torch.isfinite(dq[61:]))
    assert torch.all(torch.isnan(dk[seen])) and torch.all(torch.isfinite(dk[~seen]))
    assert torch.all(torch.isnan(dv[seen][..., 2])) and torch.all(torch.isfinite(dv[~seen])) and torch.all(torch.isfinite(dv[..., 3:]))
