"""lse of rows with an infinite score, as its formula has it: +inf with one of +inf, -inf where all are -inf, NaN with one of NaN; out is NaN in all of them."""
import pytest
import torch

from test_gpu_inner_attention import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,d", [(torch.float32, 64), (torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 200)])
@pytest.mark.parametrize("at", [0, 5, 14, 100, 207])
def test_infinite_lse(act, d, at):
    from paper_2508_15706_b200 import inner
    n = 210
    q, k, v, _ = make([n], 0, 1, 1, d, act, 71, "apart")
    q[:, 0, 0], q[3::7, 0, 0] = 1.0, -1.0
    k[at, 0, 0] = float("inf")
    out, lse = inner.attention_forward(q, k, v, causal=True)
    seen = torch.arange(n, device="cuda") >= at
    up = q[:, 0, 0] > 0
    assert torch.all(lse[0, seen & up] == float("inf")) and torch.all(torch.isnan(out[seen & up]))
    assert torch.all(torch.isfinite(lse[0, ~seen])) and torch.all(torch.isfinite(out[~seen]))
    rest = seen & ~up
    if at == 0 and rest[0]:
        assert lse[0, 0] == float("-inf")
    alone = rest & (torch.arange(n, device="cuda") == 0)
    assert torch.all(torch.isfinite(lse[0, rest & ~alone])) and torch.all(torch.isfinite(out[rest & ~alone]))
    k[at, 0, 0] = float("nan")
    out, lse = inner.attention_forward(q, k, v, causal=True)
    assert torch.equal(torch.isnan(lse[0]), seen) and torch.equal(torch.isnan(out[:, 0]).all(1), seen)


@pytest.mark.parametrize("act,d", [(torch.float32, 64), (torch.bfloat16, 64)])
def test_nothing_but_scores_of_minus_infinity(act, d):
    from paper_2508_15706_b200 import inner
    q, k, v, _ = make([70], 0, 1, 1, d, act, 72, "apart")
    q[:, 0, 0] = -1.0
    k[:20, 0, 0] = float("inf")
    out, lse = inner.attention_forward(q, k, v, causal=True)
    assert torch.all(lse[0, :20] == float("-inf")) and torch.all(torch.isnan(out[:20]))
    assert torch.all(torch.isfinite(lse[0, 20:])) and torch.all(torch.isfinite(out[20:]))
