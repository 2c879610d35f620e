"""Next-token loss of rows whose vocabulary is masked over whole threads' worth of logits while the rest lies anywhere: logits are
defined up to a constant, so a row's largest may well be -100 or -1000.  Formulas and tolerances: test_gpu_inner_loss.py (a masked
logit's gradient is 0 exactly there)."""
import pytest
import torch

from test_gpu_inner_loss import check, make

pytestmark = pytest.mark.gpu

# few rows and many; a vector per thread and several; a row spread over a cluster; rows without a common boundary; more than eight CTAs hold
SIZES = [(3, 512), (9, 1001), (400, 1024), (700, 4096), (500, 4097), (2, 32000), (400, 32000), (5, 31999), (1, 300001)]


@pytest.mark.parametrize("rows,V", SIZES)
@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [-1000.0, -100.0, -89.0, 0.0, 1000.0])
@pytest.mark.parametrize("mask", ["tail", "front", "all but a few"])
@pytest.mark.parametrize("kw", [{}, {"z": 1e-3, "mean": False, "scale": 0.5}])
def test_masked_stretches(rows, V, act, shift, mask, kw):
    from paper_2508_15706_b200 import inner
    x, t = make(rows, V, act, rows + V, ignored=0.2)
    x = (x.float() + shift).to(act)
    g = torch.Generator(device="cuda").manual_seed(5)
    if mask == "tail":
        x[:, V // 3:] = float("-inf")
        keep = torch.arange(V // 3, device="cuda")
    elif mask == "front":
        x[:, :V - V // 4] = float("-inf")
        keep = torch.arange(V - V // 4, V, device="cuda")
    else:
        keep = torch.randperm(V, generator=g, device="cuda")[:5]
        gone = torch.ones(V, dtype=torch.bool, device="cuda")
        gone[keep] = False
        x[:, gone] = float("-inf")
    t = torch.where(t == -100, t, keep[torch.randint(0, keep.numel(), (rows,), generator=g, device="cuda")])
    grad = torch.full_like(x, 9.0)
    check(x, t, inner.token_loss(x, t, grad=grad, **kw), grad, **kw)
    assert torch.all(grad[x == float("-inf")] == 0)
