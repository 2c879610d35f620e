"""AdamW where eps is small and the second moment denormal: the denominator sqrt(v) / sqrt(1 - beta2^t) + eps has to keep both terms.

Tolerance: the update from the stored moments, root and quotient 2^-22 each and a few roundings: 2^-20 relative."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-18, 1e-16, 1e-15, 1e-14, 1e-13, 1e-12, 1e-11, 1e-10, 1e-8])
@pytest.mark.parametrize("beta2,step", [(0.999, 1), (0.95, 1), (0.9999, 1), (0.999, 1000)])
def test_denormal_second_moment(eps, beta2, step):
    from paper_2508_15706_b200.inner import AdamW
    n = 4099
    opt = AdamW([(1, n)], weight_decay=0.0, betas=(0.9, beta2), eps=eps, max_norm=0.0)
    g = torch.Generator(device="cuda").manual_seed(1)
    size = 10.0 ** (-21.0 + 6.0 * torch.rand(n, generator=g, device="cuda"))  # v from below the smallest denormal to normal numbers
    grad = size * torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    theta, (m, v, _) = torch.zeros(n, device="cuda"), opt.new_state()
    opt.step(theta, grad, m, v, step=step, lr=1.0)
    e = torch.tensor(eps).double().item()  # (as fp32)
    want = -(m.double() / (1 - 0.9 ** step)) / (v.double().sqrt() / math.sqrt(1 - beta2 ** step) + torch.tensor(e, dtype=torch.float32).double().item())
    fine = torch.isfinite(want) & (want.abs() < 1e37)
    assert fine.sum() > n // 2
    assert torch.all((theta.double() - want).abs()[fine] <= 2.0 ** -20 * want.abs()[fine] + 1e-44)
