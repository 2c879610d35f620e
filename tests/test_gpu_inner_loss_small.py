"""Losses that are small beside the logits they come from: logits are defined up to a constant, and so is the loss's accuracy.

Tolerance (u = 2^-24): the sum of a row is good to r = 2 (vocab / 512 + 20) u relative, which is the error of its logarithm; the
difference to the target's logit adds 4 u of itself.  Nothing in it grows with the constant.  With smoothing, the mean of
the logits is a sum of numbers of their own size: 2^-20 of the largest."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("rows,V", [(300, 512), (5, 4097), (3, 32000), (400, 32000), (1, 300001)])
@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [0.0, 30.0, -30.0, 1000.0, -1000.0, 30000.0, 3e6, -3e6])
def test_loss_does_not_lose_by_a_constant(rows, V, act, c):
    from paper_2508_15706_b200 import inner
    g = torch.Generator(device="cuda").manual_seed(V)
    t = torch.randint(0, V, (rows,), generator=g, device="cuda")
    for low, high in ((18.0, 40.0), (0.0, 12.0)):  # well predicted; not
        x = (c - low - (high - low) * torch.rand(rows, V, generator=g, device="cuda")).to(act)
        x.scatter_(1, t[:, None], torch.full((rows, 1), c, device="cuda").to(act))
        x64 = x.double()
        want = -torch.log_softmax(x64, 1).gather(1, t[:, None])[:, 0]
        for t_ in (t, torch.roll(t, 1)):
            want = -torch.log_softmax(x64, 1).gather(1, t_[:, None])[:, 0]
            _, loss, _ = inner.token_loss(x, t_)
            assert torch.all(loss >= 0)
            assert torch.all((loss.double() - want).abs() <= 2 * (V / 512 + 20) * U + 4 * U * want), (low, (loss.double() - want).abs().max(), want.max())
            _, loss, _ = inner.token_loss(x, t_, smoothing=0.1)
            smooth = torch.logsumexp(x64 - c, 1) - 0.9 * (x64 - c).gather(1, t_[:, None])[:, 0] - 0.1 * (x64 - c).mean(1)
            assert torch.all((loss.double() - smooth).abs() <= 2 * (V / 512 + 20) * U + 4 * U * smooth.abs() + 2.0 ** -20 * 0.1 * x64.abs().amax(1))


def test_all_smoothing_takes_nothing_from_a_masked_target():
    from paper_2508_15706_b200 import inner
    x = torch.zeros(2, 64, device="cuda")
    x[0, 3] = float("-inf")
    t = torch.tensor([3, 3], device="cuda")
    _, loss, _ = inner.token_loss(x, t, smoothing=1.0)
    assert loss[0] == float("inf") and abs(loss[1].item() - 4.1588830833596715) < 1e-6
