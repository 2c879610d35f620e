"""NaN and infinities that a query sees reach its results, whichever token holds them."""
import pytest
import torch

from test_gpu_inner_attention import formula, inside, make, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,d", [(torch.float32, 64), (torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 40), (torch.bfloat16, 200)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("which", ["k", "q", "v"])
def test_nan_at_every_place_of_a_tile(act, d, causal, which):
    """One NaN at one of 32 consecutive tokens: in k (v finite), every query that sees the key is NaN, out and lse; in q that query alone; in v
    that component alone.  Everything else keeps its formula's value."""
    from paper_2508_15706_b200 import inner
    lengths, rest, at = [90, 190, 60], 9, 180
    q, k, v, _ = make(lengths, rest, 2, 1, d, act, 21, "apart")
    off, n = table(lengths), sum(lengths)
    want, tol = formula(q, k, v, lengths, causal, d ** -0.5)
    token = torch.arange(n, device="cuda")
    for t in range(at, at + 32):
        x = {"k": k, "q": q, "v": v}[which]
        kept = x[t, 0, 5].clone()
        x[t, 0, 5] = float("nan")
        out, lse = inner.attention_forward(q, k, v, off, causal=causal)
        x[t, 0, 5] = kept
        sees = (token >= (t if causal else 90)) & (token < 280)
        bad = torch.zeros(n, 2, d, dtype=torch.bool, device="cuda")
        if which == "k":
            bad[sees] = True
        elif which == "q":
            bad[t, 0] = True
        else:
            bad[..., 5] = sees[:, None]
        bad_lse = torch.zeros_like(bad[..., 0]) if which == "v" else bad[..., 0]
        assert torch.equal(torch.isnan(out[:n]), bad), t
        assert torch.equal(torch.isnan(lse[:, :n].t()), bad_lse), t
        inside(out[:n][~bad], want["out"][:n][~bad], tol["out"][:n][~bad], t)
        inside(lse[:, :n].t()[~bad_lse], want["lse"][:, :n].t()[~bad_lse], tol["lse"][:, :n].t()[~bad_lse], t)


@pytest.mark.parametrize("act,d", [(torch.float32, 64), (torch.bfloat16, 64), (torch.bfloat16, 128)])
def test_infinite_scores_at_every_place_of_a_tile(act, d):
    """An infinity in k: a score of +inf leaves no finite result, one of -inf has weight 0.  Errors of the other weights: 2^-8 of their size as
    operands in bfloat16 and below 2^-12 from scores, exponentials and sums, all of them times at most max |v|; the output's own 2^-8."""
    from paper_2508_15706_b200 import inner
    n = 200
    q, k, v, _ = make([n], 0, 1, 1, d, act, 22, "apart")
    x = (q[:, 0].double() @ k[:, 0].double().t()) * d ** -0.5
    pr = 2.0 ** -8 if act is torch.bfloat16 else 0.0
    for t in range(96, 128):
        kept = k[t, 0, 3].clone()
        k[t, 0, 3] = float("inf")
        out, lse = inner.attention_forward(q, k, v, causal=False)
        k[t, 0, 3] = kept
        up = q[:, 0, 3] > 0
        assert not torch.any(torch.isfinite(out[up])) and not torch.any(torch.isfinite(lse[0, up]))
        y = x.clone()
        y[:, t] = float("-inf")
        want = y[~up].softmax(-1) @ v[:, 0].double()
        assert torch.all((out[~up, 0].double() - want).abs() <= (pr + 2.0 ** -12) * v.abs().max().double() + pr * want.abs()), t
        assert torch.all((lse[0, ~up].double() - y[~up].logsumexp(-1)).abs() <= 2.0 ** -12), t
