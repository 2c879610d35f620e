"""Attention over more than 2^20 tokens, in the larger case 2^31 elements and more."""
import pytest
import torch

from test_gpu_inner_attention import formula, inside, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk,d", [(1, 1, 16), (16, 2, 128)])
def test_more_than_2_20_tokens(hq, hk, d):
    """Many short sequences; the first, some and the last are compared with the formula, rows behind them with 0."""
    from paper_2508_15706_b200 import inner
    lengths, rest = [128] * 8191 + [101, 128, 77], 30
    n = sum(lengths) + rest
    assert n > 2 ** 20
    g = torch.Generator(device="cuda").manual_seed(31)
    q, k, v, dout = (torch.randn(n, h, d, generator=g, device="cuda", dtype=torch.bfloat16) for h in (hq, hk, hk, hq))
    off = table(lengths)
    out, lse = inner.attention_forward(q, k, v, off)
    grads = inner.attention_backward(dout, q, k, v, out, lse, off)
    assert lse.shape == (hq, n) and torch.all(out[n - rest:] == 0) and torch.all(lse[:, n - rest:] == float("-inf"))
    bounds = off.tolist()
    for s in (0, 1, 4000, 8191, 8192, 8193):
        at = slice(bounds[s], bounds[s + 1])
        m = [bounds[s + 1] - bounds[s]]
        want, tol = formula(q[at], k[at], v[at], m, True, d ** -0.5)
        inside(out[at], want["out"], tol["out"], ("out", s))
        inside(lse[:, at], want["lse"], tol["lse"], ("lse", s))
        want, tol = formula(q[at], k[at], v[at], m, True, d ** -0.5, dout[at], out[at], lse[:, at])
        for name, x in zip(("dq", "dk", "dv"), grads):
            inside(x[at], want[name], tol[name], (name, s))
    assert all(torch.all(x[n - rest:] == 0) for x in grads)
