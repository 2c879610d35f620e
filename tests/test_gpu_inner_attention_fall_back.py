"""Tiles with infinities or NaN in masked places, formed by the fp32 code one behind the other in the same shared memory: many of them, every run with
the same bits."""
import pytest
import torch

from test_gpu_inner_attention import formula, inside, make, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("causal", [True, False])
def test_many_tiles_repeat(act, d, bad, causal):
    """Every fourth sequence holds nothing finite; the others keep their formula's values."""
    from paper_2508_15706_b200 import inner
    lengths = [53, 20, 41, 77] * 12
    n = sum(lengths)
    q, k, v, dout = make(lengths, 0, 4, 2, d, act, 61, "apart")
    off = table(lengths)
    bounds = off.tolist()
    want, tol = formula(q, k, v, lengths, causal, d ** -0.5)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    for s in range(1, len(lengths), 4):
        keep[bounds[s]:bounds[s + 1]] = False
    for x in (q, k, v, dout):
        x[~keep] = bad
    runs = []
    for _ in range(12):
        out, lse = inner.attention_forward(q, k, v, off, causal=causal)
        runs.append((out, lse.t(), *inner.attention_backward(dout, q, k, v, out, lse, off, causal=causal)))
    for r in runs:
        assert all(torch.all(torch.isfinite(x[keep])) for x in r)
        assert all(torch.equal(x[keep], y[keep]) for x, y in zip(r, runs[0]))
    inside(runs[0][0][keep], want["out"][keep], tol["out"][keep], "out")
    inside(runs[0][1][keep], want["lse"].t()[keep], tol["lse"].t()[keep], "lse")
    for s in (0, 2, 22, 47):
        at, m = slice(bounds[s], bounds[s + 1]), [lengths[s]]
        want_g, tol_g = formula(q[at], k[at], v[at], m, causal, d ** -0.5, dout[at], runs[0][0][at], runs[0][1][at].t())
        for name, x in zip(("dq", "dk", "dv"), runs[0][2:]):
            inside(x[at], want_g[name], tol_g[name], name)
