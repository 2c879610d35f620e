"""Some outputs given, others left out: rows of tokens in no sequence are left as they were in those that are given, and 0 (lse -inf) in those
allocated by the call, whatever stood in that memory."""
import itertools

import pytest
import torch

from test_gpu_inner_attention import make, table

pytestmark = pytest.mark.gpu


def spoil():
    """Leaves NaN in the memory that the next allocations get."""
    junk = [torch.full((1 << 16,), float("nan"), device="cuda") for _ in range(12)]
    junk += [torch.full((1 << 8,), float("nan"), device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    del junk


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths,rest", [([33, 100], 150), ([], 40), ([300], 7)])
def test_mixed_outputs(act, lengths, rest):
    from paper_2508_15706_b200 import inner
    q, k, v, dout = make(lengths, rest, 2, 1, 64, act, 41, "apart")
    off, n, t = table(lengths), sum(lengths), sum(lengths) + rest
    out, lse = inner.attention_forward(q, k, v, off)
    grads = inner.attention_backward(dout, q, k, v, out, lse, off)
    for mine in itertools.product([False, True], repeat=2):
        spoil()
        o, s = (x if use else None for use, x in zip(mine, (torch.full_like(out, 7.0), torch.full_like(lse, 7.0))))
        o, s = inner.attention_forward(q, k, v, off, out=o, lse=s)
        assert torch.equal(o[:n], out[:n]) and torch.equal(s[:, :n], lse[:, :n])
        assert torch.all(o[n:] == (7.0 if mine[0] else 0.0)) and torch.all(s[:, n:] == (7.0 if mine[1] else float("-inf"))), mine
    for mine in itertools.product([False, True], repeat=3):
        spoil()
        given = [torch.full_like(x, 7.0) if use else None for use, x in zip(mine, grads)]
        got = inner.attention_backward(dout, q, k, v, out, lse, off, dq=given[0], dk=given[1], dv=given[2])
        for x, y, use in zip(got, grads, mine):
            assert torch.equal(x[:n], y[:n]) and torch.all(x[n:] == (7.0 if use else 0.0)), mine
    assert t == len(out)
