"""What follows attention's backward pass in the stream comes after all of its kernels, whatever the table of sequences holds."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("entries", [[0], [0, 0, 0], [19000, 19000], [0, 5], [0, 700, 701]])
def test_workspace_is_free_behind_the_call(d, entries):
    """The workspace is overwritten behind the call: no kernel of the call may still write to it.  Tables without a live token, where no tile has
    anything to wait for, and with few."""
    from paper_2508_15706_b200 import inner
    n = 19000
    g = torch.Generator(device="cuda").manual_seed(51)
    q, k, v, dout = (torch.randn(n, h, d, generator=g, device="cuda").bfloat16() for h in (8, 2, 2, 8))
    off = torch.tensor(entries, dtype=torch.int32, device="cuda")
    out, lse = inner.attention_forward(q, k, v, off)
    want = inner.attention_backward(dout, q, k, v, out, lse, off)
    work = [inner.attention_workspace(q, k, off) for _ in range(4)]
    got = []
    for i in range(16):
        got.append(inner.attention_backward(dout, q, k, v, out, lse, off, workspace=work[i % 4]))
        work[i % 4].fill_(0xA5)
    torch.cuda.synchronize()
    assert all(torch.all(w == 0xA5) for w in work)
    live = torch.zeros(n, dtype=torch.bool, device="cuda")
    live[entries[0]:entries[-1]] = True
    for grads in got:
        for x, y in zip(grads, want):
            assert torch.equal(x, y) and torch.all(x[~live] == 0)
