"""Where the norms write: the very rows that they read, or elsewhere."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def refused(fn, *a, **k):
    from paper_2508_15706_b200 import binding as B
    with pytest.raises(B.SlError) as e:
        fn(*a, **k)
    assert e.value.status == B.SL_ERR_INVALID_ARG


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [7, 64])
def test_same_address_with_another_row_stride_is_refused(act, cols):
    from paper_2508_15706_b200 import inner
    buf = torch.randn(6 * 2 * cols, device="cuda").to(act)
    wide, narrow = buf.view(6, 2 * cols)[:, :cols], buf[:6 * cols].view(6, cols)
    other = [torch.randn(6, cols, device="cuda").to(act) for _ in range(4)]
    w, r = torch.ones(cols, device="cuda"), torch.ones(6, device="cuda")
    before = buf.clone()
    refused(inner.norm_forward, wide, w, h=narrow)
    refused(inner.norm_forward, wide, w, branch=other[0], y=narrow)
    refused(inner.norm_forward, other[0], w, branch=wide, h=narrow)
    refused(inner.norm_forward, other[0], w, branch=other[1], gate=wide, y=narrow)
    refused(inner.norm_backward, wide, other[0], other[1], w, rstd=r, dx=narrow)
    refused(inner.norm_backward, other[0], wide, other[1], w, rstd=r, dx=narrow)
    refused(inner.norm_backward, other[0], other[1], wide, w, rstd=r, dx=narrow)
    refused(inner.norm_backward, wide, None, None, branch=other[0], dbranch=narrow)
    refused(inner.norm_backward, other[0], None, None, branch=wide, gate=other[1], dgate=narrow)
    assert torch.equal(buf, before)


def test_a_single_row_has_no_row_stride():
    from paper_2508_15706_b200 import inner
    buf, w = torch.randn(1, 96, device="cuda"), torch.ones(48, device="cuda")
    x = buf[:, :48]
    want = inner.norm_forward(x.clone(), w)[1]
    inner.norm_forward(x, w, h=buf.view(-1)[:48].view(1, 48))
    assert torch.equal(x, want)
