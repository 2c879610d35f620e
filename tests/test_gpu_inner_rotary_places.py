"""Where a rotary call writes: the very elements that it reads, or elsewhere.  (No call here is expected to run with outputs that overlap.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu


def refused(fn, *a, **k):
    from paper_2508_15706_b200 import binding as B
    with pytest.raises(B.SlError) as e:
        fn(*a, **k)
    assert e.value.status == B.SL_ERR_INVALID_ARG


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
def test_same_address_with_other_strides_is_refused(act):
    from paper_2508_15706_b200.inner import Rotary
    rope = Rotary(8)
    buf = torch.randn(2 * 4 * 2 * 32, device="cuda").to(act)
    q = buf.view(2, 4, 2, 32)[..., :16]
    narrow = buf[:2 * 4 * 2 * 16].view(2, 4, 2, 16)
    before = buf.clone()
    other = torch.zeros(2, 4, 2, 16, device="cuda", dtype=act)
    refused(rope.apply, q, out_q=narrow)
    refused(rope.apply, other.clone(), q, out_q=other, out_k=narrow)
    refused(rope.apply, q, out_q=buf.view(2, 2, 4, 32).transpose(1, 2)[..., :16])  # tokens and heads the other way round
    assert torch.equal(buf, before)


def test_strides_of_single_elements_do_not_count():
    from paper_2508_15706_b200.inner import Rotary
    rope = Rotary(8)
    buf = torch.randn(4 * 2 * 16, device="cuda")
    q = buf.view(1, 4, 2, 16)
    want = torch.empty_like(q)
    rope.apply(q, out_q=want)
    rope.apply(q, out_q=buf.as_strided((1, 4, 2, 16), (7, 32, 16, 1)))
    assert torch.equal(q, want)
    one = torch.randn(1, 1, 1, 16, device="cuda")
    rope.apply(one, first=3, out_q=(w := torch.empty_like(one)))
    rope.apply(one, first=3, out_q=one.as_strided((1, 1, 1, 16), (1, 2, 3, 1)))
    assert torch.equal(one, w)


@pytest.mark.parametrize("dim", [0, 1, 2])
def test_outputs_shared_along_a_dimension_are_refused(dim):
    """A key head expanded over the query heads, one token over a sequence: fine as an input, not as what is written."""
    from paper_2508_15706_b200.inner import Rotary
    rope = Rotary(16)
    shape = [2, 5, 4, 16]
    shape[dim] = 1
    one = torch.randn(shape, device="cuda")
    shared, before = one.expand(2, 5, 4, 16), one.clone()
    refused(rope.apply, shared)
    refused(rope.apply, shared.contiguous(), shared)
    refused(rope.apply, shared.contiguous(), out_q=shared)
    assert torch.equal(one, before)
    out, want = torch.empty(2, 5, 4, 16, device="cuda"), shared.contiguous()
    rope.apply(shared, out_q=out)
    rope.apply(want)
    assert torch.equal(out, want)
