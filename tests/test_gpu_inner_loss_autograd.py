"""The loss under autograd: what arrives from above (a loss divided by the accumulated micro-batches, a loss scale) multiplies the
gradient in fp32, and the product is rounded once."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def batch(rows, V, act, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (2.0 * torch.randn(rows, V, generator=g, device="cuda")).to(act)
    t = torch.randint(0, V, (rows,), generator=g, device="cuda")
    t[::5] = -100
    return x, t


def product(got, grad, d):
    """got is grad * d (both as they are stored) up to half a unit of fp32, rounded to got's type."""
    want = grad.double() * float(d)
    low, high = (want - want.abs() * 2.0 ** -24).to(got.dtype), (want + want.abs() * 2.0 ** -24).to(got.dtype)
    assert torch.all((got >= low) & (got <= high)), (got.double() - want).abs().max()


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 7), (37, 1001), (500, 4096), (64, 32000)])
@pytest.mark.parametrize("d", [1.0, 1.0 / 3.0, 1.0 / 12.0, 65536.0, 0.0, -0.7])
def test_what_arrives_from_above(rows, V, act, d):
    from paper_2508_15706_b200 import inner
    x, t = batch(rows, V, act)
    if rows == 1:
        t[0] = 0
    grad = torch.empty_like(x)
    total, _, _ = inner.token_loss(x, t, grad=grad, smoothing=0.05, z=1e-4)
    leaf = x.clone().requires_grad_()
    d32 = torch.tensor(d, device="cuda")
    loss = inner.next_token_loss(leaf, t, smoothing=0.05, z=1e-4)
    assert torch.equal(loss.view(1), total)
    (loss * d32).backward(retain_graph=True)
    product(leaf.grad, grad, d32.item())
    first, leaf.grad = leaf.grad, None
    (loss * d32).backward()  # a second pass over the same graph
    assert torch.equal(leaf.grad, first)


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
def test_scale_acts_before_the_only_rounding(act):
    from paper_2508_15706_b200 import inner
    x, t = batch(40, 999, act)
    grad = torch.empty_like(x)
    total, _, _ = inner.token_loss(x, t, grad=grad, scale=1.0 / 3.0)
    leaf = x.clone().requires_grad_()
    loss = inner.next_token_loss(leaf, t, scale=1.0 / 3.0)
    loss.backward()
    assert torch.equal(loss.view(1), total) and torch.equal(leaf.grad, grad)


def test_any_place_and_refusals():
    """Elements off a 16-byte boundary, in place, none at all; null pointers, types and alignment refused."""
    from paper_2508_15706_b200 import binding as B
    from paper_2508_15706_b200 import inner
    L, q = inner._L, torch.cuda.current_stream().cuda_stream
    up = torch.tensor([0.3], device="cuda")
    for act, code in ((torch.float32, 0), (torch.bfloat16, 1)):
        for shift in (0, 1, 3):
            for n in (0, 1, 5, 8, 1023, 4096 * 8 + 3):
                buf = torch.randn(n + 8, device="cuda").to(act)
                x, keep = buf[shift:shift + n], buf.clone()
                out = torch.full_like(buf, 9.0)
                assert L.sl_token_loss_backward(code, n, x.data_ptr(), up.data_ptr(), out[shift:].data_ptr(), q) == B.SL_OK
                product(out[shift:shift + n], x, up.item())
                assert torch.all(out[:shift] == 9.0) and torch.all(out[shift + n:] == 9.0)
                assert L.sl_token_loss_backward(code, n, x.data_ptr(), up.data_ptr(), x.data_ptr(), q) == B.SL_OK
                assert torch.equal(x, out[shift:shift + n]) and torch.equal(buf[:shift], keep[:shift]) and torch.equal(buf[shift + n:], keep[shift + n:])
    p = up.data_ptr()
    assert L.sl_token_loss_backward(0, 4, None, p, p, q) == B.SL_ERR_INVALID_ARG and L.sl_token_loss_backward(0, 4, p, None, p, q) == B.SL_ERR_INVALID_ARG
    assert L.sl_token_loss_backward(0, -1, p, p, p, q) == B.SL_ERR_INVALID_ARG and L.sl_token_loss_backward(2, 1, p, p, p, q) == B.SL_ERR_UNSUPPORTED
    assert L.sl_token_loss_backward(0, 1, p + 2, p, p, q) == B.SL_ERR_ALIGNMENT and L.sl_token_loss_backward(0, (1 << 40) + 1, p, p, p, q) == B.SL_ERR_TOO_LARGE
