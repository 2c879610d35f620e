"""Next-token loss and its gradient (sl_token_loss) against the formulas in 64 bits, and the gradient against differences.

Tolerances (u = 2^-24): exponentials and the sum of a row are good to (vocab / 512 + 20) u relative, about 2^-17 at 32000 and 2^-19 up to 4097;
lse and the loss add 4 u of their own size; the gradient's terms carry the relative error of the exponentials (whose argument is
rounded: |x - max| u); in bfloat16 it is the rounding of such a number."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(x, t, ignore, smoothing, z, mean, scale):
    rows, V = x.shape
    counts = t != ignore
    w = scale / max(1, int(counts.sum())) if mean else scale
    lse = torch.logsumexp(x, 1)
    at = torch.where(counts, t, torch.zeros_like(t))
    xt = x.gather(1, at[:, None])[:, 0]
    loss = lse - (1 - smoothing) * xt + z * lse ** 2
    if smoothing:
        loss = loss - smoothing * x.mean(1)
    loss = torch.where(counts, loss, torch.zeros_like(loss))
    p = torch.exp(x - lse[:, None])
    hit = torch.zeros_like(x)
    hit.scatter_(1, at[:, None], 1 - smoothing)
    grad = torch.where(counts[:, None], w * (p * (1 + 2 * z * lse[:, None]) - hit - smoothing / V), torch.zeros_like(x))
    size = torch.where(counts[:, None], abs(w) * (p * (1 + 2 * abs(z) * lse.abs()[:, None]) + hit + smoothing / V), torch.zeros_like(x))
    return (w * loss.sum(), loss, lse, grad, size)


def inside(got, want, tol, what=""):
    """got is want up to tol; stored in bfloat16, the rounding of some number up to tol from want (rounding keeps order)."""
    low, high = (want - tol).to(got.dtype), (want + tol).to(got.dtype)
    bad = ~((got >= low) & (got <= high))
    assert not torch.any(bad), (what, (got.double() - want)[bad][:4], want[bad][:4])


def rel(V):
    return 2.0 ** -19 if V <= 4097 else 2.0 ** -17


def check(x, t, out, grad, **k):
    total, loss, lse = out
    wt, wl, ws, wg, size = reference(x.double(), t.long(), k.get("ignore_index", -100), k.get("smoothing", 0.0), k.get("z", 0.0), k.get("mean", True), k.get("scale", 1.0))
    r = rel(x.shape[1])
    # the arguments of exponentials that are not 0
    top = torch.where(torch.exp(x.double() - ws[:, None]) > 0, x.double().abs(), torch.zeros_like(ws)[:, None]).amax(1) + 1
    assert torch.all((lse.double() - ws).abs() <= r + 4 * 2.0 ** -24 * top)
    zs = 1 + 2 * abs(k.get("z", 0.0)) * ws.abs()
    assert torch.all((loss.double() - wl).abs() <= (r + 8 * 2.0 ** -24 * top) * zs * 2)
    assert abs(total.item() - wt.item()) <= 2.0 ** -22 * wt.abs().item() + (abs(wt.item()) * 0 + (loss.double() - wl).abs().sum().item() * abs(k.get("scale", 1.0)))
    if grad is not None:
        inside(grad, wg, (r + 2.0 ** -22 * 2 * top[:, None]) * size * 2)


def make(rows, V, act, seed, pad=0, shift=0, ignored=0.3, ignore=-100):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = (3.0 * torch.randn(rows * (V + pad) + shift + 8, generator=g, device="cuda")).to(act)
    x = buf[shift:shift + rows * (V + pad)].view(rows, V + pad)[:, :V]
    t = torch.randint(0, V, (rows,), generator=g, device="cuda")
    t[torch.rand(rows, generator=g, device="cuda") < ignored] = ignore
    return x, t


CASES = [(1, 1, 0, 0), (3, 2, 0, 0), (2, 7, 0, 0), (65, 100, 0, 0), (9, 1000, 24, 0), (5, 1001, 0, 3), (4, 4096, 0, 0), (3, 4097, 7, 1), (2, 32000, 0, 0), (1, 31999, 0, 0), (700, 512, 0, 0)]


@pytest.mark.parametrize("rows,V,pad,shift", CASES)
@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kw", [{}, {"smoothing": 0.1, "z": 1e-3}, {"mean": False, "scale": 0.25, "z": 1e-2}, {"smoothing": 1.0}])
def test_loss_and_gradient(rows, V, pad, shift, act, kw):
    from paper_2508_15706_b200 import inner
    x, t = make(rows, V, act, rows + V, pad, shift)
    grad = torch.full_like(x, 9.0, memory_format=torch.contiguous_format)
    check(x, t, inner.token_loss(x, t, grad=grad, **kw), grad, **kw)
    check(x, t, inner.token_loss(x, t, **kw), None, **kw)  # loss alone
    other = torch.full((rows, V + pad + 8), 9.0, dtype=act, device="cuda")[:, :V]  # rows elsewhere relative to 16 bytes
    inner.token_loss(x, t.int(), grad=other, **kw)
    check(x, t, inner.token_loss(x, t.int(), grad=other, **kw), other, **kw)
    y = torch.empty_strided(x.shape, x.stride(), dtype=act, device="cuda").copy_(x)
    inner.token_loss(y, t, grad=y, **kw)  # in place
    inner.token_loss(x, t, grad=grad, **kw)
    assert torch.equal(y, grad) or (x.data_ptr() - y.data_ptr()) % 16 != 0
    check(x, t, inner.token_loss(x, t, grad=grad, **kw), y, **kw)


def test_masked_logits_and_rows():
    from paper_2508_15706_b200 import inner
    for act in (torch.float32, torch.bfloat16):
        x, t = make(12, 777, act, 4, ignored=0.0)
        low = torch.finfo(act).min
        x[0, 700:] = float("-inf")
        t[0] = 5
        x[1, 1:] = float("-inf")      # one entry left, and it is the target
        t[1] = 0
        x[2] = low                     # the type's lowest value everywhere: uniform
        x[3, :776] = low               # ... everywhere but at the last entry
        t[3] = 776
        x[4, 9] = float("-inf")       # the target itself is masked
        t[4] = 9
        x[5] = float("-inf")          # nothing left
        x[6, 3] = float("inf")
        x[7, 3] = float("nan")
        t[8] = 777                     # outside
        t[9] = -1
        t[10] = -100
        grad = torch.empty_like(x)
        total, loss, lse = inner.token_loss(x, t, grad=grad, mean=False)
        keep = [0, 1, 2, 3, 10, 11]
        check(x[keep].contiguous(), t[keep], (loss[keep].sum(), loss[keep], lse[keep]), grad[keep], mean=False)
        assert torch.all(grad[0, 700:] == 0) and loss[1] == 0 and torch.all(grad[1] == 0)
        assert loss[4] == float("inf") and torch.isfinite(lse[4]) and grad[4, 9] == -1 and torch.all(torch.isfinite(grad[4]))
        assert loss[5] == float("inf") and lse[5] == float("-inf") and torch.all(grad[5] == 0)
        assert torch.isnan(loss[6]) and torch.isnan(loss[7]) and torch.isnan(grad[7]).any()
        assert torch.isnan(loss[8]) and torch.isnan(loss[9]) and torch.all(grad[8:11] == 0) and loss[10] == 0
        assert torch.isnan(total)


def test_no_row_counts_and_no_rows():
    from paper_2508_15706_b200 import inner
    x, t = make(5, 64, torch.float32, 1)
    t[:] = 7
    grad = torch.ones_like(x)
    total, loss, _ = inner.token_loss(x, t, grad=grad, ignore_index=7)
    assert total.item() == 0 and torch.all(loss == 0) and torch.all(grad == 0)
    total, loss, _ = inner.token_loss(x[:0], t[:0])
    assert total.item() == 0 and loss.numel() == 0


def test_repeats_bit_for_bit_and_on_another_stream():
    from paper_2508_15706_b200 import inner
    x, t = make(1000, 5000, torch.bfloat16, 2)
    runs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            grad = torch.empty_like(x)
            runs.append([*inner.token_loss(x, t, grad=grad, z=1e-4), grad])
        stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_gradient_against_differences():
    """Central differences of the 64-bit loss (error about 1e-10) along random directions."""
    from paper_2508_15706_b200 import inner
    x, t = make(13, 203, torch.float32, 8)
    leaf = x.clone().requires_grad_()
    inner.next_token_loss(leaf, t, smoothing=0.2, z=1e-2).backward()
    for _ in range(3):
        d = torch.randn(13, 203, dtype=torch.float64, device="cuda")
        s = 1e-5
        up, down = (reference(x.double() + k * s * d, t, -100, 0.2, 1e-2, True, 1.0)[0].item() for k in (1, -1))
        got = (leaf.grad.double() * d).sum().item()
        assert abs(got - (up - down) / (2 * s)) <= 2.0 ** -17 * (leaf.grad.double() * d).abs().sum().item()


def test_refusals():
    from paper_2508_15706_b200 import binding as B
    from paper_2508_15706_b200 import inner

    def refused(status, *a, **k):
        with pytest.raises(B.SlError) as e:
            inner.token_loss(*a, **k)
        assert e.value.status == status

    x, t = make(4, 32, torch.float32, 3)
    refused(B.SL_ERR_INVALID_ARG, x, t[:3])
    refused(B.SL_ERR_INVALID_ARG, x, t.float())
    refused(B.SL_ERR_INVALID_ARG, x.half(), t)
    refused(B.SL_ERR_INVALID_ARG, x, t, smoothing=1.5)
    refused(B.SL_ERR_INVALID_ARG, x, t, z=float("nan"))
    refused(B.SL_ERR_INVALID_ARG, x, t, grad=x[:, :31].contiguous())
    refused(B.SL_ERR_INVALID_ARG, x.t().contiguous().t(), t)
    refused(B.SL_ERR_NOMEM, x, t, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
