"""Next-token loss where logits are large numbers: masks by a finite constant (-1e9, -1e10, -1e20, the type's lowest value) over whole
threads' worth of logits, rows of nothing but such a constant, maxima on both sides of 2^30.

Tolerances (u = 2^-24), against the formula in 64 bits: exponentials and the sum of a row are good to r = 2^-17 relative (as in
test_gpu_inner_loss.py) and to the rounding of log2 e in their exponent, |x - max| u; two numbers that differ at 2^30 are 64 and more
apart, so 2^-64 may stand for e^-64: 1e-19 absolute.  lse and the loss add 8 u of the maximum's size (a loss is a difference of two
numbers of that size)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BASES = [3e8, 1e9, 1.2e9, 1.5e9, 3e9, 1e10, 1e12, 1e20, 6.8e29, 8e29, 9.9e29, 1e30, 1.2e30, 1.5e30, 1e38, 3.3e38]


def rows_for(b, V, act, g):
    """Rows around the number b (of either sign), with their targets."""
    big = torch.tensor(b, dtype=torch.float64).to(act).item()
    near = torch.tensor(b, dtype=torch.float64).to(act)
    near = torch.nextafter(near, torch.zeros_like(near)).item()  # the next one towards 0
    usual = 3.0 * torch.randn(V, generator=g, device="cuda")
    half = torch.arange(V, device="cuda") < V // 2
    full = lambda x: torch.full((V,), x, device="cuda", dtype=torch.float64)  # noqa: E731
    rows = [full(big), torch.where(half, full(big), full(near)), torch.where(half, full(near), full(big)), torch.where(half, full(big), usual.double()),
            torch.where(half, usual.double(), full(big)), torch.where(half, full(big), full(big / 4)), torch.where(half, full(0.9 * big), full(1.1 * big) if abs(1.1 * b) < 3.38e38 else full(big))]
    alone = full(near)
    alone[V // 3] = big
    rows.append(alone)
    x = torch.stack(rows).to(act)
    t = torch.randint(0, V, (len(rows),), generator=g, device="cuda")
    return x, t


@pytest.mark.parametrize("V,shift", [(512, 0), (4097, 0), (32000, 0), (1000, 1), (300001, 0)])
@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("many", [False, True])
def test_against_the_formula(V, shift, act, sign, many):
    from paper_2508_15706_b200 import inner
    if many and V > 5000:
        pytest.skip("enough rows for a CTA each are tested at the narrow sizes")
    g = torch.Generator(device="cuda").manual_seed(V)
    for b in BASES + [torch.finfo(act).max]:
        x, t = rows_for(sign * b, V, act, g)
        if many:
            x, t = x.repeat(100, 1), t.repeat(100)
        rows = x.shape[0]
        buf = torch.full((rows * V + 8,), 9.0, dtype=act, device="cuda")
        grad = buf[shift:shift + rows * V].view(rows, V)  # elsewhere relative to 16 bytes with a shift
        _, loss, lse = inner.token_loss(x, t, grad=grad, mean=False)
        x64 = x.double()
        top = x64.amax(1)
        ws = torch.logsumexp(x64, 1)
        wl = -torch.log_softmax(x64, 1).gather(1, t[:, None])[:, 0]
        p = torch.softmax(x64, 1)  # (relative to the maximum: x - lse loses log V at these sizes, in 64 bits too)
        hit = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
        tol = 2.0 ** -17 + 8 * U * torch.maximum(top.abs(), ws.abs()) + 2.0 ** -17 * wl.abs().clamp(max=1e30)
        assert torch.all((lse.double() - ws).abs() <= tol), (b, lse, ws)
        fits = wl <= torch.finfo(torch.float32).max
        bad = fits & ~((loss.double() - wl).abs() <= tol + 4 * U * wl.abs())
        assert not torch.any(bad), (b, loss[bad][:4], wl[bad][:4])
        rel = 2.0 ** -17 + 4 * U * (top[:, None] - x64).clamp(max=200.0)
        size = 2 * rel * (p + hit) + 1e-19
        want = p - hit
        low, high = (want - size).to(act), (want + size).to(act)
        assert torch.all((grad >= low) & (grad <= high)), (b, act)


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -1e15, -1e20, -1e30, "lowest"])
@pytest.mark.parametrize("rows,V", [(300, 4096), (3, 32000), (400, 32000)])
def test_a_finite_mask_is_a_mask(act, mask, rows, V):
    """Entries masked by a large finite constant take nothing: the rest of the row is as with -inf, up to the order of the sums."""
    from paper_2508_15706_b200 import inner
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (3.0 * torch.randn(rows, V, generator=g, device="cuda")).to(act)
    t = torch.randint(0, V // 4, (rows,), generator=g, device="cuda")
    out = []
    for m in (float("-inf"), torch.finfo(act).min if mask == "lowest" else mask):
        x[:, V // 4:] = m
        grad = torch.full_like(x, 9.0)
        _, loss, lse = inner.token_loss(x, t, grad=grad, z=1e-4)
        out.append((loss, lse, grad))
    for a, b in zip(*out):
        assert torch.equal(a, b)
    assert torch.all(out[1][2][:, V // 4:] == 0)
