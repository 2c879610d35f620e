"""Element offsets beyond 32 bits: the last rows of matrices of more than 2^31 elements, a tensor behind element 2^32 of the flat
buffers.  A few rows are compared with the formulas in 64 bits; tolerances as in the operators' own tests."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def test_adamw_behind_two_to_the_32():
    from paper_2508_15706_b200.inner import AdamW
    off, n = (1 << 32) + 4, 1000
    opt = AdamW([(1, n)], [off], weight_decay=0.0, state_bits=8, max_norm=0.0, param_dtype=torch.bfloat16, grad_dtype=torch.bfloat16)
    total = opt.flat_elems
    theta = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    grad = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    m, v, scales = opt.new_state()
    g = torch.Generator(device="cuda").manual_seed(3)
    grad[off:] = (torch.randn(n, generator=g, device="cuda") * 1e-2).bfloat16()
    m32, v32 = torch.zeros(total, device="cuda"), torch.zeros(total, device="cuda")
    opt.step(theta, grad, m, v, scales, step=1, lr=1e-2, seed=7)
    opt.read_state(m, v, scales, m32, v32)
    gr = grad[off:].double()
    assert torch.all((m32[off:].double() - 0.1 * gr).abs() <= (0.1 * gr).abs() / 16 + (0.1 * gr).abs().max() * 2.0 ** -17)
    want = 0.05 * gr.square()
    # a quarter of a binade's sixteenth either way, never below the smallest code of the block
    assert torch.all(((v32[off:].double() - want).abs() <= want / 16) | (want < want.max() * 2.0 ** -14))
    assert torch.all((theta[off:].double() + 1e-2 * gr.sign()).abs() <= 1e-2 * 2.0 ** -7)
    # the hash sees the offset's upper half
    f = np.float32
    gs = grad[off:].float().cpu().numpy()
    vv = (gs * gs) * f(1 - 0.95)

    def mix(x):
        x ^= x >> 16
        x = x * 0x7FEB352D & 0xFFFFFFFF
        x ^= x >> 15
        x = x * 0x846CA68B & 0xFFFFFFFF
        return x ^ (x >> 16)

    key = mix(7) ^ mix(1 * 0x9E3779B9 & 0xFFFFFFFF)
    ev = scales[1].cpu().numpy().astype(np.int64)
    x = vv * np.exp2(127.0 - ev)[np.arange(n) // 128].astype(f)
    lot = np.array([mix(((off + i) & 0xFFFFFFFF) ^ key) >> 13 for i in range(n)], dtype=np.int64)
    code = np.clip(((x.view(np.uint32).astype(np.int64) + lot) >> 19) - 1792, 1, 255)
    assert np.array_equal(v[off:].cpu().numpy(), np.where(x == 0, 0, code).astype(np.uint8))


def test_norms_beyond_two_to_the_31():
    from paper_2508_15706_b200 import inner
    rows, cols = (1 << 31) // 2048 + 500, 2048
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    b = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.rand(cols, device="cuda") + 0.5
    y, h, r, br = inner.norm_forward(x, w, branch=b, branch_weight=w, alpha=0.5)
    at = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda")
    xs, bs = x[at].double(), b[at].double()
    z = bs * (bs.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w.double()
    ys = xs + 0.5 * z
    hs = ys * (ys.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w.double()
    for got, want in ((y[at], ys), (h[at], hs)):
        tol = 2.0 ** -19 * (want.abs() + xs.abs() + z.abs())
        assert torch.all((got >= (want - tol).bfloat16()) & (got <= (want + tol).bfloat16()))
    # backward in place: dx over dy
    dy, dh = x, b  # (their values serve as gradients)
    dys, dhs = dy[at].double(), dh[at].double()
    inner.norm_backward(dy, dh, y, w, rstd=r, dx=dy)
    yh, u = y[at].double() * r[at].double()[:, None], dhs * w.double()
    want = dys + r[at].double()[:, None] * (u - yh * (u * yh).mean(1, keepdim=True))
    tol = 2.0 ** -19 * (dys.abs() + u.abs() + (yh * (u * yh).abs().mean(1, keepdim=True)).abs()) * 4
    assert torch.all((dy[at] >= (want - tol).bfloat16()) & (dy[at] <= (want + tol).bfloat16()))


def test_loss_beyond_two_to_the_31():
    from paper_2508_15706_b200 import inner
    for V in (32000, 32003):
        rows = (1 << 31) // V + 100
        x = torch.empty(rows, V, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(2))
        t = torch.randint(0, V, (rows,), device="cuda")
        at = torch.tensor([0, rows // 2, rows - 1], device="cuda")
        xs = x[at].double()
        total, loss, lse = inner.token_loss(x, t, grad=x, mean=False)
        want = torch.logsumexp(xs, 1)
        assert torch.all((lse[at].double() - want).abs() <= 2.0 ** -17 + 2.0 ** -20)
        grad = torch.exp(xs - want[:, None])
        grad[torch.arange(3), t[at]] -= 1.0
        tol = 2.0 ** -16 * (grad.abs() + 2.0 ** -20)
        assert torch.all((x[at] >= (grad - tol).bfloat16()) & (x[at] <= (grad + tol).bfloat16()))
        assert abs(total.item() - loss.double().sum().item()) <= 1e-6 * abs(total.item())
        del x


def test_rotary_beyond_two_to_the_31():
    from paper_2508_15706_b200.inner import Rotary
    S, H, D = 4096, 8, 64
    B = (1 << 31) // (S * H * D) + 1
    q = torch.empty(B, S, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(5))
    before = q[-1, -1].double()
    Rotary(D).apply(q)
    a = (S - 1) * 10000.0 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device="cuda") / D)
    u, w = before[:, :D // 2], before[:, D // 2:]
    want = torch.cat([u * a.cos() - w * a.sin(), w * a.cos() + u * a.sin()], -1)
    tol = 2.0 ** -21 * torch.cat([u.abs() + w.abs()] * 2, -1)
    assert torch.all((q[-1, -1] >= (want - tol).bfloat16()) & (q[-1, -1] <= (want + tol).bfloat16()))
