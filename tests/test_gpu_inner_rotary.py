"""Rotary positions (sl_rotary_*) against complex rotations in 64 bits.

Tolerances: sine and cosine are good to 2^-23 (an angle reduced exactly, then rounded to a float fraction of a half turn: pi 2^-25),
two products and a sum add 3 u: 2^-21 of |a| + |b|; a bfloat16 result is the rounding of such a number."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def freqs(rot, base, scaling, factor, length, low, high):
    n = rot // 2
    f = [base ** (-2.0 * i / rot) for i in range(n)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "base":
        b = base * factor ** (rot / (rot - 2.0))
        f = [b ** (-2.0 * i / rot) for i in range(n)]
    if scaling == "by_parts":
        k = [min(1.0, max(0.0, (length * x / (2 * math.pi) - low) / (high - low))) for x in f]
        f = [x * a + x / factor * (1 - a) for x, a in zip(f, k)]
    return torch.tensor(f, dtype=torch.float64, device="cuda")


def turned(x, pos, f, rot, layout, mag, inverse):
    """x [B, S, H, D] fp64, pos [B, S] int64."""
    t = torch.polar(torch.full((1,), mag, dtype=torch.float64, device="cuda"), (pos[:, :, None, None].double() * f) * (-1.0 if inverse else 1.0))
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if layout == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    z = torch.complex(a.contiguous(), b.contiguous()) * t
    out, size = x.clone(), torch.zeros_like(x)
    both = (a.abs() + b.abs()) * mag
    if layout == "half":
        out[..., :rot // 2], out[..., rot // 2:rot] = z.real, z.imag
        size[..., :rot // 2], size[..., rot // 2:rot] = both, both
    else:
        out[..., 0:rot:2], out[..., 1:rot:2] = z.real, z.imag
        size[..., 0:rot:2], size[..., 1:rot:2] = both, both
    return out, size


def inside(got, want, tol, what=""):
    """got is want up to tol; stored in bfloat16, the rounding of some number up to tol from want (rounding keeps order)."""
    low, high = (want - tol).to(got.dtype), (want + tol).to(got.dtype)
    bad = ~((got >= low) & (got <= high))
    assert not torch.any(bad), (what, (got.double() - want)[bad][:4], want[bad][:4])


def close(got, want, size):
    inside(got, want, 2.0 ** -21 * size)


SHAPES = [  # batch, seq, q heads, k heads, head_dim, rot
    (1, 1, 1, 1, 2, 2), (2, 7, 3, 1, 64, 64), (1, 33, 4, 2, 80, 32), (3, 5, 2, 2, 128, 50), (2, 40, 16, 16, 128, 128), (70, 1, 8, 2, 96, 96), (1, 900, 5, 1, 100, 20), (1, 5000, 2, 1, 64, 24),
    (1, 3, 1, 1, 7, 6), (1, 2, 2, 2, 1024, 1024)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("inverse", [False, True])
def test_against_complex_rotation(shape, layout, act, inverse):
    """Heads taken out of one packed product (so token and head strides differ), contiguous outputs, and in place."""
    from paper_2508_15706_b200.inner import Rotary
    B, S, hq, hk, D, rot = shape
    g = torch.Generator(device="cuda").manual_seed(B * 100 + S)
    qkv = torch.randn(B, S, hq + 2 * hk, D, generator=g, device="cuda").to(act)
    q, k = qkv[:, :, :hq], qkv[:, :, hq:hq + hk]
    pos = torch.randint(0, 100000, (B, S), generator=g, device="cuda")
    rope = Rotary(rot, base=10000.0, layout=layout, magnitude=1.25)
    f = freqs(rot, 10000.0, "none", 1, 0, 0, 0)
    oq, ok = torch.full((B, S, hq, D), 5.0, dtype=act, device="cuda"), torch.full((B, S, hk, D), 5.0, dtype=act, device="cuda")
    rope.apply(q, k, pos, inverse=inverse, out_q=oq, out_k=ok)
    for got, x in ((oq, q), (ok, k)):
        close(got, *turned(x.double(), pos, f, rot, layout, 1.25, inverse))
        assert torch.equal(got[..., rot:], x[..., rot:])
    v = qkv[:, :, hq + hk:].clone()
    rope.apply(q, k, pos.int(), inverse=inverse)  # in place, 32-bit positions
    assert torch.equal(q, oq) and torch.equal(k, ok) and torch.equal(qkv[:, :, hq + hk:], v)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_strides_orders_and_positions(layout):
    """[batch, heads, seq, dim] order, a shift that breaks 16-byte alignment, one row of positions shared by the batch, no
    positions, q alone, negative positions."""
    from paper_2508_15706_b200.inner import Rotary
    rope = Rotary(32, layout=layout)
    f = freqs(32, 10000.0, "none", 1, 0, 0, 0)
    for act in (torch.float32, torch.bfloat16):
        for shift in (0, 1, 2, 4):
            buf = torch.randn(2 * 3 * 50 * 48 + 8, device="cuda").to(act)
            q = buf[shift:shift + 2 * 3 * 50 * 48].view(2, 3, 50, 48).transpose(1, 2)
            before = q.clone()
            pos = torch.arange(50, device="cuda") * 3 - 70
            rope.apply(q, None, pos)
            close(q, *turned(before.double(), pos.expand(2, 50), f, 32, layout, 1.0, False))
            again = before.clone()
            rope.apply(again, None, None, first=11)
            close(again, *turned(before.double(), (torch.arange(50, device="cuda") + 11).expand(2, 50), f, 32, layout, 1.0, False))
            strided = torch.stack([pos, pos * 0], 1)[:, 0]  # stride 2
            again = before.clone()
            rope.apply(again, None, strided)
            assert torch.equal(again, q)


@pytest.mark.parametrize("head_dim,rot,stride", [(70, 64, 72), (66, 64, 80), (72, 64, 72), (100, 24, 104), (128, 50, 128), (51, 34, 64), (96, 38, 96)])
@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rest_of_the_head_of_any_width(head_dim, rot, stride, act, layout):
    """The part that turns and the part that is passed through divide into accesses of different widths; padded heads."""
    from paper_2508_15706_b200.inner import Rotary
    x = torch.randn(2, 9, 3, stride, device="cuda").to(act)
    q = x[..., :head_dim]
    out = torch.full((2, 9, 3, stride), 5.0, dtype=act, device="cuda")
    Rotary(rot, layout=layout).apply(q, None, None, first=3, out_q=out[..., :head_dim])
    pos = (torch.arange(9, device="cuda") + 3).expand(2, 9)
    close(out[..., :head_dim], *turned(q.double(), pos, freqs(rot, 10000.0, "none", 1, 0, 0, 0), rot, layout, 1.0, False))
    assert torch.equal(out[..., rot:head_dim], q[..., rot:]) and torch.all(out[..., head_dim:] == 5.0)


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "by_parts"])
@pytest.mark.parametrize("rot", [4, 64, 128])
def test_scalings_and_far_positions(scaling, rot):
    """Angles of millions of radians: the 64-bit phase keeps them.  (The reference's own angle, position x frequency in fp64, is good
    to 2^-53 x angle = 1e-9 at 2^23 radians.)"""
    from paper_2508_15706_b200.inner import Rotary
    rope = Rotary(rot, base=500000.0, scaling=scaling, factor=8.0, original_length=8192, low_turns=1.0, high_turns=32.0)
    f = freqs(rot, 500000.0, scaling, 8.0, 8192, 1.0, 32.0)
    q = torch.randn(1, 64, 2, rot, device="cuda")
    pos = (8 * 1024 * 1024 - torch.arange(64, device="cuda") * 131071).view(1, 64)
    out = torch.empty_like(q)
    rope.apply(q, None, pos, out_q=out)
    close(out, *turned(q.double(), pos, f, rot, "half", 1.0, False))


def test_inverse_is_the_gradient():
    """The operator is linear: <turn(x), w> = <x, inverse(w)> is the gradient test, and differences are exact up to rounding."""
    from paper_2508_15706_b200 import inner
    for layout in ("half", "interleaved"):
        rope = inner.Rotary(48, layout=layout, magnitude=0.75)
        pos = torch.randint(0, 5000, (2, 31), device="cuda")
        q = torch.randn(2, 31, 4, 64, device="cuda", requires_grad=True)
        k = torch.randn(2, 31, 2, 64, device="cuda", requires_grad=True)
        wq, wk = torch.randn(2, 31, 4, 64, device="cuda"), torch.randn(2, 31, 2, 64, device="cuda")
        oq, ok = inner.rotary(rope, q, k, pos)
        ((oq * wq).sum() + (ok * wk).sum()).backward()
        f = freqs(48, 10000.0, "none", 1, 0, 0, 0)
        for x, w in ((q, wq), (k, wk)):
            close(x.grad, *turned(w.double(), pos, f, 48, layout, 0.75, True))
            d = torch.randn_like(x, dtype=torch.float64)
            up, _ = turned(x.detach().double() + d, pos, f, 48, layout, 0.75, False)
            down, _ = turned(x.detach().double() - d, pos, f, 48, layout, 0.75, False)
            slope = ((up - down) * w.double()).sum().item() / 2
            got = (x.grad.double() * d).sum().item()
            assert abs(got - slope) <= 2.0 ** -20 * (x.grad.double() * d).abs().sum().item()


def test_empty_and_refusals():
    from paper_2508_15706_b200 import binding as B
    from paper_2508_15706_b200.inner import Rotary
    rope = Rotary(8)
    rope.apply(torch.empty(0, 4, 2, 8, device="cuda"))
    rope.apply(torch.empty(2, 0, 2, 8, device="cuda"))

    def refused(status, fn, *a, **k):
        with pytest.raises(B.SlError) as e:
            fn(*a, **k)
        assert e.value.status == status

    q = torch.zeros(2, 4, 2, 8, device="cuda")
    for bad in (3, 0, 2048):
        refused(B.SL_ERR_INVALID_ARG, Rotary, bad)
    refused(B.SL_ERR_INVALID_ARG, Rotary, 8, base=0.5)
    refused(B.SL_ERR_INVALID_ARG, Rotary, 8, scaling="linear", factor=0.5)
    refused(B.SL_ERR_INVALID_ARG, Rotary, 8, scaling="by_parts", factor=2.0, original_length=4096, low_turns=8.0, high_turns=8.0)
    refused(B.SL_ERR_INVALID_ARG, Rotary, 8, layout="other")
    refused(B.SL_ERR_INVALID_ARG, Rotary(16).apply, q)
    refused(B.SL_ERR_INVALID_ARG, rope.apply, q[0])
    refused(B.SL_ERR_INVALID_ARG, rope.apply, q.half())
    refused(B.SL_ERR_INVALID_ARG, rope.apply, q, q[:, :2])
    refused(B.SL_ERR_INVALID_ARG, rope.apply, q, None, torch.zeros(3, dtype=torch.int64, device="cuda"))
    refused(B.SL_ERR_INVALID_ARG, rope.apply, q, None, torch.zeros(4, device="cuda"))
    refused(B.SL_ERR_INVALID_ARG, rope.apply, q.transpose(2, 3).contiguous().transpose(2, 3))
