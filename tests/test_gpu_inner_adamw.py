"""AdamW over a tensor table (sl_adamw_*) against the formula in 64 bits, moments in 32 and in 8 bits.

Tolerances, from the arithmetic (u = 2^-24, one fp32 rounding): each moment is a sum of two products, at most four roundings
of its terms: 4 u (|beta m| + |(1 - beta) g'|), twice that for v's square.  The update divides by a denominator that is good to a few
u, with fast instructions (2^-22): 2^-19 of the update's size is ample.  bfloat16 parameters add half a unit, at most 2^-8 |theta|."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 3), (7, 5), (64, 64), (1, 4097), (33, 130), (1, 8192), (3, 1)]
U = 2.0 ** -24


def layout(align, gap):
    offs, at = [], gap
    for r, c in SHAPES:
        at = (at + align - 1) // align * align
        offs.append(at)
        at += r * c + gap
    return offs, at


def elements(offs):
    return torch.cat([torch.arange(o, o + r * c) for (r, c), o in zip(SHAPES, offs)]).cuda()


def inputs(n, seed, grad_dtype, param_dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda s: torch.randn(n, generator=g, device="cuda") * s  # noqa: E731
    return (rand(0.5).to(param_dtype), (rand(1e-2) * torch.exp(rand(1.0))).to(grad_dtype))


def reference(p, g, m, v, decay, t, lr, betas, eps, max_norm, grad_scale):
    """The formula in fp64.  Returns theta, m, v, norm and the sizes the tolerances go by."""
    p, g, m, v = (x.double() for x in (p, g, m, v))
    norm = abs(grad_scale) * g.square().sum().sqrt()
    c = grad_scale * (min(1.0, max_norm / (norm.item() + 1e-6)) if max_norm else 1.0)
    g = c * g
    tm = betas[0] * m.abs() + (1 - betas[0]) * g.abs()
    tv = betas[1] * v + (1 - betas[1]) * g * g
    m = betas[0] * m + (1 - betas[0]) * g
    den = (tv / (1 - betas[1] ** t)).sqrt() + eps
    ss = lr / (1 - betas[0] ** t)
    return p - p * (lr * decay) - ss * m / den, m, tv, norm, tm, ss * tm / den


@pytest.mark.parametrize("align,gap", [(4, 5), (8, 0), (128, 3)])
@pytest.mark.parametrize("param_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm,grad_scale", [(0.0, 1.0), (0.3, 0.25), (1e6, 2.0)])
def test_steps_with_32_bit_moments(align, gap, param_dtype, grad_dtype, max_norm, grad_scale):
    from paper_2508_15706_b200.inner import AdamW
    offs, n = layout(align, gap)
    at = elements(offs)
    wd = [0.1 * (j % 3) for j in range(len(SHAPES))]
    decay = torch.cat([torch.full((r * c,), w, dtype=torch.float64) for (r, c), w in zip(SHAPES, wd)]).cuda()
    opt = AdamW(SHAPES, offs, weight_decay=wd, betas=(0.9, 0.95), eps=1e-8, max_norm=max_norm, param_dtype=param_dtype, grad_dtype=grad_dtype)
    assert opt.flat_elems == int(at.max()) + 1
    theta, _ = inputs(n, 1, grad_dtype, param_dtype)
    m, v, norm = torch.full((n,), 3.0, device="cuda"), torch.full((n,), 5.0, device="cuda"), torch.zeros(1, device="cuda")
    m[at], v[at] = 0.0, 0.0
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    outside[at] = False
    copy = torch.full((n,), 7.0, dtype=torch.bfloat16, device="cuda") if param_dtype == torch.float32 else None
    before = theta[outside].clone()
    for t in range(1, 4):
        grad = inputs(n, 10 + t, grad_dtype, param_dtype)[1]
        want, wm, wv, wn, tm, upd = reference(theta[at], grad[at], m[at], v[at], decay, t, 3e-2, (0.9, 0.95), 1e-8, max_norm, grad_scale)
        opt.step(theta, grad, m, v, step=t, lr=3e-2, grad_scale=grad_scale, copy=copy, norm=norm)
        assert abs(norm.item() - wn.item()) <= 2 * U * wn.item()
        assert torch.all((m[at].double() - wm).abs() <= 5 * U * tm + 1e-44)
        assert torch.all((v[at].double() - wv).abs() <= 8 * U * wv + 1e-44)
        tol = 4 * U * want.abs() + 2.0 ** -19 * upd + (2.0 ** -8 * want.abs() if param_dtype == torch.bfloat16 else 0.0)
        assert torch.all((theta[at].double() - want).abs() <= tol)
        if copy is not None:
            assert torch.equal(copy[at], theta[at].bfloat16()) and torch.all(copy[outside] == 7.0)
    assert torch.equal(theta[outside], before) and torch.all(m[outside] == 3.0) and torch.all(v[outside] == 5.0)


# ---- 8-bit moments: the code format restated in numpy
def e4m3_values():
    c = np.arange(256)
    s, e, f = np.where(c >= 128, -1.0, 1.0), (c % 128) // 8, c % 8
    val = s * np.where(e == 0, f * 2.0 ** -9, np.exp2(e - 7.0) * (1 + f / 8.0))
    val[(c % 128) == 127] = np.nan
    return val


def v_values():
    c = np.arange(256)
    return np.where(c == 0, 0.0, np.exp2(c // 16 - 15.0) * (1 + c % 16 / 16.0))


def mix(x):
    x = x ^ (x >> 16)
    x = x * 0x7FEB352D & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = x * 0x846CA68B & 0xFFFFFFFF
    return x ^ (x >> 16)


def check_codes(offs, m, v, m8, v8, scales, seed, exact=True):
    """m, v: what the codes should stand for (fp64).  m within half a step of its code's neighbours; v one of the two codes
    around it, and the very one that the hash chooses unless v is within 2^-20 of the place where the choice turns."""
    m8, v8, scales = m8.cpu().numpy(), v8.cpu().numpy(), scales.cpu().numpy().astype(np.float64)
    vm, vv = e4m3_values(), v_values()
    block = 0
    for (r, c), off in zip(SHAPES, offs):
        n = r * c
        for b in range(0, n, 128):
            s = slice(off + b, off + min(n, b + 128))
            sm, sv = 2.0 ** (scales[0, block] - 127), 2.0 ** (scales[1, block] - 127)
            top_m, top_v = np.abs(m[s]).max(), v[s].max()
            if top_m > 2.0 ** -110:
                assert top_m / sm <= 448 * (1 + 1e-6) and top_m / sm > 224 * (1 - 1e-6)
            if top_v > 2.0 ** -120:
                assert 31 / 32 * (1 - 1e-6) <= top_v / sv <= 31 / 16 * (1 + 1e-6)
            x = m[s] / sm
            step = np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
            assert np.all(np.abs(vm[m8[s]] - x) <= step * (0.5 + 1e-5))
            x = v[s] / sv
            code = v8[s].astype(np.int64)
            assert np.all((code == 0) == (x == 0))
            e = np.floor(np.log2(np.where(x > 0, x, 1.0)))
            place = np.where(x > 0, 16 * (e + 15) + 16 * (x / np.exp2(e) - 1), 0.0)
            idx = np.arange(s.start, s.stop, dtype=np.int64)
            lot = (np.array([mix(int(i) ^ mix(seed)) for i in idx]) >> 13) / 2.0 ** 19
            want = np.clip(np.floor(place + lot), 1, 255)
            sure = np.abs(place + lot - np.round(place + lot)) > 1e-5
            assert np.all((code == want) | ~sure | (x == 0))
            assert np.all((np.abs(code - want) <= 1) | (x == 0))
            block += 1


@pytest.mark.parametrize("align,gap", [(4, 3), (8, 0), (128, 5)])
@pytest.mark.parametrize("param_dtype,grad_dtype", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_steps_with_8_bit_moments(align, gap, param_dtype, grad_dtype):
    from paper_2508_15706_b200.inner import AdamW
    offs, n = layout(align, gap)
    at = elements(offs)
    opt = AdamW(SHAPES, offs, weight_decay=0.1, max_norm=0.5, state_bits=8, param_dtype=param_dtype, grad_dtype=grad_dtype)
    theta, _ = inputs(n, 2, grad_dtype, param_dtype)
    m8, v8, scales = opt.new_state()
    m8, v8 = (torch.cat([x, torch.zeros(n - x.numel(), dtype=x.dtype, device="cuda")]) for x in (m8, v8))
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    outside[at] = False
    m8[outside], v8[outside] = 0x55, 0xAA
    m32, v32 = torch.full((n,), 11.0, device="cuda"), torch.full((n,), 12.0, device="cuda")
    for t in range(1, 5):
        grad = inputs(n, 20 + t, grad_dtype, param_dtype)[1]
        opt.read_state(m8, v8, scales, m32, v32)
        assert torch.all(m32[outside] == 11.0) and torch.all(v32[outside] == 12.0)
        want, wm, wv, _, tm, upd = reference(theta[at], grad[at], m32[at], v32[at], 0.1, t, 1e-2, (0.9, 0.95), 1e-8, 0.5, 1.0)
        opt.step(theta, grad, m8, v8, scales, step=t, lr=1e-2, seed=77 + t)
        tol = 4 * U * want.abs() + 2.0 ** -19 * upd + (2.0 ** -8 * want.abs() if param_dtype == torch.bfloat16 else 0.0)
        assert torch.all((theta[at].double() - want).abs() <= tol)
        full_m, full_v = np.zeros(n), np.zeros(n)
        full_m[at.cpu().numpy()], full_v[at.cpu().numpy()] = wm.cpu().numpy(), wv.cpu().numpy()
        check_codes(offs, full_m, full_v, m8, v8, scales, 77 + t)
    assert torch.all(m8[outside] == 0x55) and torch.all(v8[outside] == 0xAA)


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [0.0, 0.05])
def test_8_bit_codes_bit_for_bit(grad_dtype, max_norm):
    """A million elements against the formula in fp32, each operation rounded once, in the order the header gives them: codes and
    scales equal, the norm the rounded fp64 sum."""
    from paper_2508_15706_b200.inner import AdamW
    n = 1 << 20
    opt = AdamW([(1024, 1024)], state_bits=8, max_norm=max_norm, grad_dtype=grad_dtype)
    g = torch.Generator(device="cuda").manual_seed(31)
    theta = torch.randn(n, generator=g, device="cuda")
    state, norm = opt.new_state(), torch.zeros(1, device="cuda")
    m32, v32 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    f = np.float32
    for t in range(1, 4):
        grad = (torch.randn(n, generator=g, device="cuda") * torch.exp(torch.randn(n, generator=g, device="cuda")) * 1e-3).to(grad_dtype)
        opt.read_state(*state, m32, v32)
        m0, v0, gr = m32.cpu().numpy(), v32.cpu().numpy(), grad.float().cpu().numpy()
        opt.step(theta, grad, *state, step=t, lr=1e-3, seed=t, norm=norm)
        size = math.sqrt(np.sum(gr.astype(np.float64) ** 2))
        assert norm.item() == f(size)
        gs = gr * f(min(1.0, max_norm / (size + 1e-6)) if max_norm else 1.0)
        m = m0 * f(0.9) + gs * f(1 - 0.9)
        v = v0 * f(0.95) + (gs * gs) * f(1 - 0.95)
        top_m = np.abs(m).reshape(-1, 128).max(1).view(np.uint32)
        top_v = v.reshape(-1, 128).max(1).view(np.uint32)
        em = np.maximum((top_m >> 23).astype(np.int64) + ((top_m & 0x7FFFFF) > 0x600000) - 8, 1)
        ev = np.clip((top_v >> 23).astype(np.int64) + ((top_v & 0x7FFFFF) > 0x780000), 1, 254)
        assert np.array_equal(state[2].cpu().numpy(), np.stack([em, ev]).astype(np.uint8))
        scaled = torch.from_numpy((m.reshape(-1, 128) * np.exp2(127.0 - em)[:, None].astype(f)).reshape(-1))
        assert torch.equal(state[0].cpu(), scaled.to(torch.float8_e4m3fn).view(torch.uint8))
        x = (v.reshape(-1, 128) * np.exp2(127.0 - ev)[:, None].astype(f)).reshape(-1)
        i = np.arange(n, dtype=np.uint64) ^ np.uint64(mix(t))
        lot = i ^ (i >> np.uint64(16))
        lot = lot * np.uint64(0x7FEB352D) & np.uint64(0xFFFFFFFF)
        lot ^= lot >> np.uint64(15)
        lot = lot * np.uint64(0x846CA68B) & np.uint64(0xFFFFFFFF)
        lot = ((lot ^ (lot >> np.uint64(16))) >> np.uint64(13)).astype(np.int64)
        code = np.clip(((x.view(np.uint32).astype(np.int64) + lot) >> 19) - 1792, 1, 255)
        assert np.array_equal(state[1].cpu().numpy(), np.where(x == 0, 0, code).astype(np.uint8))


@pytest.mark.parametrize("scale", [1e-30, 1e-15, 1.0, 1e15, 1e25])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
def test_norm_over_the_whole_range(scale, grad_dtype):
    """Zeros, tiny and huge gradients beside each other: the fp64 sum of exact squares, rounded once."""
    from paper_2508_15706_b200.inner import AdamW
    n = 70001
    opt = AdamW([(1, n)], max_norm=1.0, grad_dtype=grad_dtype)
    g = torch.Generator(device="cuda").manual_seed(8)
    norm, theta = torch.zeros(1, device="cuda"), torch.zeros(n, device="cuda")
    for mixed in (False, True):
        grad = torch.randn(n, generator=g, device="cuda") * scale
        if mixed:
            grad[::3] = 0.0
            grad[1::3] *= 1e-9
        grad = grad.to(grad_dtype)
        opt.step(theta, grad, *opt.new_state()[:2], step=1, lr=0.0, norm=norm)
        want = grad.double().square().sum().sqrt().item()
        assert norm.item() == np.float32(want)
    opt.step(theta, torch.zeros_like(grad), *opt.new_state()[:2], step=1, lr=0.0, norm=norm)
    assert norm.item() == 0.0


def test_8_bit_state_round_trip_and_ranges():
    """Blocks of zeros, denormals, huge values, one outlier, infinities and NaN; a state that was read back keeps its values
    when it is written again (they are code points: nothing to round)."""
    from paper_2508_15706_b200.inner import AdamW
    offs, n = layout(4, 0)
    opt = AdamW(SHAPES, offs, state_bits=8)
    g = torch.Generator(device="cuda").manual_seed(5)
    m = torch.randn(n, generator=g, device="cuda")
    v = torch.rand(n, generator=g, device="cuda")
    o = offs[4]  # the 4097-element vector: 33 blocks
    m[o:o + 128] = 0.0
    v[o:o + 128] = 0.0
    m[o + 128:o + 256] *= 1e-41
    v[o + 128:o + 256] *= 1e-41
    m[o + 256:o + 384] *= 1e37
    v[o + 256:o + 384] = 3e38
    m[o + 384], v[o + 384] = 1e6, 1e12
    m8, v8, s = opt.new_state()
    opt.write_state(m, v, m8, v8, s, seed=3)
    fm, fv = m.double().cpu().numpy(), v.double().cpu().numpy()
    fv[o + 256:o + 384] = np.minimum(fv[o + 256:o + 384], 2.0 ** 127 * 1.9375)
    keep = np.ones(n, dtype=bool)
    keep[o + 128:o + 256] = False
    m_out, v_out = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    opt.read_state(m8, v8, s, m_out, v_out)
    at = elements(offs)
    # below the smallest scale (2^-126) the grid of m ends at 2^-135, that of v at its smallest code
    tiny = slice(o + 128, o + 256)
    assert torch.all((m_out[tiny] - m[tiny]).abs() <= 2.0 ** -135) and torch.all(v_out[tiny][v[tiny] > 0] > 0)
    assert torch.all(m_out[o:o + 128] == 0) and torch.all(v_out[o:o + 128] == 0)
    assert torch.all((v_out[o + 256:o + 384] / 3e38 - 1).abs() < 1 / 16)
    ok = torch.ones(n, dtype=torch.bool, device="cuda")
    ok[tiny] = False
    ok[o + 384:o + 512] = False  # under the outlier's scale
    ok = ok[at]
    assert torch.all(((m_out - m)[at].abs() <= m[at].abs() / 16 + 1e-3 * 4)[ok])
    assert torch.all(((v_out - v)[at].abs() <= v[at] / 16 + 2.0 ** -15)[ok])
    assert m_out[o + 384] / 1e6 - 1 < 1 / 16 and torch.all(v_out[o + 385:o + 512] > 0)
    again, m_two, v_two = opt.new_state(), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    opt.write_state(m_out, v_out, *again, seed=99)
    opt.read_state(*again, m_two, v_two)
    assert torch.equal(m_two[at], m_out[at]) and torch.equal(v_two[at], v_out[at])
    # non-finite values: m becomes NaN, v the largest code; the block's other elements keep their scale
    m[o + 600], m[o + 601], v[o + 602], v[o + 603] = float("inf"), float("nan"), float("inf"), float("nan")
    ref = [x.clone() for x in (m8, v8, s)]
    opt.write_state(m, v, m8, v8, s, seed=3)
    opt.read_state(m8, v8, s, m_out, v_out)
    assert torch.isnan(m_out[o + 600]) and torch.isnan(m_out[o + 601])
    assert v8[o + 602] == 255 and v8[o + 603] == 255
    assert torch.equal(m8[o + 604:o + 640], ref[0][o + 604:o + 640]) and torch.equal(v8[o + 604:o + 640], ref[1][o + 604:o + 640])


def test_8_bit_rounding_of_v_is_unbiased():
    """The mean over seeds is the value itself: a step of the grid is at most v/16, the mean of N draws is within 5 standard
    deviations (half a step at most, over sqrt(N)) for every element."""
    from paper_2508_15706_b200.inner import AdamW
    opt = AdamW([(8, 128)], state_bits=8)
    v = torch.rand(1024, device="cuda") * 0.9 + 0.1
    m = torch.zeros(1024, device="cuda")
    state, total, N = opt.new_state(), torch.zeros(1024, dtype=torch.float64, device="cuda"), 400
    m_out, v_out = torch.zeros(1024, device="cuda"), torch.zeros(1024, device="cuda")
    for seed in range(N):
        opt.write_state(m, v, *state, seed=seed)
        opt.read_state(*state, m_out, v_out)
        total += v_out.double()
    assert torch.all((total / N - v.double()).abs() <= 5 * (v / 32) / math.sqrt(N))
    assert abs((total / N / v).mean().item() - 1) <= 5 / 32 / math.sqrt(N * 1024)


def test_8_bit_training_follows_32_bit():
    """A noisy quadratic: both end near the minimum, beta2 = 0.999 included (where rounding v to nearest would freeze it)."""
    from paper_2508_15706_b200.inner import AdamW
    n = 4096
    g = torch.Generator(device="cuda").manual_seed(9)
    goal = torch.randn(n, generator=g, device="cuda")
    scale = torch.exp(torch.randn(n, generator=g, device="cuda"))
    ends = []
    for bits in (32, 8):
        opt = AdamW([(32, 128)], weight_decay=0.0, betas=(0.9, 0.999), max_norm=0.0, state_bits=bits)
        theta, state = torch.zeros(n, device="cuda"), opt.new_state()
        gen = torch.Generator(device="cuda").manual_seed(10)
        for t in range(1, 601):
            grad = scale * (theta - goal) + 0.3 * torch.randn(n, generator=gen, device="cuda")
            opt.step(theta, grad, *state, step=t, lr=2e-2 * (1 - t / 601))
        ends.append((scale * (theta - goal).square()).mean().item())
    start = (scale * goal.square()).mean().item()
    assert ends[0] < 0.02 * start and ends[1] < 2 * ends[0] + 1e-3 * start


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_non_finite_gradients(bits, bad):
    from paper_2508_15706_b200.inner import AdamW
    shapes = [(5, 1000)]
    theta, grad = inputs(5000, 3, torch.float32, torch.float32)
    grad[4321] = bad
    for skip in (True, False):
        opt = AdamW(shapes, state_bits=bits, skip_nonfinite=skip, max_norm=1.0 if skip else 0.0)
        state, p, norm = opt.new_state(), theta.clone(), torch.zeros(1, device="cuda")
        kept = [x.clone() for x in state if x is not None]
        opt.step(p, grad, *state, step=1, lr=1e-2, norm=norm)
        assert not torch.isfinite(norm).item()
        if skip:
            assert torch.equal(p, theta) and all(torch.equal(a, b) for a, b in zip(kept, [x for x in state if x is not None]))
        else:
            wrong = ~torch.isfinite(p)
            # a NaN reaches the parameter; an infinite gradient has an infinite v: inf / inf is NaN too
            assert wrong[4321].item()
            assert not torch.any(wrong[:4321]) and not torch.any(wrong[4322:])
        grad2 = inputs(5000, 4, torch.float32, torch.float32)[1]
        if skip:  # the next step is an ordinary one
            opt.step(p, grad2, *state, step=2, lr=1e-2, norm=norm)
            assert torch.isfinite(norm).item() and torch.all(torch.isfinite(p)) and not torch.equal(p, theta)


@pytest.mark.parametrize("bits", [32, 8])
def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph(bits):
    from paper_2508_15706_b200.inner import AdamW
    n = 300 * 1000
    shapes = [(300, 1000)]
    theta, grad = inputs(n, 6, torch.float32, torch.float32)
    opt = AdamW(shapes, state_bits=bits)
    ends = []
    for how in ("plain", "stream", "graph"):
        p, state, norm = theta.clone(), opt.new_state(), torch.zeros(1, device="cuda")
        if how == "plain":
            for _ in range(3):
                opt.step(p, grad, *state, step=5, lr=1e-3, norm=norm)
        else:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                if how == "stream":
                    for _ in range(3):
                        opt.step(p, grad, *state, step=5, lr=1e-3, norm=norm)
                else:
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=side):
                        opt.step(p, grad, *state, step=5, lr=1e-3, norm=norm)
                    for _ in range(3):
                        graph.replay()
            side.synchronize()
        ends.append([p, norm, *[x for x in state if x is not None]])
    for other in ends[1:]:
        assert all(torch.equal(a, b) for a, b in zip(ends[0], other))


def test_refusals():
    from paper_2508_15706_b200 import binding as B
    from paper_2508_15706_b200.inner import AdamW

    def refused(status, fn, *a, **k):
        with pytest.raises(B.SlError) as e:
            fn(*a, **k)
        assert e.value.status == status

    refused(B.SL_ERR_INVALID_ARG, AdamW, [(4, 4), (4, 4)], [0, 12])  # overlap
    refused(B.SL_ERR_ALIGNMENT, AdamW, [(4, 4)], [2])
    refused(B.SL_ERR_UNSUPPORTED, AdamW, [(4, 4)], state_bits=16)
    refused(B.SL_ERR_INVALID_ARG, AdamW, [(4, 4)], betas=(1.0, 0.9))
    refused(B.SL_ERR_INVALID_ARG, AdamW, [(4, 4)], eps=float("nan"))
    refused(B.SL_ERR_INVALID_ARG, AdamW, [(4, 4)], weight_decay=[0.1, 0.1])
    refused(B.SL_ERR_INVALID_ARG, AdamW, [(4, 4)], grad_dtype=torch.float16)
    refused(B.SL_ERR_TOO_LARGE, AdamW, [(1 << 30, 1 << 20)])
    opt, opt8 = AdamW([(4, 4)]), AdamW([(4, 4)], state_bits=8)
    t = [torch.zeros(64, device="cuda") for _ in range(4)]
    refused(B.SL_ERR_INVALID_ARG, opt.step, *t, step=0, lr=1e-3)
    refused(B.SL_ERR_INVALID_ARG, opt.step, *t, step=1, lr=float("inf"))
    refused(B.SL_ERR_INVALID_ARG, opt.step, t[0], t[0], t[1], t[2], step=1, lr=1e-3)
    refused(B.SL_ERR_INVALID_ARG, opt.step, t[0], t[1], t[2], t[3][:8], step=1, lr=1e-3)
    refused(B.SL_ERR_INVALID_ARG, opt.step, t[0], t[1], t[2], t[3].half(), step=1, lr=1e-3)
    refused(B.SL_ERR_INVALID_ARG, opt.step, t[0].cpu(), t[1], t[2], t[3], step=1, lr=1e-3)
    refused(B.SL_ERR_ALIGNMENT, opt.step, t[0][1:], t[1], t[2], t[3], step=1, lr=1e-3)
    m, v, s = opt8.new_state()
    refused(B.SL_ERR_INVALID_ARG, opt8.step, t[0], t[1], m, v, None, step=1, lr=1e-3)
    refused(B.SL_ERR_INVALID_ARG, opt8.read_state, m, v, s, t[0], t[0])
    bf = AdamW([(4, 4)], param_dtype=torch.bfloat16)
    refused(B.SL_ERR_INVALID_ARG, bf.step, t[0].bfloat16(), t[1], t[2], t[3], step=1, lr=1e-3, copy=torch.zeros(64, dtype=torch.bfloat16, device="cuda"))
