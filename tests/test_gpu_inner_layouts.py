"""The autograd functions on tensors as a model hands them over: transposed, expanded over rows or tokens, slices of something larger.
Results and gradients are those of contiguous copies, bit for bit (the kernels' order of sums does not depend on strides here)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def transposed(t):
    """The same values, last and first axis the other way round in memory."""
    return t.detach().transpose(0, -1).contiguous().transpose(0, -1)


def sliced(t):
    wide = torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype, device=t.device)
    wide[..., 1::2] = t
    return wide[..., 1::2]


def same(f, args, changed):
    """f of the changed tensors against f of contiguous ones: outputs, and gradients of every floating-point argument."""
    results = []
    for given in (args, changed):
        leaf = [t.detach().requires_grad_(t.is_floating_point()) for t in given]
        out = [o for o in f(*leaf) if o is not None]
        w = [torch.linspace(-1.0, 1.0, o.numel(), device="cuda").view(o.shape).to(o.dtype) for o in out]
        wanted = [t for t in leaf if t.requires_grad]
        results.append(out + list(torch.autograd.grad(sum((o * x).sum() for o, x in zip(out, w)), wanted)))
    for a, b in zip(*results):
        assert a.shape == b.shape and torch.equal(a, b)


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("change", [transposed, sliced])
@pytest.mark.parametrize("gate", ["none", "column", "row", "full"])
def test_block_norm(act, change, gate):
    from paper_2508_15706_b200 import inner
    x, b = (torch.randn(2, 35, 96, device="cuda").to(act) for _ in range(2))
    w, bw = (torch.rand(96, device="cuda") for _ in range(2))
    g = {"none": [], "column": [torch.rand(96, device="cuda")], "row": [torch.rand(2, 35, 1, device="cuda").to(act)], "full": [torch.rand(2, 35, 96, device="cuda").to(act)]}[gate]

    def f(x, b, w, bw, g=None):
        return inner.block_norm(x, w, branch=b, branch_weight=bw, gate=g, alpha=0.5)

    args = [x, b, w, bw] + g
    same(f, args, [sliced(t) if t.dim() == 1 else change(t) for t in args])
    same(lambda x, w: inner.block_norm(x, w), [x[0], w], [change(x[0]), w])


def test_block_norm_of_expanded_tensors():
    """One row for all tokens, one gate row for all of them: gradients are summed over what was shared."""
    from paper_2508_15706_b200 import inner
    x, b, g, w = torch.randn(7, 64, device="cuda"), torch.randn(1, 64, device="cuda"), torch.rand(1, 64, device="cuda"), torch.rand(64, device="cuda")
    leaf = [t.requires_grad_() for t in (x, b, g, w)]
    y, h = inner.block_norm(x, w, branch=b.expand(7, 64), gate=g.expand(7, 64))
    y2, h2 = inner.block_norm(x, w, branch=b.expand(7, 64).contiguous(), gate=g.expand(7, 64).contiguous())
    assert torch.equal(y, y2) and torch.equal(h, h2)
    for a, c in zip(torch.autograd.grad((h * y).sum(), leaf), torch.autograd.grad((h2 * y2).sum(), leaf)):
        assert torch.equal(a, c)


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("change", [transposed, sliced])
def test_rotary(act, change):
    from paper_2508_15706_b200 import inner
    rope = inner.Rotary(32)
    q, k = torch.randn(2, 9, 3, 48, device="cuda").to(act), torch.randn(2, 9, 1, 48, device="cuda").to(act)
    same(lambda q, k: inner.rotary(rope, q, k, first=5), [q, k], [change(q), change(k)])


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("change", [transposed, sliced])
def test_loss(act, change):
    from paper_2508_15706_b200 import inner
    x, t = torch.randn(3, 20, 257, device="cuda").to(act), torch.randint(0, 257, (3, 20), device="cuda")
    same(lambda x, t: (inner.next_token_loss(x, t, smoothing=0.1),), [x, t], [change(x), sliced(t)])
    flat, to = x.view(60, 257), t.view(60)
    same(lambda x, t: (inner.next_token_loss(x, t),), [flat, to], [change(flat), sliced(to)])
