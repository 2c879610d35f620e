"""Norms of far more rows than are resident, in the forms with one exchange between a row's warps (no branch weight, or no h):
every team takes row after row, and a warp's sums must not meet those of the next row.

The formulas and tolerances are those of test_gpu_inner_norm.py; repeated runs leave the same bits."""
import pytest
import torch

from test_gpu_inner_norm import close, d64, forward64, make

pytestmark = pytest.mark.gpu

# rows of one warp, two warps, many warps on 16-byte boundaries; of several warps by single and by pairs of values; of many columns a thread
SIZES = [(20000, 512), (20000, 1280), (20000, 2048), (4000, 4096), (4000, 5000), (20000, 1003), (8000, 2050), (1500, 9001), (1500, 16384)]
FORMS = {"norm": {}, "residual and norm": {"branch": True}, "residual with its norm, no h": {"branch": True, "post": True, "norm": False}, "both norms": {"branch": True, "post": True}}


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gate", ["none", "full"])
def test_forward(rows, cols, form, act, gate):
    from paper_2508_15706_b200 import inner
    f = FORMS[form]
    if gate == "full" and not f.get("branch"):
        pytest.skip("a gate needs a branch")
    s = make(rows, cols, act, torch.float32, gate, bool(f.get("post")), cols)
    norm = f.get("norm", True)
    k = {"branch": s["branch"], "branch_weight": s["branch_weight"], "gate": s["gate"], "alpha": 0.6} if f.get("branch") else {}
    weight = s["weight"] if norm else None
    runs = [inner.norm_forward(s["x"], weight, eps=1e-5, norm=norm, **k) for _ in range(4)]
    for other in runs[1:]:
        assert all(a is b or torch.equal(a, b) for a, b in zip(runs[0], other))
    y, h, r, br = runs[0]
    x64 = s["x"].double()
    wy, wh, wr, wbr = forward64(x64, *(d64(k.get(n)) for n in ("branch",)), d64(weight), d64(k.get("branch_weight")), d64(k.get("gate")), 0.6, 1e-5)
    step = (wy - x64).abs()
    rel = 2.0 ** -19 if cols <= 4096 else 2.0 ** -16
    if k:
        close(y, wy, x64.abs() + step, cols, "y")
    if norm:
        close(h, wh, (x64.abs() + step) * wr[:, None] * d64(weight).abs() + wh.abs(), cols, "h")
        assert torch.all((r.double() / wr - 1).abs() <= rel * (1 + (x64.abs() + step).square().mean(1) * wr ** 2))
    if f.get("post"):
        assert torch.all((br.double() / wbr - 1).abs() <= rel)
