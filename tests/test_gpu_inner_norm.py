"""Residual update and norms around a block (sl_norm_forward / sl_norm_backward) against the formulas in 64 bits, and the
gradients against differences.

Tolerances (u = 2^-24): a row sum of n positive terms in 32 threads or more is good to about (n / 32 + 10) u, at most 2^-14.9 at
the widest row and far below that elsewhere: 2^-19 up to 4096 columns, 2^-16 beyond; outputs are a few products of such numbers.
An output that is stored in bfloat16 is the rounding of such a number."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)]


def make(rows, cols, act, wt, gate, post, seed, pad=0, shift=0):
    """Inputs; `pad` extra columns between rows, `shift` elements off the allocation's start."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def mat(sigma=1.0, dtype=act):
        buf = torch.empty(rows * (cols + pad) + shift + 8, device="cuda").normal_(0.0, sigma, generator=g).to(dtype)
        return buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]

    def vec(mean, dtype=wt):
        return (mean + 0.3 * torch.empty(cols + shift, device="cuda").normal_(generator=g)).to(dtype)[shift:]

    return {"x": mat(2.0), "branch": mat(0.5), "weight": vec(1.0), "branch_weight": vec(0.7) if post else None,
            "gate": {"none": None, "column": vec(0.5), "row": mat(1.0)[:, :1] if cols > 1 else mat(1.0)[:, 0], "full": mat(1.0)}[gate]}


def forward64(x, branch, weight, branch_weight, gate, alpha, eps):
    z, br = branch, None
    if branch is not None and branch_weight is not None:
        br = (branch.square().mean(1) + eps).rsqrt()
        z = branch * br[:, None] * branch_weight
    y = x
    if branch is not None:
        if gate is not None and gate.dim() == 1 and gate.shape[0] != x.shape[1]:
            gate = gate[:, None]
        y = x + alpha * (z if gate is None else gate * z)
    r = (y.square().mean(1) + eps).rsqrt()
    h = y * r[:, None] * (1.0 if weight is None else weight)
    return y, h, r, br


def d64(t):
    return None if t is None else t.double()


def inside(got, want, tol, what=""):
    """got is want up to tol; stored in bfloat16, the rounding of some number up to tol from want (rounding keeps order)."""
    low, high = (want - tol).to(got.dtype), (want + tol).to(got.dtype)
    bad = ~((got >= low) & (got <= high))
    assert not torch.any(bad), (what, (got.double() - want)[bad][:4], want[bad][:4])


def close(got, want, size, cols, what):
    rel = 2.0 ** -19 if cols <= 4096 else 2.0 ** -16
    inside(got, want, rel * size + 1e-30, what)


CASES = [(1, 1, 0, 0), (3, 2, 0, 0), (5, 31, 0, 0), (7, 64, 0, 0), (33, 100, 4, 0), (9, 256, 8, 8), (300, 257, 0, 0), (2, 1000, 0, 0), (700, 1280, 0, 0), (130, 2048, 16, 0),
         (17, 2050, 3, 1), (1, 2048, 0, 0), (6, 4104, 0, 0), (3, 8192, 0, 0), (2, 9001, 0, 0), (3, 16384, 0, 0), (2, 16383, 1, 0)]


@pytest.mark.parametrize("rows,cols,pad,shift", CASES)
@pytest.mark.parametrize("act,wt", TYPES)
@pytest.mark.parametrize("gate,post", [("none", False), ("column", True), ("row", True), ("full", True), ("row", False), ("full", False), ("none", True), ("column", False)])
def test_forward_and_backward(rows, cols, pad, shift, act, wt, gate, post):
    from paper_2508_15706_b200 import inner
    if gate == "column" and cols == 1 or gate == "row" and rows == cols:
        pytest.skip("a one-dimensional gate of this size would be ambiguous")
    s = make(rows, cols, act, wt, gate, post, rows * 1000 + cols, pad, shift)
    alpha, eps = 0.6, 1e-5
    y, h, r, br = inner.norm_forward(s["x"], s["weight"], branch=s["branch"], branch_weight=s["branch_weight"], gate=s["gate"], alpha=alpha, eps=eps)
    x64, b64, w64, bw64, g64 = (d64(s[k]) for k in ("x", "branch", "weight", "branch_weight", "gate"))
    wy, wh, wr, wbr = forward64(x64, b64, w64, bw64, g64, alpha, eps)
    step = (wy - x64).abs()
    close(y, wy, x64.abs() + step, cols, "y")
    close(h, wh, (x64.abs() + step) * wr[:, None] * w64.abs() + wh.abs(), cols, "h")
    # rstd moves with the relative error of y's square mean
    assert torch.all((r.double() / wr - 1).abs() <= (2.0 ** -19 if cols <= 4096 else 2.0 ** -16) * (1 + ((x64.abs() + step).square().mean(1) * wr ** 2)))
    if post:
        assert torch.all((br.double() / wbr - 1).abs() <= (2.0 ** -19 if cols <= 4096 else 2.0 ** -16))

    # backward, at the y, rstd and branch_rstd that the forward pass left
    g = torch.Generator(device="cuda").manual_seed(7)
    dy = torch.randn(rows, cols, generator=g, device="cuda").to(act)
    dh = torch.randn(rows, cols, generator=g, device="cuda").to(act)
    out = {k: torch.full_like(v, 9.0, memory_format=torch.contiguous_format) if v is not None else None for k, v in
           (("dx", y), ("dweight", s["weight"]), ("dbranch_weight", s["branch_weight"]))}
    out["dbranch"] = torch.empty_strided(s["branch"].shape, s["branch"].stride(), dtype=act, device="cuda")
    out["dgate"] = None if s["gate"] is None else torch.empty_strided(s["gate"].shape, s["gate"].stride(), dtype=s["gate"].dtype, device="cuda")
    inner.norm_backward(dy, dh, y, s["weight"], rstd=r, branch=s["branch"], branch_weight=s["branch_weight"], branch_rstd=br, gate=s["gate"], alpha=alpha, **out)
    y64, dy64, dh64, r64 = y.double(), dy.double(), dh.double(), r.double()[:, None]
    yh, u = y64 * r64, dh64 * w64
    dx = dy64 + r64 * (u - yh * (u * yh).mean(1, keepdim=True))
    size_x = dy64.abs() + r64 * (u.abs() + yh.abs() * (u * yh).abs().mean(1, keepdim=True))
    close(out["dx"], dx, size_x, cols, "dx")
    close(out["dweight"], (dh64 * yh).sum(0), (dh64 * yh).abs().sum(0), cols, "dweight")
    rb = br.double()[:, None] if post else 1.0
    bh = b64 * rb
    z = bh * (bw64 if post else 1.0)
    gg = 1.0 if g64 is None else (g64[:, None] if g64.dim() == 1 and gate == "row" else g64)
    if gate == "column":
        close(out["dgate"], (alpha * dx * z).sum(0), (alpha * size_x * z.abs()).sum(0), cols, "dgate")
    elif gate == "row":
        close(out["dgate"].view(-1), (alpha * dx * z).sum(1), (alpha * size_x * z.abs()).sum(1), cols, "dgate")
    elif gate == "full":
        close(out["dgate"], alpha * dx * z, alpha * size_x * z.abs(), cols, "dgate")
    dz, size_z = alpha * dx * gg, alpha * size_x * (gg.abs() if torch.is_tensor(gg) else gg)
    if post:
        q, sq = dz * bw64, size_z * bw64.abs()
        close(out["dbranch"], rb * (q - bh * (q * bh).mean(1, keepdim=True)), rb * (sq + bh.abs() * (sq * bh.abs()).mean(1, keepdim=True)), cols, "dbranch")
        close(out["dbranch_weight"], (dz * bh).sum(0), (size_z * bh.abs()).sum(0), cols, "dbranch_weight")
    else:
        close(out["dbranch"], dz, size_z, cols, "dbranch")


@pytest.mark.parametrize("cols", [5, 640, 2048])
def test_norm_alone_and_its_absences(cols):
    """Without a branch (the first norm of a stack), without weights, without dy, without dh, outputs left out."""
    from paper_2508_15706_b200 import inner
    s = make(50, cols, torch.float32, torch.float32, "none", False, cols)
    y, h, r, br = inner.norm_forward(s["x"], s["weight"], eps=1e-6)
    assert y is s["x"] and br is None
    x, w = s["x"].double(), s["weight"].double()
    wr = (x.square().mean(1) + 1e-6).rsqrt()
    close(h, x * wr[:, None] * w, (x * wr[:, None] * w).abs(), cols, "h")
    _, h1, _, _ = inner.norm_forward(s["x"], eps=1e-6)
    close(h1, x * wr[:, None], (x * wr[:, None]).abs(), cols, "h without weight")
    y2, h2, r2, _ = inner.norm_forward(s["x"], branch=s["branch"], alpha=2.0, norm=False)
    assert h2 is None and r2 is None
    close(y2, x + 2.0 * s["branch"].double(), x.abs() + 2 * s["branch"].double().abs(), cols, "y")
    dh = torch.randn(50, cols, device="cuda")
    dx, dw = torch.empty_like(dh), torch.empty(cols, device="cuda")
    inner.norm_backward(None, dh, s["x"], s["weight"], rstd=r, dx=dx, dweight=dw)
    yh, u = x * r.double()[:, None], dh.double() * w
    close(dx, r.double()[:, None] * (u - yh * (u * yh).mean(1, keepdim=True)), r.double()[:, None] * (u.abs() + yh.abs() * (u * yh).abs().mean(1, keepdim=True)), cols, "dx")
    close(dw, (dh.double() * yh).sum(0), (dh.double() * yh).abs().sum(0), cols, "dw")
    db = torch.empty_like(dh)
    inner.norm_backward(dh, None, None, branch=s["branch"], alpha=2.0, dbranch=db)
    assert torch.equal(db, 2.0 * dh)


def test_in_place_and_repeatable():
    """y over x, h over branch, dx over dy, dbranch over dh; column sums repeat bit for bit."""
    from paper_2508_15706_b200 import inner
    for cols in (96, 1280, 2051, 5000):
        s = make(333, cols, torch.bfloat16, torch.float32, "column", True, cols)
        y, h, r, br = inner.norm_forward(s["x"], s["weight"], branch=s["branch"], branch_weight=s["branch_weight"], gate=s["gate"])
        x2, b2 = s["x"].clone(), s["branch"].clone()
        inner.norm_forward(x2, s["weight"], branch=b2, branch_weight=s["branch_weight"], gate=s["gate"], y=x2, h=b2)
        assert torch.equal(x2, y) and torch.equal(b2, h)
        dy, dh = torch.randn_like(y), torch.randn_like(y)
        runs = []
        for k in range(2):
            o = {"dx": torch.empty_like(y) if k == 0 else dy, "dbranch": torch.empty_like(y) if k == 0 else dh, "dweight": torch.empty_like(s["weight"]),
                 "dbranch_weight": torch.empty_like(s["weight"]), "dgate": torch.empty_like(s["weight"])}
            inner.norm_backward(dy, dh, y, s["weight"], rstd=r, branch=s["branch"], branch_weight=s["branch_weight"], branch_rstd=br, gate=s["gate"], **o)
            runs.append([t.clone() for t in o.values()])
        assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_zero_rows():
    from paper_2508_15706_b200 import inner
    z = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    y, h, r, br = inner.norm_forward(z, w, branch=z.clone(), branch_weight=w)
    assert y.shape == (0, 64) and r.numel() == 0
    dw, dbw = torch.full_like(w, 3.0), torch.full_like(w, 3.0)
    inner.norm_backward(z, z, y, w, rstd=r, branch=z, branch_weight=w, branch_rstd=br, dweight=dw, dbranch_weight=dbw)
    assert torch.all(dw == 0) and torch.all(dbw == 0)


def test_zeros_and_non_finite_rows_stay_in_their_row():
    from paper_2508_15706_b200 import inner
    x = torch.randn(6, 512, device="cuda")
    x[1] = 0.0
    x[3, 100] = float("inf")
    x[4, 7] = float("nan")
    _, h, r, _ = inner.norm_forward(x, eps=1e-6)
    assert torch.all(h[1] == 0) and abs(r[1].item() - 1e3) < 1e-2
    assert torch.all(torch.isfinite(h[[0, 1, 2, 5]])) and torch.isnan(h[3, 100]) and torch.all(torch.isnan(h[4]))


@pytest.mark.parametrize("gate", ["none", "column", "row", "full"])
@pytest.mark.parametrize("post", [False, True])
def test_gradients_against_differences(gate, post):
    """Directional derivatives of a scalar of (y, h), central differences of the 64-bit formula, against the kernels' gradients
    through autograd.  The difference's own error is about h^2 = 1e-10 and 1e-16 / h = 1e-11 of the scalar's scale."""
    from paper_2508_15706_b200 import inner
    rows, cols, alpha, eps = 21, 72, 0.7, 1e-5
    s = make(rows, cols, torch.float32, torch.float32, gate, post, 12)
    names = [k for k in ("x", "branch", "weight", "branch_weight", "gate") if s[k] is not None]
    leaf = {k: s[k].clone().contiguous().requires_grad_() for k in names}
    cy, ch = torch.randn(rows, cols, device="cuda"), torch.randn(rows, cols, device="cuda")
    y, h = inner.block_norm(leaf["x"], leaf["weight"], branch=leaf["branch"], branch_weight=leaf.get("branch_weight"), gate=leaf.get("gate"), alpha=alpha, eps=eps)
    ((y * cy).sum() + (h * ch).sum()).backward()

    def scalar(v):
        a, b, _, _ = forward64(v["x"], v["branch"], v["weight"], v.get("branch_weight"), v.get("gate"), alpha, eps)
        return ((a * cy.double()).sum() + (b * ch.double()).sum()).item()

    base = {k: s[k].double() for k in names}
    for k in names:
        d = torch.randn_like(base[k])
        t = 1e-5
        slope = (scalar({**base, k: base[k] + t * d}) - scalar({**base, k: base[k] - t * d})) / (2 * t)
        got = (leaf[k].grad.double() * d).sum().item()
        size = (leaf[k].grad.double() * d).abs().sum().item()
        assert abs(got - slope) <= 2.0 ** -18 * size + 1e-7 * size, (k, got, slope)


def test_refusals():
    from paper_2508_15706_b200 import binding as B
    from paper_2508_15706_b200 import inner
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    r = torch.ones(4, device="cuda")

    def refused(status, fn, *a, **k):
        with pytest.raises(B.SlError) as e:
            fn(*a, **k)
        assert e.value.status == status

    refused(B.SL_ERR_INVALID_ARG, inner.norm_forward, x, w[:32])
    refused(B.SL_ERR_INVALID_ARG, inner.norm_forward, x, w, branch=x[:, :32])
    refused(B.SL_ERR_INVALID_ARG, inner.norm_forward, x, w, branch_weight=w)
    refused(B.SL_ERR_INVALID_ARG, inner.norm_forward, x, w, gate=w)
    refused(B.SL_ERR_INVALID_ARG, inner.norm_forward, x, w, eps=-1.0)
    refused(B.SL_ERR_INVALID_ARG, inner.norm_forward, x.half(), w)
    refused(B.SL_ERR_INVALID_ARG, inner.norm_forward, x.t(), None)
    refused(B.SL_ERR_UNSUPPORTED, inner.norm_forward, x, w.bfloat16())
    refused(B.SL_ERR_TOO_LARGE, inner.norm_forward, torch.zeros(1, 16385, device="cuda"))
    refused(B.SL_ERR_INVALID_ARG, inner.norm_backward, None, None, x, w, rstd=r, dx=x)
    refused(B.SL_ERR_INVALID_ARG, inner.norm_backward, None, x, x, w, dx=x.clone())
    refused(B.SL_ERR_INVALID_ARG, inner.norm_backward, x, None, None, dbranch=x.clone())
    refused(B.SL_ERR_NOMEM, inner.norm_backward, None, x, x, w, rstd=r, dweight=w.clone(), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
