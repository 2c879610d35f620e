"""The operators of the inner phase (H local steps of every worker between two outer steps): their plain forms in
elementary torch operations, their definitions in 64 bits, and the cases they are timed and compared on.

  adamw   one AdamW step over the whole tensor table, gradient clipping by the global norm included; moments kept in 32
          bits, or in 8 bits with one power-of-two scale per 128 elements
  norm    residual update and norms around a block: y = x + alpha * gate * norm(branch), h = norm(y); forward and backward
  rotary  rotary positions of queries and keys; forward and backward
  loss    next-token loss and its gradient with respect to the logits

Sizes follow the decoder stacks this repository trains between outer steps (widths 768 to 2048, head dimension 64 or 128,
a vocabulary of 32000), with odd and ragged ones around them.
"""
import math

import torch

own = False

M32 = 0xFFFFFFFF
BLOCK = 128  # elements that share one scale of an 8-bit moment
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the norm vectors of the 1280-wide stack alone (25 small tensors): what a step costs when nothing is large
        {"name": "adamw vectors 32-bit", "op": "adamw", "width": 1280, "ffn": 0, "layers": 12, "vocab": 0, "bits": 32, "grad": "fp32", "copy": False, "clip": 1.0},
        # one 1024 x 1024 matrix (the smallest outer-step workload), moments in 8 bits
        {"name": "adamw 1024x1024 8-bit", "op": "adamw", "width": 1024, "ffn": 0, "layers": 0, "vocab": 1024, "bits": 8, "grad": "fp32", "copy": False, "clip": 1.0},
        # four decoder layers 1280 wide: fp32 master parameters, bfloat16 gradients and working copy
        {"name": "adamw d1280 32-bit", "op": "adamw", "width": 1280, "ffn": 5120, "layers": 4, "vocab": 0, "bits": 32, "grad": "bf16", "copy": True, "clip": 1.0},
        # embedding and two decoder layers 2048 wide, moments in 8 bits, the moments read out afterwards
        {"name": "adamw d2048 8-bit", "op": "adamw", "width": 2048, "ffn": 8192, "layers": 2, "vocab": 32000, "bits": 8, "grad": "fp32", "copy": False, "clip": 1.0},
        # one token of a 2048-wide stack (generation): branch norm, learned gate, residual, next norm
        {"name": "norm forward one token", "op": "norm", "rows": 1, "cols": 2048, "act": "bf16", "weight": "bf16", "gate": "channel", "post": True, "alpha": 0.5, "backward": False},
        # a training batch of 16 x 1024 tokens, 2048 wide
        {"name": "norm forward 16384x2048", "op": "norm", "rows": 16384, "cols": 2048, "act": "bf16", "weight": "fp32", "gate": "channel", "post": True, "alpha": 0.5, "backward": False},
        # its gradients on a ragged packed batch of the 1280-wide stack
        {"name": "norm backward 10007x1280", "op": "norm", "rows": 10007, "cols": 1280, "act": "bf16", "weight": "fp32", "gate": "channel", "post": True, "alpha": 0.5, "backward": True},
        # packed training batch, 16 heads of 128, keys and queries taken out of one qkv product
        {"name": "rotary half 8x4096", "op": "rotary", "batch": 8, "seq": 4096, "q_heads": 16, "k_heads": 16, "head_dim": 128, "rot": 128, "layout": "half", "act": "bf16", "inverse": False, "scaling": "none", "far": 0},
        # gradients of a grouped-query stack with half of each head rotated, fp32
        {"name": "rotary interleaved backward", "op": "rotary", "batch": 3, "seq": 1021, "q_heads": 10, "k_heads": 5, "head_dim": 128, "rot": 64, "layout": "interleaved", "act": "fp32", "inverse": True, "scaling": "none", "far": 0},
        # sixteen sequences, one new token each, far into a context stretched eight times
        {"name": "rotary decode far", "op": "rotary", "batch": 16, "seq": 1, "q_heads": 16, "k_heads": 16, "head_dim": 128, "rot": 128, "layout": "half", "act": "bf16", "inverse": False, "scaling": "by_parts", "far": 200000},
        # a short ragged batch with label smoothing
        {"name": "loss 37x32000", "op": "loss", "rows": 37, "vocab": 32000, "act": "fp32", "smoothing": 0.1, "z": 0.0, "ignored": 0.2, "masked": 0},
        # 8 x 1024 tokens, the vocabulary of every model here
        {"name": "loss 8192x32000", "op": "loss", "rows": 8192, "vocab": 32000, "act": "bf16", "smoothing": 0.0, "z": 1e-4, "ignored": 0.05, "masked": 0},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["adamw", "adamw", "norm", "norm", "rotary", "loss"])
    act = rng.choice(["bf16", "bf16", "fp32"])
    if op == "adamw":
        width, layers = _log(rng, 65, 2048), rng.randint(1, 3)
        grad = rng.choice(["bf16", "fp32"])
        return {"op": op, "width": width, "ffn": rng.choice([0, 2 * width + rng.randint(0, 9), 4 * width]), "layers": layers, "vocab": rng.choice([0, _log(rng, 100, 16000)]),
                "bits": rng.choice([32, 8]), "grad": grad, "copy": rng.random() < 0.5, "clip": rng.choice([0.0, 0.05, 1.0])}
    if op == "norm":
        rows, cols = _log(rng, 1, 12000), rng.choice([_log(rng, 16, 2048), 64 * rng.randint(1, 32)])
        gate = rng.choice(["none", "channel", "token", "full"])
        return {"op": op, "rows": rows, "cols": cols, "act": act, "weight": rng.choice(["fp32", act]), "gate": gate, "post": rng.random() < 0.7, "alpha": rng.choice([1.0, 0.5, 0.22]), "backward": rng.random() < 0.5}
    if op == "rotary":
        hd = rng.choice([64, 80, 96, 128])
        batch, seq = rng.choice([(_log(rng, 1, 64), 1), (rng.randint(1, 6), _log(rng, 2, 4096))])
        kh = rng.choice([1, 2, 4, 8])
        return {"op": op, "batch": batch, "seq": seq, "q_heads": kh * rng.choice([1, 2]), "k_heads": kh, "head_dim": hd, "rot": rng.choice([hd, hd // 2, 2 * (hd // 5)]),
                "layout": rng.choice(["half", "interleaved"]), "act": act, "inverse": rng.random() < 0.4, "scaling": rng.choice(["none", "linear", "by_parts"]), "far": rng.choice([0, _log(rng, 100, 500000)])}
    rows, vocab = _log(rng, 1, 4096), rng.choice([32000, _log(rng, 500, 50000)])
    smoothing = rng.choice([0.0, 0.0, 0.1])
    return {"op": op, "rows": rows, "vocab": vocab, "act": act, "smoothing": smoothing, "z": rng.choice([0.0, 1e-4]), "ignored": rng.choice([0.0, 0.1, 0.5]), "masked": 0 if smoothing else rng.choice([0, 0, 37])}


# --------------------------------------------------------------------------------------------------------------- inputs
def _shapes(case):
    """(rows, cols, decays) of every parameter tensor: `vocab` embedding rows, decoder layers, a final norm vector."""
    d, f, t = case["width"], case["ffn"], []
    if case["vocab"]:
        t.append((case["vocab"], d, True))
    for _ in range(case["layers"]):
        if f:
            t += [(d, d, True)] * 4 + [(f, d, True)] * 2 + [(d, f, True)]
        t += [(1, d, False)] * 2
    if case["layers"]:
        t.append((1, d, False))
    return t


def _table(case):
    """Shapes, element offsets (each on a 128-element boundary, so the plain form can see blocks as rows) and length."""
    at, offsets = 0, []
    shapes = _shapes(case)
    for rows, cols, _ in shapes:
        offsets.append(at)
        at += (rows * cols + BLOCK - 1) // BLOCK * BLOCK
    return shapes, offsets, at


def _gen(seed, *more):
    g = torch.Generator(device="cuda")
    s = int(seed) + 1
    for x in more:
        s = (s * 1000003 + int(x)) & 0x7FFFFFFFFFFF
    g.manual_seed(s)
    return g


def prepare(case, seed):
    return {"adamw": _prepare_adamw, "norm": _prepare_norm, "rotary": _prepare_rotary, "loss": _prepare_loss}[case["op"]](case, seed)


def _prepare_adamw(case, seed):
    shapes, offsets, n = _table(case)
    g, dev = _gen(seed, 1), "cuda"
    theta, grad = torch.zeros(n, device=dev), torch.zeros(n, device=dev)
    m, v = torch.zeros(n, device=dev), torch.zeros(n, device=dev)
    decay = torch.zeros(n // BLOCK, 1, device=dev)
    for i, ((rows, cols, decays), off) in enumerate(zip(shapes, offsets)):
        s = slice(off, off + rows * cols)
        sigma = 10.0 ** (-4.0 + 1.5 * ((i * 37) % 11) / 10.0)  # gradient scale of this tensor
        theta[s].normal_(0.0 if decays else 1.0, 0.02, generator=g)
        # heavier than normal, as gradients are: a normal times a log-normal of the same element
        grad[s].normal_(0.0, 0.7, generator=g).exp_()
        grad[s] *= torch.randn(rows * cols, generator=g, device=dev) * sigma
        m[s].normal_(0.0, 0.3 * sigma, generator=g)
        v[s].normal_(0.0, 1.0, generator=g).exp_()
        v[s] *= sigma * sigma
        decay[off // BLOCK:(off + rows * cols + BLOCK - 1) // BLOCK] = 0.1 if decays else 0.0
    state = {"case": case, "theta": theta, "grad": grad.to(DTYPES[case["grad"]]), "decay": decay, "seed": int(seed) & 0xFFFF, "t": 250, "lr": 4e-4,
             "norm": torch.zeros(1, device=dev), "copy": torch.zeros(n, dtype=torch.bfloat16, device=dev) if case["copy"] else None}
    if case["bits"] == 32:
        state.update(m=m, v=v, scales=None)
    else:
        nb = n // BLOCK
        em, ev = _block_exponents(m, v)
        scales = torch.cat([em, ev]).to(torch.uint8).view(2, nb)
        state.update(m=_code_m(m, em), v=_code_v(v, ev, torch.full((nb, BLOCK), 1 << 18, device=dev, dtype=torch.int32)), scales=scales,
                     m_out=torch.zeros(n, device=dev), v_out=torch.zeros(n, device=dev))
    if own:
        from paper_2508_15706_b200.inner import AdamW
        state["opt"] = AdamW([(r, c) for r, c, _ in shapes], offsets, weight_decay=[0.1 if d else 0.0 for _, _, d in shapes], betas=(0.9, 0.95), eps=1e-8,
                             max_norm=case["clip"], state_bits=case["bits"], grad_dtype=DTYPES[case["grad"]])
    return state


def _prepare_norm(case, seed):
    g, dev = _gen(seed, 2), "cuda"
    T, D, act, wt = case["rows"], case["cols"], DTYPES[case["act"]], DTYPES[case["weight"]]

    def rand(*shape, sigma=1.0, mean=0.0, dtype=act):
        return torch.empty(*shape, device=dev).normal_(mean, sigma, generator=g).to(dtype)

    s = {"case": case, "x": rand(T, D, sigma=2.0), "branch": rand(T, D, sigma=0.6), "w": rand(D, mean=1.0, sigma=0.2, dtype=wt), "bw": rand(D, mean=0.6, sigma=0.2, dtype=wt) if case["post"] else None, "eps": 1e-5}
    s["gate"] = {"none": lambda: None, "channel": lambda: rand(D, mean=0.5, sigma=0.3, dtype=wt), "token": lambda: rand(T, 1, mean=0.5, sigma=0.3), "full": lambda: rand(T, D, mean=0.5, sigma=0.3)}[case["gate"]]()
    if case["backward"]:
        # the forward pass left the new residual y (in x's place) and the reciprocal norms
        s["rstd"] = torch.rsqrt(s["x"].float().square().mean(1) + s["eps"])
        s["brstd"] = torch.rsqrt(s["branch"].float().square().mean(1) + s["eps"]) if case["post"] else None
        s["dy"], s["dh"] = rand(T, D, sigma=1e-2), rand(T, D, sigma=1e-2)
        s["out"] = [torch.empty_like(s["x"]), torch.empty_like(s["branch"]), torch.empty_like(s["w"]), None if s["bw"] is None else torch.empty_like(s["bw"]), None if s["gate"] is None else torch.empty_like(s["gate"])]
        if own:
            from paper_2508_15706_b200.inner import norm_backward_workspace
            s["workspace"] = norm_backward_workspace(T, D, dtype=act)
    else:
        s["out"] = [torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(T, device=dev), torch.empty(T, device=dev) if case["post"] else None]
    return s


def _frequencies(case):
    """Radians per position of every pair, and the factor on the rotated values."""
    n, base = case["rot"] // 2, 500000.0
    f = [base ** (-2.0 * i / case["rot"]) for i in range(n)]
    if case["scaling"] == "linear":
        return [x / 8.0 for x in f], 1.0
    if case["scaling"] == "by_parts":  # slow pairs stretched 8 times, fast ones kept, a ramp in turns over 8192 positions between
        keep = [min(1.0, max(0.0, (8192.0 * x / (2.0 * math.pi) - 1.0) / (32.0 - 1.0))) for x in f]
        return [x * k + x / 8.0 * (1.0 - k) for x, k in zip(f, keep)], 0.1 * math.log(8.0) + 1.0
    return f, 1.0


def _prepare_rotary(case, seed):
    g, dev = _gen(seed, 3), "cuda"
    B, S, hq, hk, hd = case["batch"], case["seq"], case["q_heads"], case["k_heads"], case["head_dim"]
    qkv = torch.empty(B, S, hq + 2 * hk, hd, device=dev).normal_(0.0, 1.0, generator=g).to(DTYPES[case["act"]])
    start = torch.randint(0, S + 1, (B, 1), generator=g, device=dev)
    pos = torch.arange(S, device=dev).view(1, S)
    # a sequence of its own that ends inside the row and another that begins there; or sequences far into their context
    pos = torch.where(pos < start, pos, pos - start) if not case["far"] else case["far"] - torch.randint(0, 1 + case["far"] // 2, (B, 1), generator=g, device=dev) + pos
    f, mag = _frequencies(case)
    s = {"case": case, "q": qkv[:, :, :hq], "k": qkv[:, :, hq:hq + hk], "pos": pos.contiguous(), "freq": torch.tensor(f, dtype=torch.float64, device=dev), "mag": mag,
         "out": [torch.empty(B, S, hq, hd, device=dev, dtype=qkv.dtype), torch.empty(B, S, hk, hd, device=dev, dtype=qkv.dtype)]}
    if own:
        from paper_2508_15706_b200.inner import Rotary
        s["rope"] = Rotary(case["rot"], base=500000.0, layout=case["layout"], scaling=case["scaling"], factor=8.0, original_length=8192, low_turns=1.0, high_turns=32.0, magnitude=mag)
    return s


def _prepare_loss(case, seed):
    g, dev = _gen(seed, 4), "cuda"
    T, V = case["rows"], case["vocab"]
    logits = torch.empty(T, V, device=dev).normal_(0.0, 2.0, generator=g)
    targets = torch.randint(0, V - case["masked"], (T,), generator=g, device=dev)
    logits.scatter_add_(1, targets.view(T, 1), torch.full((T, 1), 6.0, device=dev))  # a model that has learned something
    if case["masked"]:
        logits[:, V - case["masked"]:] = float("-inf")  # a vocabulary padded to a round number
    logits = logits.to(DTYPES[case["act"]])
    drop = torch.rand(T, generator=g, device=dev) < case["ignored"]
    drop[0] = False
    targets[drop] = -100
    s = {"case": case, "logits": logits, "targets": targets, "grad": torch.empty_like(logits), "out": [torch.empty(T, device=dev), torch.empty(T, device=dev), torch.empty(1, device=dev)]}
    if own:
        from paper_2508_15706_b200.inner import loss_workspace
        s["workspace"] = loss_workspace()
    return s


# ---------------------------------------------------------------------------------------------------------- plain forms
def run(state):
    return {"adamw": _run_adamw, "norm": _run_norm, "rotary": _run_rotary, "loss": _run_loss}[state["case"]["op"]](state)


def _mix(x):
    """A 32-bit integer hash (two multiplications, three shifts) on int64 tensors or Python integers."""
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & M32
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & M32
    return x ^ (x >> 16)


def _block_exponents(m, v):
    """Scale byte of every block: 2^(byte - 127) brings the block's largest |m| to at most 448, its largest v to at most
    31/16, the largest code's value (so that no rounding of v is cut off)."""
    top = torch.where(torch.isfinite(m), m.abs(), torch.zeros_like(m)).view(-1, BLOCK).amax(1).view(torch.int32)
    em = ((top >> 23) + ((top & 0x7FFFFF) > 0x600000).int() - 8).clamp(min=1)
    top = torch.where(torch.isfinite(v), v, torch.zeros_like(v)).view(-1, BLOCK).amax(1).view(torch.int32)
    return em, ((top >> 23) + ((top & 0x7FFFFF) > 0x780000).int()).clamp(min=1, max=254)


def _code_m(m, em):
    """First moment in float8 (4 exponent, 3 mantissa bits), nearest even."""
    inv = ((254 - em) << 23).view(torch.float32).view(-1, 1)
    return (m.view(-1, BLOCK) * inv).to(torch.float8_e4m3fn).view(torch.uint8).view(-1)


def _code_v(v, ev, bits19):
    """Second moment in an unsigned float of 4 exponent and 4 mantissa bits, rounded up with the probability of the
    remainder by 19 random bits; only an exact zero is coded 0."""
    inv = ((254 - ev) << 23).clamp(min=1 << 22).view(torch.float32).view(-1, 1)  # (2^-127 is no normal number)
    s = v.view(-1, BLOCK) * inv
    fine = torch.isfinite(s)
    c = ((torch.where(fine, s, torch.zeros_like(s)).view(torch.int32) + bits19) >> 19) - 1792
    c = torch.where(fine, c.clamp(1, 255), torch.full_like(c, 255))
    return torch.where(s == 0, torch.zeros_like(c), c).to(torch.uint8).view(-1)


def _value_m(code, em):
    return (code.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * (em.int() << 23).view(torch.float32).view(-1, 1)).view(-1)


def _value_v(code, ev):
    c = code.int().view(-1, BLOCK)
    s = torch.where(c == 0, torch.zeros_like(c), (c + 1792) << 19).view(torch.float32)
    return (s * (ev.int() << 23).view(torch.float32).view(-1, 1)).view(-1)


def _run_adamw(s):
    case, b1, b2, eps, t, lr = s["case"], 0.9, 0.95, 1e-8, s["t"], s["lr"]
    if own:
        s["opt"].step(s["theta"], s["grad"], s["m"], s["v"], s["scales"], step=t, lr=lr, seed=s["seed"], copy=s["copy"], norm=s["norm"])
        if case["bits"] == 32:
            return [s["theta"], s["m"], s["v"], s["norm"], s["copy"]]
        s["opt"].read_state(s["m"], s["v"], s["scales"], s["m_out"], s["v_out"])
        return [s["theta"], s["m_out"], s["v_out"], s["norm"], s["copy"]]
    g = s["grad"].float()
    norm = torch.sqrt(torch.sum(torch.square(g.double())))
    ok = torch.isfinite(norm)
    if case["clip"]:
        g = g * torch.clamp(case["clip"] / (norm + 1e-6), max=1.0).float()
    if case["bits"] == 32:
        m0, v0 = s["m"], s["v"]
    else:
        m0, v0 = _value_m(s["m"], s["scales"][0]), _value_v(s["v"], s["scales"][1])
    m = m0 * b1 + g * (1 - b1)
    v = v0 * b2 + (g * g) * (1 - b2)
    denom = torch.sqrt(v) * (1.0 / math.sqrt(1 - b2 ** t)) + eps
    p = s["theta"].view(-1, BLOCK)
    p = (p - p * (lr * s["decay"])).view(-1) - (lr / (1 - b1 ** t)) * (m / denom)
    s["theta"].copy_(torch.where(ok, p, s["theta"]))
    s["norm"].copy_(norm.float())
    if s["copy"] is not None:
        s["copy"].copy_(s["theta"])
    if case["bits"] == 32:
        s["m"].copy_(torch.where(ok, m, m0))
        s["v"].copy_(torch.where(ok, v, v0))
        return [s["theta"], s["m"], s["v"], s["norm"], s["copy"]]
    em, ev = _block_exponents(m, v)
    index = torch.arange(g.numel(), device=g.device)
    bits19 = (_mix(index ^ _mix(s["seed"])) >> 13).int().view(-1, BLOCK)
    s["m"].copy_(torch.where(ok, _code_m(m, em), s["m"]))
    s["v"].copy_(torch.where(ok, _code_v(v, ev, bits19), s["v"]))
    s["scales"].copy_(torch.where(ok, torch.stack([em, ev]).to(torch.uint8), s["scales"]))
    return [s["theta"], _value_m(s["m"], s["scales"][0]), _value_v(s["v"], s["scales"][1]), s["norm"], s["copy"]]


def _run_norm(s):
    case, a, eps = s["case"], s["case"]["alpha"], s["eps"]
    if own:
        from paper_2508_15706_b200 import inner
        o = s["out"]
        if case["backward"]:
            inner.norm_backward(s["dy"], s["dh"], s["x"], s["w"], rstd=s["rstd"], branch=s["branch"], branch_weight=s["bw"], branch_rstd=s["brstd"], gate=s["gate"], alpha=a,
                                dx=o[0], dbranch=o[1], dweight=o[2], dbranch_weight=o[3], dgate=o[4], workspace=s["workspace"])
        else:
            inner.norm_forward(s["x"], s["w"], branch=s["branch"], branch_weight=s["bw"], gate=s["gate"], alpha=a, eps=eps, y=o[0], h=o[1], rstd=o[2], branch_rstd=o[3])
        return list(o)
    x, b, w = s["x"].float(), s["branch"].float(), s["w"].float()
    bw = None if s["bw"] is None else s["bw"].float()
    gate = 1.0 if s["gate"] is None else s["gate"].float()
    if not case["backward"]:
        br = None
        if bw is not None:
            br = torch.rsqrt(torch.mean(b * b, 1) + eps)
            b = b * br.view(-1, 1) * bw
        y = x + a * (gate * b)
        r = torch.rsqrt(torch.mean(y * y, 1) + eps)
        return [y.to(s["x"].dtype), (y * r.view(-1, 1) * w).to(s["x"].dtype), r, br]
    # gradients: `x` holds the y of the forward pass
    r, dh = s["rstd"].view(-1, 1), s["dh"].float()
    hat, dhw = x * r, dh * w
    dx = s["dy"].float() + r * (dhw - hat * torch.mean(dhw * hat, 1, keepdim=True))
    dw = torch.sum(dh * hat, 0)
    dz = a * dx
    z = b
    if bw is not None:
        br = s["brstd"].view(-1, 1)
        bhat = b * br
        z = bhat * bw
    dgate = None
    if case["gate"] == "channel":
        dgate = torch.sum(dz * z, 0)
    elif case["gate"] == "token":
        dgate = torch.sum(dz * z, 1, keepdim=True)
    elif case["gate"] == "full":
        dgate = dz * z
    dz = dz * gate
    dbw, db = None, dz
    if bw is not None:
        dbw = torch.sum(dz * bhat, 0).to(s["bw"].dtype)
        q = dz * bw
        db = br * (q - bhat * torch.mean(q * bhat, 1, keepdim=True))
    return [dx.to(s["x"].dtype), db.to(s["x"].dtype), dw.to(s["w"].dtype), dbw, None if dgate is None else dgate.to(s["gate"].dtype)]


def _run_rotary(s):
    case, rot = s["case"], s["case"]["rot"]
    if own:
        s["rope"].apply(s["q"], s["k"], s["pos"], inverse=case["inverse"], out_q=s["out"][0], out_k=s["out"][1])
        return list(s["out"])
    angle = s["pos"].double().view(case["batch"], case["seq"], 1) * s["freq"]  # far positions need more than 24 bits
    c, n = (torch.cos(angle) * s["mag"]).float().unsqueeze(2), (torch.sin(angle) * s["mag"]).float().unsqueeze(2)
    n = -n if case["inverse"] else n
    return [_turned(s["q"], c, n, rot, case["layout"]), _turned(s["k"], c, n, rot, case["layout"])]


def _turned(x, c, n, rot, layout):
    u = x[..., :rot].float()
    if layout == "half":
        a, b = u[..., :rot // 2], u[..., rot // 2:]
        u = torch.cat([a * c - b * n, b * c + a * n], -1)
    else:
        a, b = u[..., 0::2], u[..., 1::2]
        u = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    return torch.cat([u.to(x.dtype), x[..., rot:]], -1)


def _run_loss(s):
    case, eps, z = s["case"], s["case"]["smoothing"], s["case"]["z"]
    if own:
        from paper_2508_15706_b200 import inner
        inner.token_loss(s["logits"], s["targets"], grad=s["grad"], ignore_index=-100, smoothing=eps, z=z, row_loss=s["out"][0], lse=s["out"][1], total=s["out"][2], workspace=s["workspace"])
        return [s["grad"], *s["out"]]
    x, t = s["logits"].float(), s["targets"]
    valid = t != -100
    n = torch.sum(valid).float()
    at = torch.where(valid, t, torch.zeros_like(t)).view(-1, 1)
    top = torch.amax(x, 1, keepdim=True)
    e = torch.exp(x - top)
    total = torch.sum(e, 1, keepdim=True)
    lse = top + torch.log(total)
    loss = lse - (1 - eps) * x.gather(1, at) + z * lse * lse
    if eps:
        loss = loss - eps * torch.mean(x, 1, keepdim=True)
    loss = torch.where(valid, loss.view(-1), torch.zeros_like(n))
    grad = (e / total) * (1 + 2 * z * lse) - eps / x.shape[1]
    grad = grad.scatter_add(1, at, torch.full_like(lse, eps - 1.0))
    grad = torch.where(valid.view(-1, 1), grad / n, torch.zeros_like(n))
    return [grad.to(s["logits"].dtype), loss, lse.view(-1), (torch.sum(loss) / n).view(1)]


# ------------------------------------------------------------------------------------------------------------------ work
def work(case):
    if case["op"] == "adamw":
        n = sum(r * c for r, c, _ in _shapes(case))
        g = 4 if case["grad"] == "fp32" else 2
        moments = 16 if case["bits"] == 32 else 4 + 4.0 / BLOCK + 8  # 8 bits: codes and scales in and out, the values once out
        return {"bytes": n * (8 + g + moments + (2 if case["copy"] else 0)), "flops": 16 * n}
    a = 4 if case.get("act") == "fp32" else 2
    if case["op"] == "norm":
        n, w = case["rows"] * case["cols"], 4 if case["weight"] == "fp32" else 2
        vectors = 1 + (1 if case["post"] else 0) + (1 if case["gate"] == "channel" else 0)
        full = 1 if case["gate"] == "full" else 0
        stats = 4 * case["rows"] * (2 if case["post"] else 1) + (a * case["rows"] if case["gate"] == "token" else 0)
        if case["backward"]:
            return {"bytes": a * n * (6 + 2 * full) + 2 * w * vectors * case["cols"] + stats, "flops": 25 * n}
        return {"bytes": a * n * (4 + full) + w * vectors * case["cols"] + stats, "flops": 10 * n}
    if case["op"] == "rotary":
        rows = case["batch"] * case["seq"]
        n = rows * (case["q_heads"] + case["k_heads"]) * case["head_dim"]
        return {"bytes": 2 * a * n + 8 * rows, "flops": 3 * n}
    n = case["rows"] * case["vocab"]
    return {"bytes": 2 * a * n + 16 * case["rows"], "flops": 6 * n}


# --------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"adamw": _exact_adamw, "norm": _exact_norm, "rotary": _exact_rotary, "loss": _exact_loss}[case["op"]](s)


def _exact_adamw(s):
    case, b1, b2, t = s["case"], 0.9, 0.95, s["t"]
    g = s["grad"].double()
    norm = g.norm()
    g = g * min(1.0, case["clip"] / (norm.item() + 1e-6)) if case["clip"] else g
    if case["bits"] == 32:
        m0, v0 = s["m"].double(), s["v"].double()
    else:
        scale = torch.exp2(s["scales"].double() - 127.0)
        c = s["m"].double()
        sign, e, f = torch.where(c >= 128, -1.0, 1.0), torch.floor(c % 128 / 8), c % 8
        m0 = (sign * torch.where(e == 0, f * 2.0 ** -9, torch.exp2(e - 7) * (1 + f / 8))).view(-1, BLOCK) * scale[0].view(-1, 1)
        c = s["v"].double()
        v0 = torch.where(c == 0, 0.0, torch.exp2(torch.floor(c / 16) - 15) * (1 + c % 16 / 16)).view(-1, BLOCK) * scale[1].view(-1, 1)
        m0, v0 = m0.view(-1), v0.view(-1)
    m = b1 * m0 + (1 - b1) * g
    v = b2 * v0 + (1 - b2) * g ** 2
    p = s["theta"].double() * (1 - s["lr"] * s["decay"].double()).expand(-1, BLOCK).reshape(-1)
    p = p - s["lr"] * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + 1e-8)
    copy = p if case["copy"] else None
    if case["bits"] == 32:
        return [p, m, v, norm.view(1), copy]
    m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
    # first moment: largest |m| of the block in (224, 448], then the nearest multiple of the step at its size, halves to even
    top = m.abs().amax(1, keepdim=True)
    k = torch.ceil(torch.log2(top / 448.0)).clamp(min=-126.0)
    k = torch.where(top > 0, k, torch.full_like(k, -126.0))
    x = m * torch.exp2(-k)
    step = torch.exp2(torch.floor(torch.log2(x.abs())).clamp(min=-6.0) - 3)
    mq = torch.where(x == 0, x, torch.round(x / step) * step) * torch.exp2(k)
    # second moment: steps of 1/16 of a power of two, up with the probability of the remainder, kept within 255 codes
    top = v.amax(1, keepdim=True)
    k = torch.floor(torch.log2(top))
    k = k + (top * torch.exp2(-k) > 1.9375)
    k = torch.where(torch.isfinite(k), k, torch.full_like(k, -126.0)).clamp(-126.0, 127.0)
    x = v * torch.exp2(-k)
    e = torch.floor(torch.log2(x))
    place = torch.where(x > 0, 16 * (e + 15) + 16 * (x * torch.exp2(-e) - 1), torch.zeros_like(x))
    lot = _mix(torch.arange(x.numel(), device=x.device) ^ _mix(s["seed"])) >> 13
    code = torch.floor(place + lot.double().view(-1, BLOCK) / 2.0 ** 19).clamp(1, 255)
    vq = torch.where(x > 0, torch.exp2(torch.floor(code / 16) - 15) * (1 + code % 16 / 16), 0.0) * torch.exp2(k)
    return [p, mq.view(-1), vq.view(-1), norm.view(1), copy]


def _exact_norm(s):
    case = s["case"]
    x, b, w = s["x"].double(), s["branch"].double(), s["w"].double()
    bw = s["bw"].double() if case["post"] else None
    gate = s["gate"].double() if s["gate"] is not None else None
    if not case["backward"]:
        br = None
        z = b
        if case["post"]:
            br = (b.pow(2).mean(1) + s["eps"]).pow(-0.5)
            z = br[:, None] * b * bw
        y = x + case["alpha"] * (z if gate is None else gate * z)
        r = (y.pow(2).mean(1) + s["eps"]).pow(-0.5)
        return [y, r[:, None] * y * w, r, br]
    # the vector-Jacobian products of y -> rstd-normalised y and of branch -> y, written row by row with projections
    D = x.shape[1]
    r, dh, dy = s["rstd"].double()[:, None], s["dh"].double(), s["dy"].double()
    u = dh * w
    dx = dy + r * u - r ** 3 * x * (u * x).sum(1, keepdim=True) / D
    dw = (dh * x * r).sum(0)
    if case["post"]:
        br = s["brstd"].double()[:, None]
        z = b * br * bw
    else:
        z = b
    up = case["alpha"] * dx
    dgate = None if gate is None else {"channel": lambda: (up * z).sum(0), "token": lambda: (up * z).sum(1, keepdim=True), "full": lambda: up * z}[case["gate"]]()
    dz = up if gate is None else up * gate
    if not case["post"]:
        return [dx, dz, dw, None, dgate]
    db = br * bw * dz - br ** 3 * b * (bw * dz * b).sum(1, keepdim=True) / D
    return [dx, db, dw, (dz * b * br).sum(0), dgate]


def _exact_rotary(s):
    case, rot = s["case"], s["case"]["rot"]
    turn = torch.exp(1j * (s["pos"].double()[:, :, None, None] * s["freq"]) * (-1.0 if case["inverse"] else 1.0)) * s["mag"]

    def one(x):
        x = x.double()
        u = x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["layout"] == "half" else x[..., :rot].unflatten(-1, (rot // 2, 2))
        u = torch.view_as_real(torch.view_as_complex(u.contiguous()) * turn)
        u = u.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else u.flatten(-2)
        return torch.cat([u, x[..., rot:]], -1)

    return [one(s["q"]), one(s["k"])]


def _exact_loss(s):
    case, eps, z = s["case"], s["case"]["smoothing"], s["case"]["z"]
    x, t = s["logits"].double(), s["targets"]
    rows = torch.arange(x.shape[0], device=x.device)
    keep = t >= 0
    n = int(keep.sum())
    lse = torch.logsumexp(x, 1)
    hit = torch.zeros_like(x)
    hit[rows[keep], t[keep]] = 1.0 - eps
    wanted = (hit + eps / x.shape[1]) * keep[:, None]
    loss = (lse + z * lse ** 2) * keep - torch.where(wanted > 0, wanted * x, 0.0).sum(1)
    grad = (torch.exp(x - lse[:, None]) * (1 + 2 * z * lse[:, None]) * keep[:, None] - wanted) / n
    return [grad, loss, lse, (loss.sum() / n).view(1)]
