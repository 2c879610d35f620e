"""The operators of the inner phase together: a small decoder's gradients against the same decoder in plain torch, and the whole
of Algorithm 1 (local AdamW steps, compressed outer step) on synthetic sequences."""
import os
import sys

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain_logits(p, tokens, layers, heads, rot_base=10000.0):
    """The decoder in fp64 torch operations."""
    x = p["embed"][tokens]
    B, S, d = x.shape
    hd = d // heads

    def norm(v, w):
        return v * (v.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w.view(-1)

    def turn(v):
        f = rot_base ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64, device=v.device) / hd)
        a = torch.arange(S, dtype=torch.float64, device=v.device)[:, None] * f
        c, s = a.cos()[:, None], a.sin()[:, None]
        u, w = v[..., :hd // 2], v[..., hd // 2:]
        return torch.cat([u * c - w * s, w * c + u * s], -1)

    mask = torch.ones(S, S, dtype=torch.bool, device=x.device).tril()
    for l in range(layers):
        h = norm(x, p[f"l{l}.norm1"])
        q, k, v = ((h @ p[f"l{l}.{n}"].t()).view(B, S, heads, hd) for n in "qkv")
        q, k = turn(q), turn(k)
        s = torch.einsum("bihd,bjhd->bhij", q, k) / hd ** 0.5
        a = torch.einsum("bhij,bjhd->bihd", s.masked_fill(~mask, float("-inf")).softmax(-1), v).reshape(B, S, d)
        x = x + a @ p[f"l{l}.o"].t()
        h = norm(x, p[f"l{l}.norm2"])
        x = x + (F.silu(h @ p[f"l{l}.gate"].t()) * (h @ p[f"l{l}.up"].t())) @ p[f"l{l}.down"].t()
    return norm(x, p["final_norm"]) @ p["lm_head"].t()


def test_decoder_gradients_against_plain_torch():
    """fp32 parameters and activations; what differs from fp64 are fp32 products (torch's, a few 1e-6 of their size) through two
    layers: 1e-4 of every gradient's norm is a bound with room and far below what a wrong term would do."""
    from local_steps import Decoder
    from paper_2508_15706_b200 import inputs as I
    specs = I.dense_transformer(64, 2, 160, 203)
    g = torch.Generator(device="cuda").manual_seed(4)
    leaf, ref = {}, {}
    for t in specs:
        w = torch.randn(t.rows, t.cols, generator=g, device="cuda") * (0.15 if t.rows > 1 else 0.1) + (0.0 if t.rows > 1 else 1.0)
        leaf[t.name], ref[t.name] = w.clone().requires_grad_(), w.double().requires_grad_()
    tokens = torch.randint(0, 203, (3, 38), generator=g, device="cuda")
    model = Decoder(64, 2, 4)
    loss = model.loss(leaf, tokens)
    loss.backward()
    x = plain_logits(ref, tokens[:, :-1], 2, 4)
    lse = torch.logsumexp(x, -1)
    want = (lse - x.gather(-1, tokens[:, 1:, None])[..., 0] + 1e-4 * lse ** 2).mean()
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * abs(want.item())
    for name in leaf:
        d = (leaf[name].grad.double() - ref[name].grad).norm() / ref[name].grad.norm()
        assert d <= 1e-4, (name, d.item())


@pytest.mark.parametrize("bits", [32, 8])
def test_local_steps_and_outer_steps_learn(bits):
    from local_steps import train
    history, theta = train(R=2, outer=4, inner_steps=12, bits=bits, say=lambda *_: None)
    assert torch.all(torch.isfinite(theta))
    assert history[0] > 4.0 and history[-1] < 0.75 * history[0], history
    again, theta2 = train(R=2, outer=1, inner_steps=3, bits=bits, say=lambda *_: None)
    assert all(torch.isfinite(torch.tensor(again)))
