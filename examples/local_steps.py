"""SparseLoCo end to end on one GPU: R workers, each taking H local AdamW steps on a small decoder (the inner phase), then the
compressed outer step (Algorithm 1).

    python examples/local_steps.py [--bits 8] [--outer 6] [--inner 15]

Parameters live in the flat buffers of the tensor table throughout: theta_local[r] is what AdamW updates and what the outer step
reads; the model runs on a bfloat16 working copy that AdamW writes alongside, and autograd accumulates into views of one flat
bfloat16 gradient.  Norms, rotary positions and the loss are the library's; matrix products and attention are torch's.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2508_15706_b200 import inputs as I  # noqa: E402
from paper_2508_15706_b200 import inner  # noqa: E402
from paper_2508_15706_b200.binding import SparseLoCo  # noqa: E402


class Decoder:
    """LLaMA-style decoder over named parameter tensors (the names of `inputs.dense_transformer`)."""

    def __init__(self, d_model: int, n_layers: int, heads: int, scaling: str = "none"):
        self.layers, self.heads = n_layers, heads
        self.rope = inner.Rotary(d_model // heads, base=10000.0, scaling=scaling, factor=4.0 if scaling != "none" else 1.0, original_length=256)

    def logits(self, p, tokens):
        batch, seq = tokens.shape
        x = F.embedding(tokens, p["embed"])
        branch = None
        for l in range(self.layers):
            # the residual update of the block before and this block's norm are one operator
            x, h = inner.block_norm(x, p[f"l{l}.norm1"].view(-1), branch=branch)
            q, k, v = (F.linear(h, p[f"l{l}.{n}"]).view(batch, seq, -1, x.shape[-1] // self.heads) for n in "qkv")
            q, k = inner.rotary(self.rope, q, k)
            a = F.scaled_dot_product_attention(q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2), is_causal=True, enable_gqa=q.shape[2] != k.shape[2])
            branch = F.linear(a.transpose(1, 2).reshape(batch, seq, -1), p[f"l{l}.o"])
            x, h = inner.block_norm(x, p[f"l{l}.norm2"].view(-1), branch=branch)
            branch = F.linear(F.silu(F.linear(h, p[f"l{l}.gate"])) * F.linear(h, p[f"l{l}.up"]), p[f"l{l}.down"])
        _, h = inner.block_norm(x, p["final_norm"].view(-1), branch=branch)
        return F.linear(h, p["lm_head"])

    def loss(self, p, tokens):
        logits = self.logits(p, tokens[:, :-1])
        return inner.next_token_loss(logits, tokens[:, 1:], z=1e-4)


class Worker:
    """One worker's state: fp32 parameters, their bfloat16 copy, one flat gradient, the moments."""

    def __init__(self, specs, offsets, theta, bits: int):
        self.opt = inner.AdamW([(t.rows, t.cols) for t in specs], offsets, weight_decay=[0.1 if t.rows > 1 else 0.0 for t in specs], betas=(0.9, 0.95), max_norm=1.0, state_bits=bits,
                               grad_dtype=torch.bfloat16)
        self.theta, self.copy = theta.clone(), theta.bfloat16()
        self.grad, self.norm = torch.zeros_like(self.copy), torch.zeros(1, device=theta.device)
        self.moments, self.t = self.opt.new_state(), 0
        self.params = {}
        for t, off in zip(specs, offsets):
            s = slice(off, off + t.numel)
            w = self.copy[s].view(t.rows, t.cols).detach().requires_grad_()
            w.grad = self.grad[s].view(t.rows, t.cols)
            self.params[t.name] = w

    def receive(self, theta):
        """The synchronised parameters, after an outer step."""
        self.theta.copy_(theta)
        self.copy.copy_(theta)

    def step(self, model, tokens, lr: float):
        self.t += 1
        self.grad.zero_()
        loss = model.loss(self.params, tokens)
        loss.backward()
        self.opt.step(self.theta, self.grad, *self.moments, step=self.t, lr=lr, copy=self.copy, norm=self.norm)
        return loss.detach()


def batches(n, batch, seq, vocab, seed, device):
    """Sequences with something to learn: the next token follows from the last one, one time in eight at random."""
    g = torch.Generator(device=device).manual_seed(seed)
    for _ in range(n):
        t = torch.randint(0, vocab, (batch, seq + 1), generator=g, device=device)
        noise = torch.rand(batch, seq + 1, generator=g, device=device) < 0.125
        for i in range(1, seq + 1):
            t[:, i] = torch.where(noise[:, i], t[:, i], (t[:, i - 1] * 7 + 3) % vocab)
        yield t


def train(R=4, outer=6, inner_steps=15, bits=32, d_model=256, n_layers=2, ffn=512, vocab=512, heads=4, batch=8, seq=64, lr=2e-3, k=64, device="cuda", say=print):
    specs = I.dense_transformer(d_model, n_layers, ffn, vocab)
    offsets = I.offsets(specs, align=64)
    g = torch.Generator(device=device).manual_seed(0)
    theta = torch.zeros(I.flat_numel(specs, align=64), device=device)
    for t, off in zip(specs, offsets):
        theta[off:off + t.numel] = torch.empty(t.numel, device=device).normal_(0.0, 0.02, generator=g) if t.rows > 1 else 1.0
    model = Decoder(d_model, n_layers, heads)
    sl = SparseLoCo([(t.rows, t.cols) for t in specs], offsets, k=k, R=R, H=inner_steps, beta=0.95, outer_lr=1.0)
    workers = [Worker(specs, offsets, theta, bits) for _ in range(R)]
    e = [torch.zeros_like(theta) for _ in range(R)]
    payloads = [torch.zeros(sl.payload_bytes(), dtype=torch.uint8, device=device) for _ in range(R)]
    history = []
    for o in range(outer):
        losses = []
        for r, w in enumerate(workers):
            w.receive(theta)
            losses += [w.step(model, tokens, lr) for tokens in batches(inner_steps, batch, seq, vocab, 1000 * r + o, device)]
        sl.outer_step(theta, [w.theta for w in workers], e, payloads)
        history.append(torch.stack(losses).mean().item())
        say(f"outer step {o}: mean loss of {R} x {inner_steps} local steps {history[-1]:.3f}, gradient norm {workers[0].norm.item():.3f}, payload {sl.payload_bytes()} of {4 * theta.numel()} bytes")
    return history, theta


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--outer", type=int, default=6)
    ap.add_argument("--inner", type=int, default=15)
    ap.add_argument("--bits", type=int, default=32, choices=(8, 32))
    a = ap.parse_args()
    train(R=a.workers, outer=a.outer, inner_steps=a.inner, bits=a.bits)
