"""The inner phase (Algorithm 1, a worker's H local steps): AdamW over the tensor table, the norms around a block, rotary
positions and the next-token loss.  Wrappers over libsparseloco's C entry points (include/sparseloco.h has the formulas).

Two layers.  `AdamW`, `Rotary`, `norm_forward` / `norm_backward` and `token_loss` marshal arguments only: buffers are the
caller's (allocated here where an output is left out), work goes on torch's current stream, nothing synchronises.
`block_norm`, `rotary` and `next_token_loss` are the same operators as autograd functions, for a model that runs under
torch's autograd.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from .binding import SlError, SL_ERR_INVALID_ARG, _check, _L, _stream, _TensorDesc

P, I32, I64, F32, F64 = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_double
DTYPES = {torch.float32: 0, torch.bfloat16: 1}
GATES = {"none": 0, "column": 1, "row": 2, "full": 3}
LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "base": 2, "by_parts": 3}


class _AdamWConfig(C.Structure):
    _fields_ = [("param_dtype", I32), ("grad_dtype", I32), ("state_bits", I32), ("skip_nonfinite", I32), ("beta1", F64), ("beta2", F64), ("eps", F64), ("max_norm", F64)]


class _NormDesc(C.Structure):
    _fields_ = [("rows", I64), ("cols", I64), ("dtype", I32), ("weight_dtype", I32), ("gate_kind", I32), ("alpha", F32), ("eps", F32),
                ("ld_x", I64), ("ld_branch", I64), ("ld_gate", I64), ("ld_y", I64), ("ld_h", I64), ("ld_dy", I64), ("ld_dh", I64)]


class _RotaryConfig(C.Structure):
    _fields_ = [("rot_dim", I32), ("layout", I32), ("scaling", I32), ("base", F64), ("factor", F64), ("original_length", F64), ("low_turns", F64), ("high_turns", F64), ("magnitude", F64)]


class _RotaryHeads(C.Structure):
    _fields_ = [("inp", P), ("out", P), ("heads", I64), ("in_batch", I64), ("in_token", I64), ("in_head", I64), ("out_batch", I64), ("out_token", I64), ("out_head", I64)]


class _RotaryDesc(C.Structure):
    _fields_ = [("dtype", I32), ("position_bits", I32), ("inverse", I32), ("batch", I64), ("seq", I64), ("head_dim", I64), ("first", I64), ("pos_batch", I64), ("pos_token", I64)]


class _LossDesc(C.Structure):
    _fields_ = [("rows", I64), ("vocab", I64), ("dtype", I32), ("target_bits", I32), ("ld_logits", I64), ("ld_grad", I64), ("ignore_index", I64), ("smoothing", F32), ("z", F32), ("scale", F32), ("mean", I32)]


_L.sl_adamw_create.argtypes = [P, P, P, I32, C.POINTER(P)]
_L.sl_adamw_destroy.argtypes = [P]
_L.sl_adamw_sizes.argtypes = [P, C.POINTER(I64), C.POINTER(I64)]
_L.sl_adamw_step.argtypes = [P, P, P, P, P, P, P, P, I64, F64, F64, C.c_uint32, P]
_L.sl_adamw_read_state.argtypes = [P, P, P, P, P, P, P]
_L.sl_adamw_write_state.argtypes = [P, P, P, P, P, P, C.c_uint32, P]
_L.sl_norm_forward.argtypes = [P] * 11
_L.sl_norm_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
_L.sl_norm_backward.argtypes = [P] * 16 + [C.c_size_t, P]
_L.sl_rotary_create.argtypes = [P, C.POINTER(P)]
_L.sl_rotary_destroy.argtypes = [P]
_L.sl_rotary_apply.argtypes = [P, P, P, P, P, P]
_L.sl_loss_workspace_bytes.restype = C.c_size_t
_L.sl_token_loss.argtypes = [P] * 8 + [C.c_size_t, P]


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise SlError(SL_ERR_INVALID_ARG, f"libsparseloco: {what}")


def _dtype(t: torch.dtype) -> int:
    _need(t in DTYPES, f"{t} is not one of float32, bfloat16")
    return DTYPES[t]


def _ptr(t: Optional[torch.Tensor], dtype=None, numel: Optional[int] = None, what: str = "tensor") -> Optional[int]:
    """Address of a contiguous tensor on the current device."""
    if t is None:
        return None
    _need(t.is_cuda and t.is_contiguous(), f"{what} must be a contiguous CUDA tensor")
    _need(dtype is None or t.dtype == dtype, f"{what} must be {dtype}, got {t.dtype}")
    _need(numel is None or t.numel() >= numel, f"{what} has {t.numel()} elements, {numel} are needed")
    return t.data_ptr()


def _rows(t: Optional[torch.Tensor], rows: int, cols: int, dtype, what: str):
    """(address, row stride) of a [rows, cols] matrix with a unit column stride."""
    if t is None:
        return None, 0
    _need(t.is_cuda and t.dtype == dtype, f"{what} must be a CUDA tensor of {dtype}")
    _need(t.dim() == 2 and t.shape[0] == rows and t.shape[1] == cols, f"{what} must be [{rows}, {cols}], got {tuple(t.shape)}")
    _need(t.stride(1) == 1 or cols == 1, f"{what} must have a unit column stride")
    _need(rows <= 1 or t.stride(0) >= cols, f"{what}: rows overlap")
    return t.data_ptr(), t.stride(0) if rows > 1 else cols


class AdamW:
    """AdamW over a tensor table (shapes and element offsets as for `SparseLoCo`), gradients clipped by their global norm.

    Parameters, gradients and moments are flat buffers of one layout: let every parameter's `.grad` be a view of the flat
    gradient, and theta_local[r] of the outer step is the very buffer that `step` updates.  `state_bits=8` keeps the moments
    in 8-bit codes with one power-of-two scale per 128 elements: 2 bytes per parameter in place of 8."""

    def __init__(self, shapes: Sequence[Sequence[int]], offsets: Optional[Sequence[int]] = None, *, weight_decay=0.1, betas=(0.9, 0.95),
                 eps: float = 1e-8, max_norm: float = 1.0, state_bits: int = 32, param_dtype=torch.float32, grad_dtype=torch.float32, skip_nonfinite: bool = True):
        n = len(shapes)
        descs, pos = (_TensorDesc * n)(), 0
        for j, sh in enumerate(shapes):
            rows, cols = (1, sh[0]) if len(sh) == 1 else (sh[0], sh[1])
            off = offsets[j] if offsets is not None else (pos + 3) // 4 * 4
            descs[j] = _TensorDesc(rows, cols, off)
            pos = off + rows * cols
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        _need(len(decay) == n, f"{len(decay)} weight decays for {n} tensors")
        cfg = _AdamWConfig(_dtype(param_dtype), _dtype(grad_dtype), state_bits, int(skip_nonfinite), betas[0], betas[1], eps, max_norm)
        self._h = P()
        _check(_L.sl_adamw_create(C.byref(cfg), descs, (F32 * n)(*decay), n, C.byref(self._h)))
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.state_bits, self.param_dtype, self.grad_dtype = state_bits, param_dtype, grad_dtype
        flat, blocks = I64(), I64()
        _check(_L.sl_adamw_sizes(self._h, C.byref(flat), C.byref(blocks)))
        self.flat_elems, self.blocks = flat.value, blocks.value
        self._moment = torch.float32 if state_bits == 32 else torch.uint8

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            _L.sl_adamw_destroy(self._h)
            self._h = P()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def new_state(self):
        """(m, v, scales) of zero moments; scales is None with 32-bit moments."""
        m, v = (torch.zeros(self.flat_elems, dtype=self._moment, device=self.device) for _ in range(2))
        return m, v, None if self.state_bits == 32 else torch.zeros(2, self.blocks, dtype=torch.uint8, device=self.device)

    def _state(self, m, v, scales):
        return (_ptr(m, self._moment, self.flat_elems, "m"), _ptr(v, self._moment, self.flat_elems, "v"),
                _ptr(scales, torch.uint8, 2 * self.blocks, "scales"))

    def step(self, theta, grad, m, v, scales=None, *, step: int, lr: float, grad_scale: float = 1.0, seed: Optional[int] = None, copy=None, norm=None) -> None:
        """One step, in place.  `step` counts from 1; `grad_scale` multiplies the gradient (1 / accumulated micro-batches);
        `copy` receives a bfloat16 copy of the new parameters, `norm` (one fp32) the gradient's norm before clipping;
        `seed` (default: the step) seeds the rounding of an 8-bit second moment."""
        pm, pv, ps = self._state(m, v, scales)
        _check(_L.sl_adamw_step(self._h, _ptr(theta, self.param_dtype, self.flat_elems, "theta"), _ptr(grad, self.grad_dtype, self.flat_elems, "grad"), pm, pv, ps,
                                _ptr(copy, torch.bfloat16, self.flat_elems, "copy"), _ptr(norm, torch.float32, 1, "norm"), step, lr, grad_scale,
                                (step if seed is None else seed) & 0xFFFFFFFF, _stream()))

    def read_state(self, m, v, scales, m_out, v_out) -> None:
        """8-bit moments as fp32 values, in flat buffers of the same layout."""
        pm, pv, ps = self._state(m, v, scales)
        _check(_L.sl_adamw_read_state(self._h, pm, pv, ps, _ptr(m_out, torch.float32, self.flat_elems, "m_out"), _ptr(v_out, torch.float32, self.flat_elems, "v_out"), _stream()))

    def write_state(self, m_in, v_in, m, v, scales, *, seed: int = 0) -> None:
        """fp32 moments into the 8-bit form, rounded as a step rounds them."""
        pm, pv, ps = self._state(m, v, scales)
        _check(_L.sl_adamw_write_state(self._h, _ptr(m_in, torch.float32, self.flat_elems, "m_in"), _ptr(v_in, torch.float32, self.flat_elems, "v_in"), pm, pv, ps,
                                       seed & 0xFFFFFFFF, _stream()))


# ------------------------------------------------------------------------------------------------------------- norms
def _gate(gate, rows, cols, act, wt):
    """(kind, address, stride): [cols] = per column, [rows, 1] or (rows != cols) [rows] = per row, [rows, cols] = per element."""
    if gate is None:
        return GATES["none"], None, 0
    if gate.dim() == 1 and gate.shape[0] == cols:
        return GATES["column"], _ptr(gate, wt, cols, "column gate"), 0
    _need(gate.is_cuda and gate.dtype == act, f"a row or element gate must be a CUDA tensor of {act}")
    if gate.dim() == 1 and gate.shape[0] == rows or gate.dim() == 2 and tuple(gate.shape) == (rows, 1) and cols != 1:
        _need(rows <= 1 or gate.stride(0) >= 1, "a row gate needs a positive stride")
        return GATES["row"], gate.data_ptr(), gate.stride(0) if rows > 1 else 1
    ptr, ld = _rows(gate, rows, cols, act, "element gate")
    return GATES["full"], ptr, ld


def _norm_desc(x, weight, branch_weight, gate, alpha, eps):
    _need(x.dim() == 2, "activations must be [rows, cols]")
    rows, cols = x.shape
    wt = next((w.dtype for w in (weight, branch_weight) if w is not None), gate.dtype if gate is not None and gate.dim() == 1 and gate.shape[0] == cols else torch.float32)
    d = _NormDesc(rows, cols, _dtype(x.dtype), _dtype(wt), 0, alpha, eps)
    d.gate_kind, g, d.ld_gate = _gate(gate, rows, cols, x.dtype, wt)
    return d, rows, cols, wt, g


def norm_forward(x, weight=None, *, branch=None, branch_weight=None, gate=None, alpha: float = 1.0, eps: float = 1e-6, norm: bool = True, y=None, h=None, rstd=None, branch_rstd=None):
    """y = x + alpha * gate * norm(branch) (the norm only with `branch_weight`), h = norm(y) * weight (`norm=False`: no h).
    Returns (y, h, rstd, branch_rstd); y is x itself without a branch.  Outputs left out are allocated."""
    d, rows, cols, wt, g = _norm_desc(x, weight, branch_weight, gate, alpha, eps)
    act = x.dtype
    if branch is not None and y is None:
        y = torch.empty(rows, cols, dtype=act, device=x.device)
    if norm and h is None:
        h = torch.empty(rows, cols, dtype=act, device=x.device)
    if norm and rstd is None:
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    if branch_weight is not None and branch_rstd is None:
        branch_rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    px, d.ld_x = _rows(x, rows, cols, act, "x")
    pb, d.ld_branch = _rows(branch, rows, cols, act, "branch")
    py, d.ld_y = _rows(y, rows, cols, act, "y") if branch is not None else (None, 0)
    ph, d.ld_h = _rows(h, rows, cols, act, "h") if norm else (None, 0)
    _check(_L.sl_norm_forward(C.byref(d), px, pb, _ptr(branch_weight, wt, cols, "branch_weight"), g, _ptr(weight, wt, cols, "weight"), py, ph,
                              _ptr(branch_rstd, torch.float32, rows, "branch_rstd"), _ptr(rstd, torch.float32, rows, "rstd"), _stream()))
    return y if branch is not None else x, h, rstd, branch_rstd


def norm_backward_workspace(rows: int, cols: int, *, dtype=torch.bfloat16) -> torch.Tensor:
    """Scratch memory for `norm_backward` on [rows, cols] activations: the column sums before they are added up."""
    d, n = _NormDesc(rows, cols, _dtype(dtype), 0, 0, 1.0, 0.0), C.c_size_t()
    _check(_L.sl_norm_workspace_bytes(C.byref(d), C.byref(n)))
    return torch.empty(max(n.value, 16), dtype=torch.uint8, device="cuda")


def norm_backward(dy, dh, y, weight=None, *, rstd=None, branch=None, branch_weight=None, branch_rstd=None, gate=None, alpha: float = 1.0, dx=None, dbranch=None, dweight=None,
                  dbranch_weight=None, dgate=None, workspace=None) -> None:
    """Gradients of `norm_forward`, written into the outputs that are given.  `y`, `rstd`, `branch_rstd` as the forward pass left them;
    dy (gradient that reaches y from elsewhere) or dh may be None."""
    ref = y if y is not None else dy
    d, rows, cols, wt, g = _norm_desc(ref, weight, branch_weight, gate, alpha, 0.0)
    act = ref.dtype
    pdy, d.ld_dy = _rows(dy, rows, cols, act, "dy")
    pdh, d.ld_dh = _rows(dh, rows, cols, act, "dh")
    py, d.ld_y = _rows(y, rows, cols, act, "y")
    pb, d.ld_branch = _rows(branch, rows, cols, act, "branch")
    pdx, d.ld_x = _rows(dx, rows, cols, act, "dx")
    pdb, ld = _rows(dbranch, rows, cols, act, "dbranch")
    _need(dbranch is None or rows <= 1 or ld == d.ld_branch, "dbranch must have the row stride of branch")
    pdg = None
    if dgate is not None:
        _need(gate is not None and dgate.shape == gate.shape, "dgate must have the shape of gate")
        kind, pdg, ld = _gate(dgate, rows, cols, act, wt)
        _need(kind == d.gate_kind and (ld == d.ld_gate or rows <= 1), "dgate must have the strides of gate")
    if workspace is None and (dweight is not None or dbranch_weight is not None or (dgate is not None and d.gate_kind == GATES["column"])):
        workspace = norm_backward_workspace(rows, cols, dtype=act)
    _check(_L.sl_norm_backward(C.byref(d), pdy, pdh, py, pb, _ptr(branch_weight, wt, cols, "branch_weight"), g, _ptr(weight, wt, cols, "weight"),
                               _ptr(branch_rstd, torch.float32, rows, "branch_rstd"), _ptr(rstd, torch.float32, rows, "rstd"), pdx, pdb, _ptr(dweight, wt, cols, "dweight"),
                               _ptr(dbranch_weight, wt, cols, "dbranch_weight"), pdg, _ptr(workspace, torch.uint8, 0, "workspace"),
                               0 if workspace is None else workspace.numel(), _stream()))


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, branch, weight, branch_weight, gate, alpha, eps):
        y, h, rstd, brstd = norm_forward(x, weight, branch=branch, branch_weight=branch_weight, gate=gate, alpha=alpha, eps=eps)
        ctx.save_for_backward(y, branch, weight, branch_weight, gate, rstd, brstd)
        ctx.alpha = alpha
        if branch is None:
            y = x.clone()
        return y, h

    @staticmethod
    def backward(ctx, dy, dh):
        y, branch, weight, branch_weight, gate, rstd, brstd = ctx.saved_tensors
        need = ctx.needs_input_grad

        def like(t, needed):
            return torch.empty_like(t, memory_format=torch.contiguous_format) if t is not None and needed else None

        branch = None if branch is None else branch.contiguous()
        gate = None if gate is None else gate.contiguous()
        out = [torch.empty_like(y, memory_format=torch.contiguous_format) if need[0] else None, like(branch, need[1]), like(weight, need[2]), like(branch_weight, need[3]), like(gate, need[4])]
        if any(o is not None for o in out):
            norm_backward(dy.contiguous(), dh.contiguous(), y, weight, rstd=rstd, branch=branch, branch_weight=branch_weight, branch_rstd=brstd, gate=gate, alpha=ctx.alpha,
                          dx=out[0], dbranch=out[1], dweight=out[2], dbranch_weight=out[3], dgate=out[4])
        return (*out, None, None)


def block_norm(x, weight=None, *, branch=None, branch_weight=None, gate=None, alpha: float = 1.0, eps: float = 1e-6):
    """(y, h) of `norm_forward` under autograd, on [..., cols] activations; a gate is [cols], [..., 1] or [..., cols]."""
    shape = x.shape
    flat = [None if t is None else t.reshape(-1, shape[-1]) for t in (x, branch)]
    if gate is not None and gate.dim() > 1:
        gate = gate.reshape(-1, gate.shape[-1])
    y, h = _BlockNorm.apply(flat[0], flat[1], weight, branch_weight, gate, alpha, eps)
    return y.view(shape), h.view(shape)


# ------------------------------------------------------------------------------------------------------------ rotary
class Rotary:
    """Rotary positions for the first `rot_dim` values of every head; see the header for the layouts and scalings."""

    def __init__(self, rot_dim: int, *, base: float = 10000.0, layout: str = "half", scaling: str = "none", factor: float = 1.0, original_length: float = 0.0, low_turns: float = 1.0,
                 high_turns: float = 32.0, magnitude: float = 1.0):
        _need(layout in LAYOUTS and scaling in SCALINGS, f"layout {layout!r} / scaling {scaling!r} unknown")
        cfg = _RotaryConfig(rot_dim, LAYOUTS[layout], SCALINGS[scaling], base, factor, original_length, low_turns, high_turns, magnitude)
        self._h, self.rot_dim = P(), rot_dim
        _check(_L.sl_rotary_create(C.byref(cfg), C.byref(self._h)))

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            _L.sl_rotary_destroy(self._h)
            self._h = P()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def apply(self, q, k=None, positions=None, *, first: int = 0, inverse: bool = False, out_q=None, out_k=None) -> None:
        """Turns q (and k), [batch, seq, heads, head_dim] with any strides but a unit one inside a head: in place, or into
        out_q / out_k.  `positions`: int32 or int64 [seq] or [batch, seq]; None: first + token.  `inverse`: the backward pass."""
        _need(q.dim() == 4, "q must be [batch, seq, heads, head_dim]")
        batch, seq, _, head_dim = q.shape

        def heads(x, out, what):
            if x is None:
                return None
            out = x if out is None else out
            _need(x.dim() == 4 and x.shape[0] == batch and x.shape[1] == seq and x.shape[3] == head_dim and out.shape == x.shape, f"{what}: shapes {tuple(x.shape)}, {tuple(out.shape)}")
            _need(x.is_cuda and out.is_cuda and x.dtype == q.dtype and out.dtype == q.dtype, f"{what} must be CUDA tensors of {q.dtype}")
            _need(head_dim == 1 or (x.stride(3) == 1 and out.stride(3) == 1), f"{what} must have a unit stride inside a head")
            return _RotaryHeads(x.data_ptr(), out.data_ptr(), x.shape[2], *x.stride()[:3], *out.stride()[:3])

        hq, hk = heads(q, out_q, "q"), heads(k, out_k, "k")
        d = _RotaryDesc(_dtype(q.dtype), 64, int(inverse), batch, seq, head_dim, first)
        pos = None
        if positions is not None:
            _need(positions.is_cuda and positions.dtype in (torch.int32, torch.int64), "positions must be a CUDA tensor of int32 or int64")
            _need(tuple(positions.shape) in ((seq,), (batch, seq)), f"positions must be [{seq}] or [{batch}, {seq}], got {tuple(positions.shape)}")
            d.position_bits = 32 if positions.dtype == torch.int32 else 64
            d.pos_token = positions.stride(-1)
            d.pos_batch = positions.stride(0) if positions.dim() == 2 else 0
            pos = positions.data_ptr()
        if batch * seq == 0:
            return
        _check(_L.sl_rotary_apply(self._h, C.byref(d), C.byref(hq), C.byref(hk) if hk is not None else None, pos, _stream()))


class _Turn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, rope, positions, first):
        ctx.rope, ctx.positions, ctx.first = rope, positions, first
        out_q, out_k = torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(k.shape, dtype=k.dtype, device=k.device)
        rope.apply(q, k, positions, first=first, out_q=out_q, out_k=out_k)
        return out_q, out_k

    @staticmethod
    def backward(ctx, dq, dk):
        out_q, out_k = torch.empty(dq.shape, dtype=dq.dtype, device=dq.device), torch.empty(dk.shape, dtype=dk.dtype, device=dk.device)
        dq, dk = (t if t.stride(-1) == 1 else t.contiguous() for t in (dq, dk))
        ctx.rope.apply(dq, dk, ctx.positions, first=ctx.first, inverse=True, out_q=out_q, out_k=out_k)
        return out_q, out_k, None, None, None


def rotary(rope: Rotary, q, k, positions=None, *, first: int = 0):
    """`rope.apply` under autograd: new q and k."""
    return _Turn.apply(q, k, rope, positions, first)


# -------------------------------------------------------------------------------------------------------------- loss
def loss_workspace() -> torch.Tensor:
    return torch.empty(_L.sl_loss_workspace_bytes(), dtype=torch.uint8, device="cuda")


def token_loss(logits, targets, *, grad=None, ignore_index: int = -100, smoothing: float = 0.0, z: float = 0.0, mean: bool = True, scale: float = 1.0, row_loss=None, lse=None, total=None,
               workspace=None):
    """Loss of every row of [rows, vocab] logits and, into `grad` (which may be `logits`), its gradient.  Returns (total, row_loss, lse):
    total = sum of the row losses, divided by the rows that count with `mean`, times `scale`; the gradient is total's."""
    _need(logits.dim() == 2, "logits must be [rows, vocab]")
    rows, vocab = logits.shape
    _need(targets.is_cuda and targets.is_contiguous() and tuple(targets.shape) == (rows,) and targets.dtype in (torch.int32, torch.int64), f"targets must be [{rows}] int32 or int64, contiguous, on the GPU")
    d = _LossDesc(rows, vocab, _dtype(logits.dtype), 32 if targets.dtype == torch.int32 else 64, 0, 0, ignore_index, smoothing, z, scale, int(mean))
    px, d.ld_logits = _rows(logits, rows, vocab, logits.dtype, "logits")
    pg, d.ld_grad = _rows(grad, rows, vocab, logits.dtype, "grad")
    dev = logits.device
    row_loss = torch.empty(rows, device=dev) if row_loss is None else row_loss
    lse = torch.empty(rows, device=dev) if lse is None else lse
    total = torch.empty(1, device=dev) if total is None else total
    workspace = loss_workspace() if workspace is None else workspace
    _check(_L.sl_token_loss(C.byref(d), px, targets.data_ptr(), pg, _ptr(row_loss, torch.float32, rows, "row_loss"), _ptr(lse, torch.float32, rows, "lse"),
                            _ptr(total, torch.float32, 1, "total"), _ptr(workspace, torch.uint8, 0, "workspace"), workspace.numel(), _stream()))
    return total, row_loss, lse


class _NextTokenLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, ignore_index, smoothing, z):
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device) if ctx.needs_input_grad[0] else None
        total, _, _ = token_loss(logits, targets, grad=grad, ignore_index=ignore_index, smoothing=smoothing, z=z)
        ctx.save_for_backward(grad)
        return total.view(())

    @staticmethod
    def backward(ctx, d):
        (grad,) = ctx.saved_tensors
        return grad * d.to(grad.dtype), None, None, None, None


def next_token_loss(logits, targets, *, ignore_index: int = -100, smoothing: float = 0.0, z: float = 0.0):
    """Mean loss over the rows that count, under autograd; the gradient is formed in the forward pass."""
    return _NextTokenLoss.apply(logits.reshape(-1, logits.shape[-1]), targets.reshape(-1), ignore_index, smoothing, z)
