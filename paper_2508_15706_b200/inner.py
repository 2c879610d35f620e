"""The inner phase (Algorithm 1, a worker's H local steps): AdamW over the tensor table, the norms around a block, rotary
positions and the next-token loss.  Wrappers over libsparseloco's C entry points (include/sparseloco.h has the formulas).

Two layers.  `AdamW`, `Rotary`, `norm_forward` / `norm_backward` and `token_loss` marshal arguments only: buffers are the
caller's (allocated here where an output is left out), work goes on torch's current stream, nothing synchronises.
`block_norm`, `rotary` and `next_token_loss` are the same operators as autograd functions, for a model that runs under
torch's autograd.  Their backward passes are kernels without derivatives of their own: a second derivative raises.
"""
from __future__ import annotations

import ctypes as C
import struct
import sys
from typing import Optional, Sequence

import torch
from torch.autograd.function import once_differentiable

try:
    from . import _checks
    if _checks.built_for != f"built for torch {torch.__version__} {sys.implementation.cache_tag}":
        raise ImportError(f"it was {_checks.built_for}")
except (ImportError, AttributeError) as e:
    raise ImportError("the extension _checks.so is missing or was built for another torch: build it with `python -c 'import __graft_entry__ as g; g.build()'`") from e
from .binding import SlError, SL_ERR_INVALID_ARG, _check, _L, _TensorDesc

P, I32, I64, F32, F64 = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_double
DTYPES = {torch.float32: 0, torch.bfloat16: 1}
LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "base": 2, "by_parts": 3}


class _AdamWConfig(C.Structure):
    _fields_ = [("param_dtype", I32), ("grad_dtype", I32), ("state_bits", I32), ("skip_nonfinite", I32), ("beta1", F64), ("beta2", F64), ("eps", F64), ("max_norm", F64)]


class _NormDesc(C.Structure):
    _fields_ = [("rows", I64), ("cols", I64), ("dtype", I32), ("weight_dtype", I32), ("gate_kind", I32), ("alpha", F32), ("eps", F32),
                ("ld_x", I64), ("ld_branch", I64), ("ld_gate", I64), ("ld_y", I64), ("ld_h", I64), ("ld_dy", I64), ("ld_dh", I64)]


class _RotaryConfig(C.Structure):
    _fields_ = [("rot_dim", I32), ("layout", I32), ("scaling", I32), ("base", F64), ("factor", F64), ("original_length", F64), ("low_turns", F64), ("high_turns", F64), ("magnitude", F64)]


class _RotaryDesc(C.Structure):
    _fields_ = [("dtype", I32), ("position_bits", I32), ("inverse", I32), ("batch", I64), ("seq", I64), ("head_dim", I64), ("first", I64), ("pos_batch", I64), ("pos_token", I64)]


class _LossDesc(C.Structure):
    _fields_ = [("rows", I64), ("vocab", I64), ("dtype", I32), ("target_bits", I32), ("ld_logits", I64), ("ld_grad", I64), ("ignore_index", I64), ("smoothing", F32), ("z", F32), ("scale", F32), ("mean", I32)]


# The descriptions of a call as bytes in the C layout: packing is several times faster than filling a ctypes structure.
_norm_bytes = struct.Struct("@qqiiiffqqqqqqq").pack      # _NormDesc
_rotary_bytes = struct.Struct("@iiiqqqqqq").pack          # _RotaryDesc
_loss_bytes = struct.Struct("@qqiiqqqfffi").pack          # _LossDesc (without the padding at its end)

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
_L.sl_token_loss_backward.argtypes = [I32, I64, P, P, P, P]


def _refuse(what: str):
    raise SlError(SL_ERR_INVALID_ARG, "libsparseloco: " + what)


def _dtype(t: torch.dtype) -> int:
    code = DTYPES.get(t)
    if code is None:
        _refuse(f"{t} is not one of float32, bfloat16")
    return code


_here = torch._C._cuda_getDevice            # the current device
_queue = torch._C._cuda_getCurrentRawStream  # its current stream

# The checks of every tensor of a call, compiled (csrc/checks.cpp): in Python they took half of a small call.
#   _ptr(t, device, numel, dtype, what)           address of a contiguous tensor of at least numel elements, None of None
#   _rows(t, device, rows, cols, dtype, what)     (address, row stride) of a matrix with a unit column stride, (None, 0) of None
#   _heads(x, out, device, batch, seq, head_dim, dtype, what)   a sl_rotary_heads as bytes
_ptr, _rows, _heads = _checks.ptr, _checks.rows, _checks.heads


def _refuse_tensor(what, t, wanted):
    got = f"{t.dtype} {tuple(t.shape)} strides {t.stride() if t.layout is torch.strided else t.layout} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
    _refuse(f"{what} must be {wanted}, got {got}")


_checks.set_refuse(_refuse_tensor)


class AdamW:
    """AdamW over a tensor table (shapes and element offsets as for `SparseLoCo`), gradients clipped by their global norm.

    Parameters, gradients and moments are flat buffers of one layout: let every parameter's `.grad` be a view of the flat
    gradient, and theta_local[r] of the outer step is the very buffer that `step` updates.  `state_bits=8` keeps the moments
    in 8-bit codes with one power-of-two scale per 128 elements: 2 bytes per parameter in place of 8.

    One object holds scratch memory for the gradient's norm: its steps must not overlap on the device (two streams want two objects)."""

    def __init__(self, shapes: Sequence[Sequence[int]], offsets: Optional[Sequence[int]] = None, *, weight_decay=0.1, betas=(0.9, 0.95),
                 eps: float = 1e-8, max_norm: float = 1.0, state_bits: int = 32, param_dtype=torch.float32, grad_dtype=torch.float32, skip_nonfinite: bool = True):
        n = len(shapes)
        if offsets is not None and len(offsets) != n:
            _refuse(f"{len(offsets)} offsets for {n} tensors")
        descs, pos = (_TensorDesc * n)(), 0
        for j, sh in enumerate(shapes):
            if len(sh) not in (1, 2):
                _refuse(f"tensor {j} must be [rows, cols] or a vector, got {tuple(sh)}")
            rows, cols = (1, sh[0]) if len(sh) == 1 else (sh[0], sh[1])
            off = offsets[j] if offsets is not None else (pos + 3) // 4 * 4
            descs[j] = _TensorDesc(rows, cols, off)
            pos = off + rows * cols
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        if len(decay) != n:
            _refuse(f"{len(decay)} weight decays for {n} tensors")
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

    def _state(self, dev, m, v, scales):
        if dev != self.device.index:
            _refuse(f"this AdamW was made on {self.device}, the current device is {dev}")
        return (_ptr(m, dev, self.flat_elems, self._moment, "m"), _ptr(v, dev, self.flat_elems, self._moment, "v"), _ptr(scales, dev, 2 * self.blocks, torch.uint8, "scales"))

    def step(self, theta, grad, m, v, scales=None, *, step: int, lr: float, grad_scale: float = 1.0, seed: Optional[int] = None, copy=None, norm=None) -> None:
        """One step, in place.  `step` counts from 1; `grad_scale` multiplies the gradient (1 / accumulated micro-batches);
        `copy` receives a bfloat16 copy of the new parameters, `norm` (one fp32) the gradient's norm before clipping;
        `seed` (default: the step) seeds the rounding of an 8-bit second moment."""
        dev, n = _here(), self.flat_elems
        pm, pv, ps = self._state(dev, m, v, scales)
        _check(_L.sl_adamw_step(self._h, _ptr(theta, dev, n, self.param_dtype, "theta"), _ptr(grad, dev, n, self.grad_dtype, "grad"), pm, pv, ps,
                                _ptr(copy, dev, n, torch.bfloat16, "copy"), _ptr(norm, dev, 1, torch.float32, "norm"), step, lr, grad_scale,
                                (step if seed is None else seed) & 0xFFFFFFFF, _queue(dev)))

    def read_state(self, m, v, scales, m_out, v_out) -> None:
        """8-bit moments as fp32 values, in flat buffers of the same layout."""
        dev, n = _here(), self.flat_elems
        pm, pv, ps = self._state(dev, m, v, scales)
        _check(_L.sl_adamw_read_state(self._h, pm, pv, ps, _ptr(m_out, dev, n, torch.float32, "m_out"), _ptr(v_out, dev, n, torch.float32, "v_out"), _queue(dev)))

    def write_state(self, m_in, v_in, m, v, scales, *, seed: int = 0) -> None:
        """fp32 moments into the 8-bit form, rounded as a step rounds them."""
        dev, n = _here(), self.flat_elems
        pm, pv, ps = self._state(dev, m, v, scales)
        _check(_L.sl_adamw_write_state(self._h, _ptr(m_in, dev, n, torch.float32, "m_in"), _ptr(v_in, dev, n, torch.float32, "v_in"), pm, pv, ps, seed & 0xFFFFFFFF, _queue(dev)))


def _laid_out(t):
    """A matrix as the kernels take it, unit column stride and rows apart: itself, or (transposed, expanded) a copy."""
    if t is None or ((t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1])):
        return t
    return t.contiguous()


# ------------------------------------------------------------------------------------------------------------- norms
def _gate(gate, dev, rows, cols, act, wt):
    """(kind, address, stride): [cols] = per column, [rows, 1] or (rows != cols) [rows] = per row, [rows, cols] = per element."""
    sh = gate.shape
    if len(sh) == 1 and sh[0] == cols:
        return 1, _ptr(gate, dev, cols, wt, "column gate"), 0
    if sh == (rows,) or (sh == (rows, 1) and cols != 1):
        st = gate.stride(0)
        if gate.get_device() != dev or gate.dtype is not act or (rows > 1 and st < 1):
            _refuse(f"a row gate must be a CUDA tensor of {act} on device {dev} with a positive stride")
        return 2, gate.data_ptr(), st if rows > 1 else 1
    return (3, *_rows(gate, dev, rows, cols, act, "element gate"))


def _norm_case(x, dev, weight, branch_weight, gate):
    """Rows, columns, types, and the gate's kind, address and stride."""
    if x.dim() != 2:
        _refuse("activations must be [rows, cols]")
    rows, cols = x.shape
    act = x.dtype
    if weight is not None:
        wt = weight.dtype
    elif branch_weight is not None:
        wt = branch_weight.dtype
    else:
        wt = gate.dtype if gate is not None and gate.shape == (cols,) else torch.float32
    kind, g, ld = (0, None, 0) if gate is None else _gate(gate, dev, rows, cols, act, wt)
    return rows, cols, act, wt, kind, g, ld


def norm_forward(x, weight=None, *, branch=None, branch_weight=None, gate=None, alpha: float = 1.0, eps: float = 1e-6, norm: bool = True, y=None, h=None, rstd=None, branch_rstd=None):
    """y = x + alpha * gate * norm(branch) (the norm only with `branch_weight`), h = norm(y) * weight (`norm=False`: no h).
    Returns (y, h, rstd, branch_rstd); y is x itself without a branch.  Outputs left out are allocated."""
    dev = _here()
    rows, cols, act, wt, kind, g, ld_g = _norm_case(x, dev, weight, branch_weight, gate)
    if branch is not None and y is None:
        y = torch.empty(rows, cols, dtype=act, device=x.device)
    if norm and h is None:
        h = torch.empty(rows, cols, dtype=act, device=x.device)
    if norm and rstd is None:
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    if branch_weight is not None and branch_rstd is None:
        branch_rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    px, ld_x = _rows(x, dev, rows, cols, act, "x")
    pb, ld_b = _rows(branch, dev, rows, cols, act, "branch")
    py, ld_y = _rows(y, dev, rows, cols, act, "y") if branch is not None else (None, 0)
    ph, ld_h = _rows(h, dev, rows, cols, act, "h") if norm else (None, 0)
    d = _norm_bytes(rows, cols, _dtype(act), _dtype(wt), kind, alpha, eps, ld_x, ld_b, ld_g, ld_y, ld_h, 0, 0)
    _check(_L.sl_norm_forward(d, px, pb, _ptr(branch_weight, dev, cols, wt, "branch_weight"), g, _ptr(weight, dev, cols, wt, "weight"), py, ph,
                              _ptr(branch_rstd, dev, rows, torch.float32, "branch_rstd"), _ptr(rstd, dev, rows, torch.float32, "rstd"), _queue(dev)))
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
    dev = _here()
    rows, cols, act, wt, gate_kind, g, ld_g = _norm_case(y if y is not None else dy, dev, weight, branch_weight, gate)
    pdy, ld_dy = _rows(dy, dev, rows, cols, act, "dy")
    pdh, ld_dh = _rows(dh, dev, rows, cols, act, "dh")
    py, ld_y = _rows(y, dev, rows, cols, act, "y")
    pb, ld_b = _rows(branch, dev, rows, cols, act, "branch")
    pdx, ld_x = _rows(dx, dev, rows, cols, act, "dx")
    pdb, ld = _rows(dbranch, dev, rows, cols, act, "dbranch")
    if dbranch is not None and ld != ld_b:
        _refuse("dbranch must have the row stride of branch")
    pdg = None
    if dgate is not None:
        if gate is None or dgate.shape != gate.shape:
            _refuse("dgate must have the shape of gate")
        kind, pdg, ld = _gate(dgate, dev, rows, cols, act, wt)
        if ld != ld_g:
            _refuse("dgate must have the strides of gate")
    if workspace is None and (dweight is not None or dbranch_weight is not None or (dgate is not None and gate_kind == 1)):
        workspace = norm_backward_workspace(rows, cols, dtype=act)
    d = _norm_bytes(rows, cols, _dtype(act), _dtype(wt), gate_kind, alpha, 0.0, ld_x, ld_b, ld_g, ld_y, 0, ld_dy, ld_dh)
    _check(_L.sl_norm_backward(d, pdy, pdh, py, pb, _ptr(branch_weight, dev, cols, wt, "branch_weight"), g, _ptr(weight, dev, cols, wt, "weight"),
                               _ptr(branch_rstd, dev, rows, torch.float32, "branch_rstd"), _ptr(rstd, dev, rows, torch.float32, "rstd"), pdx, pdb, _ptr(dweight, dev, cols, wt, "dweight"),
                               _ptr(dbranch_weight, dev, cols, wt, "dbranch_weight"), pdg, _ptr(workspace, dev, 0, torch.uint8, "workspace"),
                               0 if workspace is None else workspace.numel(), _queue(dev)))


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
    @once_differentiable
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
    """(y, h) of `norm_forward` under autograd, on [..., cols] activations of any strides; a gate is [cols], [..., 1] or [..., cols]."""
    shape = x.shape
    flat = [None if t is None else _laid_out(t.reshape(-1, shape[-1])) for t in (x, branch)]
    if gate is not None:
        gate = gate.contiguous() if gate.dim() < 2 else _laid_out(gate.reshape(-1, gate.shape[-1]))
    vectors = [None if t is None else t.contiguous() for t in (weight, branch_weight)]
    y, h = _BlockNorm.apply(flat[0], flat[1], vectors[0], vectors[1], gate, alpha, eps)
    return y.view(shape), h.view(shape)


# ------------------------------------------------------------------------------------------------------------ rotary
class Rotary:
    """Rotary positions for the first `rot_dim` values of every head; see the header for the layouts and scalings."""

    def __init__(self, rot_dim: int, *, base: float = 10000.0, layout: str = "half", scaling: str = "none", factor: float = 1.0, original_length: float = 0.0, low_turns: float = 1.0,
                 high_turns: float = 32.0, magnitude: float = 1.0):
        if layout not in LAYOUTS or scaling not in SCALINGS:
            _refuse(f"layout {layout!r} / scaling {scaling!r} unknown")
        cfg = _RotaryConfig(rot_dim, LAYOUTS[layout], SCALINGS[scaling], base, factor, original_length, low_turns, high_turns, magnitude)
        self._h, self.rot_dim = P(), rot_dim
        self.device = torch.device("cuda", torch.cuda.current_device())
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
        dev = _here()
        if dev != self.device.index or q.dim() != 4:
            _refuse(f"q must be [batch, seq, heads, head_dim] on {self.device}, where this Rotary was made, and that the current device")
        batch, seq, _, head_dim = q.shape
        dtype = q.dtype
        hq = _heads(q, q if out_q is None else out_q, dev, batch, seq, head_dim, dtype, "q")
        hk = None if k is None else _heads(k, k if out_k is None else out_k, dev, batch, seq, head_dim, dtype, "k")
        bits, pos, pos_batch, pos_token = 64, None, 0, 0
        if positions is not None:
            sh, bits = positions.shape, 64 if positions.dtype is torch.int64 else 32 if positions.dtype is torch.int32 else 0
            if positions.get_device() != dev or not bits or (sh != (batch, seq) and sh != (seq,)):
                _refuse(f"positions must be a CUDA tensor [{seq}] or [{batch}, {seq}] of int32 or int64, got {positions.dtype} {tuple(sh)}")
            st = positions.stride()
            pos, pos_token, pos_batch = positions.data_ptr(), st[-1], st[0] if len(st) == 2 else 0
        if batch * seq == 0:
            return
        d = _rotary_bytes(_dtype(dtype), bits, inverse, batch, seq, head_dim, first, pos_batch, pos_token)
        _check(_L.sl_rotary_apply(self._h, d, hq, hk, pos, _queue(dev)))


class _Turn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, rope, positions, first):
        ctx.rope, ctx.first = rope, first
        ctx.save_for_backward(positions)
        out = [None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k)]
        rope.apply(q, k, positions, first=first, out_q=out[0], out_k=out[1])
        return tuple(out)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        out = [None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (dq, dk)]
        dq, dk = (t if t is None or t.stride(-1) == 1 else t.contiguous() for t in (dq, dk))
        ctx.rope.apply(dq, dk, ctx.saved_tensors[0], first=ctx.first, inverse=True, out_q=out[0], out_k=out[1])
        return (*out, None, None, None)


def rotary(rope: Rotary, q, k=None, positions=None, *, first: int = 0):
    """`rope.apply` under autograd, for any strides: new q and k (None without k)."""
    q, k = (t if t is None or t.stride(-1) == 1 else t.contiguous() for t in (q, k))
    return _Turn.apply(q, k, rope, positions, first)


# -------------------------------------------------------------------------------------------------------------- loss
def loss_workspace() -> torch.Tensor:
    return torch.empty(_L.sl_loss_workspace_bytes(), dtype=torch.uint8, device="cuda")


def token_loss(logits, targets, *, grad=None, ignore_index: int = -100, smoothing: float = 0.0, z: float = 0.0, mean: bool = True, scale: float = 1.0, row_loss=None, lse=None, total=None,
               workspace=None):
    """Loss of every row of [rows, vocab] logits and, into `grad` (which may be `logits`), its gradient.  Returns (total, row_loss, lse):
    total = sum of the row losses, divided by the rows that count with `mean`, times `scale`; the gradient is total's."""
    if logits.dim() != 2:
        _refuse("logits must be [rows, vocab]")
    dev = _here()
    rows, vocab = logits.shape
    act = logits.dtype
    bits = 64 if targets.dtype is torch.int64 else 32 if targets.dtype is torch.int32 else 0
    if not bits or targets.shape != (rows,):
        _refuse(f"targets must be [{rows}] of int32 or int64, got {targets.dtype} {tuple(targets.shape)}")
    pt = _ptr(targets, dev, rows, targets.dtype, "targets")
    px, ld_x = _rows(logits, dev, rows, vocab, act, "logits")
    pg, ld_g = _rows(grad, dev, rows, vocab, act, "grad")
    row_loss = torch.empty(rows, dtype=torch.float32, device=logits.device) if row_loss is None else row_loss
    lse = torch.empty(rows, dtype=torch.float32, device=logits.device) if lse is None else lse
    total = torch.empty(1, dtype=torch.float32, device=logits.device) if total is None else total
    workspace = loss_workspace() if workspace is None else workspace
    d = _loss_bytes(rows, vocab, _dtype(act), bits, ld_x, ld_g, ignore_index, smoothing, z, scale, mean)
    _check(_L.sl_token_loss(d, px, pt, pg, _ptr(row_loss, dev, rows, torch.float32, "row_loss"), _ptr(lse, dev, rows, torch.float32, "lse"),
                            _ptr(total, dev, 1, torch.float32, "total"), _ptr(workspace, dev, 0, torch.uint8, "workspace"), workspace.numel(), _queue(dev)))
    return total, row_loss, lse


class _NextTokenLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, ignore_index, smoothing, z, scale):
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device) if ctx.needs_input_grad[0] else None
        total, _, _ = token_loss(logits, targets, grad=grad, ignore_index=ignore_index, smoothing=smoothing, z=z, scale=scale)
        ctx.save_for_backward(grad)
        return total.view(())

    @staticmethod
    @once_differentiable
    def backward(ctx, d):
        (grad,) = ctx.saved_tensors
        dev, out = _here(), torch.empty_like(grad)
        _check(_L.sl_token_loss_backward(_dtype(grad.dtype), grad.numel(), grad.data_ptr(), _ptr(d, dev, 1, torch.float32, "the loss's gradient"), out.data_ptr(), _queue(dev)))
        return out, None, None, None, None, None


def next_token_loss(logits, targets, *, ignore_index: int = -100, smoothing: float = 0.0, z: float = 0.0, scale: float = 1.0):
    """Mean loss over the rows that count, times `scale`, under autograd; the gradient is formed in the forward pass.  A factor known
    beforehand (1 / accumulated micro-batches) belongs into `scale`: a bfloat16 gradient is then rounded once, by
    `(loss * factor).backward()` twice."""
    return _NextTokenLoss.apply(_laid_out(logits.reshape(-1, logits.shape[-1])), targets.reshape(-1).contiguous(), ignore_index, smoothing, z, scale)
