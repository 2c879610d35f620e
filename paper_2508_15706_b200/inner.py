"""The inner phase (Algorithm 1, a worker's H local steps): AdamW over the tensor table, the norms around a block, rotary
positions, attention over packed sequences, the router of a mixture of experts with the rows it sends, and the next-token loss.
Wrappers over libsparseloco's C entry points (include/sparseloco.h has the formulas).

Two layers.  `AdamW`, `Rotary`, `norm_forward` / `norm_backward`, `attention_forward` / `attention_backward`, `route_forward` /
`route_backward`, `dispatch_rows`, `combine_rows` / `combine_backward` and `token_loss` marshal arguments only: buffers are the
caller's (allocated here where an output is left out), work goes on torch's current stream, nothing synchronises.
`block_norm`, `rotary`, `attention`, `route`, `dispatch`, `combine` and `next_token_loss` are the same operators as autograd
functions, for a model that runs under torch's autograd.  Their backward passes are kernels without derivatives of their own: a second derivative raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import struct
import sys
from typing import NamedTuple, Optional, Sequence

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


class _AttentionDesc(C.Structure):
    _fields_ = [("tokens", I64), ("sequences", I64), ("seq", I64), ("q_heads", I32), ("kv_heads", I32), ("head_dim", I32), ("dtype", I32), ("causal", I32), ("fill_rest", I32), ("scale", F32)] + \
        [(f"{x}_{y}", I64) for x in ("q", "k", "v", "o", "do", "dq", "dk", "dv") for y in ("token", "head")]


class _RouteDesc(C.Structure):
    _fields_ = [("rows", I64), ("experts", I32), ("k", I32), ("dtype", I32), ("renormalize", I32), ("ld_logits", I64), ("ld_dlogits", I64)]


class _RowsDesc(C.Structure):
    _fields_ = [("rows", I64), ("cols", I64), ("k", I32), ("dtype", I32), ("ld_tokens", I64), ("ld_out", I64), ("ld_residual", I64), ("ld_rows", I64), ("ld_drows", I64)]


# The descriptions of a call as bytes in the C layout: packing is several times faster than filling a ctypes structure.
_norm_bytes = struct.Struct("@qqiiiffqqqqqqq").pack      # _NormDesc
_rotary_bytes = struct.Struct("@iiiqqqqqq").pack          # _RotaryDesc
_loss_bytes = struct.Struct("@qqiiqqqfffi").pack          # _LossDesc (without the padding at its end)
_attention_bytes = struct.Struct("@qqqiiiiiif16q").pack   # _AttentionDesc
_route_bytes = struct.Struct("@qiiiiqq").pack             # _RouteDesc
_rows_bytes = struct.Struct("@qqiiqqqqq").pack            # _RowsDesc

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
_L.sl_attention_forward.argtypes = [P] * 8
_L.sl_attention_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
_L.sl_attention_backward.argtypes = [P] * 12 + [C.c_size_t, P]
_L.sl_route_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
_L.sl_route_forward.argtypes = [P] * 12 + [C.c_size_t, P]
_L.sl_route_backward.argtypes = [P] * 11
_L.sl_rows_dispatch.argtypes = [P] * 6
_L.sl_rows_combine.argtypes = [P] * 7
_L.sl_rows_combine_backward.argtypes = [P] * 9


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
#   _tokens(x, device, tokens, heads, head_dim, dtype, what)    (address, token stride, head stride), (None, 0, 0) of None
#   _empties(device, dtype, rows, cols, ...)      new CUDA tensors [rows, cols], or [rows] where cols is negative, in one piece of memory
_ptr, _rows, _heads, _tokens, _empties = _checks.ptr, _checks.rows, _checks.heads, _checks.tokens, _checks.empties


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
    if t is None or t.dim() != 2 or ((t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1])):
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


# --------------------------------------------------------------------------------------------------------- attention
def _attention_case(q, k, v, offsets, dev, scale):
    """Tokens, heads, shared heads, head width, type, sequences, their common length, the offsets' address, the scale."""
    if q.dim() not in (3, 4) or k.shape[:-2] != q.shape[:-2] or v.shape != k.shape:
        _refuse(f"q, k and v must be [tokens, heads, head_dim] or [batch, seq, heads, head_dim], of the same tokens, got {tuple(q.shape)}, {tuple(k.shape)}, {tuple(v.shape)}")
    heads, dim = q.shape[-2:]
    seq = q.shape[-3]
    tokens = seq if q.dim() == 3 else q.shape[0] * seq
    table, sequences = None, 0
    if offsets is not None:
        if q.dim() == 4 or offsets.dim() != 1 or offsets.numel() < 1:
            _refuse("offsets are int32 [sequences + 1], for [tokens, heads, head_dim]")
        table, sequences = _ptr(offsets, dev, 1, torch.int32, "offsets"), offsets.numel() - 1
    return tokens, heads, k.shape[-2], dim, q.dtype, sequences, seq, table, (dim ** -0.5 if dim else 1.0) if scale is None else scale


def attention_forward(q, k, v, offsets=None, *, causal: bool = True, scale: Optional[float] = None, out=None, lse=None):
    """Attention over packed sequences: q [tokens, heads, head_dim], k and v with heads that divide q's, sequence s being the tokens
    offsets[s] .. offsets[s + 1] - 1 (int32 on the device; None: one sequence); or [batch, seq, heads, head_dim] without offsets.
    Strides are free outside a head.  `scale` defaults to head_dim ** -0.5.  Returns (out, lse), lse fp32 [heads, tokens].  Rows of tokens in no sequence: 0
    in an `out` allocated here and -inf in such an `lse`, left as they were in one that is given."""
    dev = _here()
    tokens, heads, kv, dim, act, sequences, seq, table, scale = _attention_case(q, k, v, offsets, dev, scale)
    fill = out is None and lse is None
    apart = not fill and table is not None  # (the kernels fill the rest of both or of neither: of one alone it is set beforehand)
    if out is None:
        out = (torch.zeros if apart else torch.empty)(q.shape, dtype=act, device=q.device)
    if lse is None:
        (lse,) = _empties(dev, torch.float32, heads, tokens)
        if apart:
            lse.fill_(float("-inf"))
    pq, pk, pv = _tokens(q, dev, tokens, heads, dim, act, "q"), _tokens(k, dev, tokens, kv, dim, act, "k"), _tokens(v, dev, tokens, kv, dim, act, "v")
    po = _tokens(out, dev, tokens, heads, dim, act, "out")
    d = _attention_bytes(tokens, sequences, seq, heads, kv, dim, _dtype(act), causal, fill, scale, *pq[1:], *pk[1:], *pv[1:], *po[1:], 0, 0, 0, 0, 0, 0, 0, 0)
    _check(_L.sl_attention_forward(d, pq[0], pk[0], pv[0], table, po[0], _ptr(lse, dev, heads * tokens, torch.float32, "lse"), _queue(dev)))
    return out, lse


def _attention_scratch(d) -> torch.Tensor:
    n = C.c_size_t()
    _check(_L.sl_attention_workspace_bytes(d, C.byref(n)))
    return torch.empty(max(n.value, 16), dtype=torch.uint8, device="cuda")


def attention_workspace(q, k, offsets=None, *, causal: bool = True) -> torch.Tensor:
    """Scratch memory for `attention_backward` on tensors of these shapes: two fp32 per token and query head, and sums where tiles are few."""
    tokens, heads, kv, dim, act, sequences, seq, _, _ = _attention_case(q, k, k, offsets, _here(), 1.0)
    return _attention_scratch(_attention_bytes(tokens, sequences, seq, heads, kv, dim, _dtype(act), causal, 0, 1.0, *[0] * 16))


def attention_backward(dout, q, k, v, out, lse, offsets=None, *, causal: bool = True, scale: Optional[float] = None, dq=None, dk=None, dv=None, workspace=None):
    """Gradients of `attention_forward`, from its out and lse: (dq, dk, dv).  Those left out are allocated.  Rows of tokens in no
    sequence: 0 in those allocated here, left as they were in those given."""
    dev = _here()
    tokens, heads, kv, dim, act, sequences, seq, table, scale = _attention_case(q, k, v, offsets, dev, scale)
    fill = dq is None and dk is None and dv is None
    make = torch.empty if fill or table is None else torch.zeros  # (the kernels fill the rest of all three or of none)
    dq, dk, dv = (make(x.shape, dtype=act, device=x.device) if g is None else g for g, x in ((dq, q), (dk, k), (dv, v)))
    pq, pk, pv = _tokens(q, dev, tokens, heads, dim, act, "q"), _tokens(k, dev, tokens, kv, dim, act, "k"), _tokens(v, dev, tokens, kv, dim, act, "v")
    po, pd = _tokens(out, dev, tokens, heads, dim, act, "out"), _tokens(dout, dev, tokens, heads, dim, act, "dout")
    gq, gk, gv = _tokens(dq, dev, tokens, heads, dim, act, "dq"), _tokens(dk, dev, tokens, kv, dim, act, "dk"), _tokens(dv, dev, tokens, kv, dim, act, "dv")
    d = _attention_bytes(tokens, sequences, seq, heads, kv, dim, _dtype(act), causal, fill, scale, *pq[1:], *pk[1:], *pv[1:], *po[1:], *pd[1:], *gq[1:], *gk[1:], *gv[1:])
    workspace = _attention_scratch(d) if workspace is None else workspace
    _check(_L.sl_attention_backward(d, pd[0], pq[0], pk[0], pv[0], po[0], _ptr(lse, dev, heads * tokens, torch.float32, "lse"), table, gq[0], gk[0], gv[0],
                                    _ptr(workspace, dev, 0, torch.uint8, "workspace"), workspace.numel(), _queue(dev)))
    return dq, dk, dv


def _in_tokens(t):
    """A tensor as the attention kernels take it, a unit stride inside a head and sequences one behind the other: itself or a copy."""
    if t.dim() < 3 or ((t.shape[-1] <= 1 or t.stride(-1) == 1) and (t.dim() == 3 or t.shape[0] <= 1 or t.shape[1] <= 1 or t.stride(0) == t.shape[1] * t.stride(1))):
        return t  # (of fewer dimensions: refused by the call)
    return t.contiguous()


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, offsets, causal, scale):
        out, lse = attention_forward(q, k, v, offsets, causal=causal, scale=scale)
        ctx.save_for_backward(q, k, v, offsets, out, lse)
        ctx.causal, ctx.scale = causal, scale
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, offsets, out, lse = ctx.saved_tensors
        return (*attention_backward(_in_tokens(dout), q, k, v, out, lse, offsets, causal=ctx.causal, scale=ctx.scale), None, None, None)


def attention(q, k, v, offsets=None, *, causal: bool = True, scale: Optional[float] = None):
    """`attention_forward`'s out under autograd, for any strides."""
    return _Attention.apply(_in_tokens(q), _in_tokens(k), _in_tokens(v), offsets, causal, scale)


# ----------------------------------------------------------------------------------------------------------- experts
class Routing(NamedTuple):
    """What a router decides for [tokens, experts] logits; see `route_forward`."""
    weights: torch.Tensor  # fp32 [tokens, k]
    experts: torch.Tensor  # int32 [tokens, k], -1: the token does not count
    slots: torch.Tensor    # int32 [tokens, k], the choice's row in expert order, -1: none
    counts: torch.Tensor   # int32 [experts]
    offsets: torch.Tensor  # int32 [experts + 1], first row of every expert, then the number of rows used
    balance: torch.Tensor  # fp32 [1]
    z: torch.Tensor        # fp32 [1]
    lse: torch.Tensor      # fp32 [tokens]


@functools.lru_cache(maxsize=1024)
def _route_workspace_bytes(rows: int, experts: int, k: int) -> int:
    n = C.c_size_t()
    _check(_L.sl_route_workspace_bytes(_route_bytes(rows, experts, k, 0, 0, 0, 0), C.byref(n)))
    return max(n.value, 16)


def route_workspace(rows: int, experts: int, k: int) -> torch.Tensor:
    """Scratch memory for `route_forward`: a table of counts and sums."""
    return torch.empty(_route_workspace_bytes(rows, experts, k), dtype=torch.uint8, device="cuda")


def route_forward(logits, k: int, *, mask=None, renormalize: bool = True, workspace=None) -> Routing:
    """The k experts of every row of [tokens, experts] logits with their weights (softmax, over the chosen alone with `renormalize`), places in
    expert order, counts, balance loss and z loss.  `mask`: bool [tokens], False for tokens that do not count.  The results lie in one piece of memory: it lives as
    long as any of them."""
    if logits.dim() != 2:
        _refuse("logits must be [tokens, experts]")
    dev = _here()
    rows, E = logits.shape
    act = logits.dtype
    px, ld = _rows(logits, dev, rows, E, act, "logits")
    if mask is not None and mask.shape != (rows,):
        _refuse(f"mask must be bool [{rows}], got {mask.dtype} {tuple(mask.shape)}")
    pm = _ptr(mask, dev, rows, torch.bool, "mask")
    i32, f32 = torch.int32, torch.float32
    scratch = _route_workspace_bytes(rows, E, k) if workspace is None else 0
    # (scratch of up to 16 KB lies with the results, which saves a visit to the allocator; more of it would live as long as they do)
    weights, experts, slots, counts, offsets, balance, z, lse, spare = r = _empties(dev, f32, rows, k, i32, rows, k, i32, rows, k, i32, E, -1, i32, E + 1, -1, f32, 1, -1, f32, 1, -1, f32, rows, -1,
                                                                                    torch.uint8, scratch if scratch <= 16384 else 0, -1)
    if workspace is None:
        workspace = spare if scratch <= 16384 else _empties(dev, torch.uint8, scratch, -1)[0]
    _check(_L.sl_route_forward(_route_bytes(rows, E, k, _dtype(act), renormalize, ld, 0), px, pm, weights.data_ptr(), experts.data_ptr(), slots.data_ptr(), counts.data_ptr(),
                               offsets.data_ptr(), lse.data_ptr(), balance.data_ptr(), z.data_ptr(), _ptr(workspace, dev, 0, torch.uint8, "workspace"), workspace.numel(), _queue(dev)))
    return Routing(*r[:8])


def route_backward(logits, experts, weights, counts, lse, *, dweights=None, dbalance=None, dz=None, renormalize: bool = True, dlogits=None):
    """Gradient of the logits from that of the weights ([tokens, k]) and those of the balance and the z loss (one fp32 each); a
    gradient left out is 0.  `dlogits` may be `logits`."""
    if logits.dim() != 2 or experts.dim() != 2:
        _refuse("logits must be [tokens, experts], experts [tokens, k]")
    dev = _here()
    rows, E = logits.shape
    k, act = experts.shape[1], logits.dtype
    if experts.shape[0] != rows:
        _refuse(f"experts must be [{rows}, k], got {tuple(experts.shape)}")
    if dlogits is None:
        dlogits = torch.empty(rows, E, dtype=act, device=logits.device)
    px, ld = _rows(logits, dev, rows, E, act, "logits")
    pd, ld_d = _rows(dlogits, dev, rows, E, act, "dlogits")
    f32 = torch.float32
    _check(_L.sl_route_backward(_route_bytes(rows, E, k, _dtype(act), renormalize, ld, ld_d), px, _ptr(experts, dev, rows * k, torch.int32, "experts"), _ptr(weights, dev, rows * k, f32, "weights"),
                                _ptr(counts, dev, E, torch.int32, "counts"), _ptr(lse, dev, rows, f32, "lse"), _ptr(dweights, dev, rows * k, f32, "dweights"),
                                _ptr(dbalance, dev, 1, f32, "dbalance"), _ptr(dz, dev, 1, f32, "dz"), pd, _queue(dev)))
    return dlogits


def _slots_of(slots, rows, dev):
    if slots.dim() != 2 or (rows is not None and slots.shape[0] != rows):
        _refuse(f"slots must be int32 [{'tokens' if rows is None else rows}, k], got {slots.dtype} {tuple(slots.shape)}")
    return _ptr(slots, dev, 0, torch.int32, "slots")


def _used_of(offsets, dev):
    return None if offsets is None else _ptr(offsets, dev, 1, torch.int32, "offsets") + 4 * (offsets.numel() - 1)


def dispatch_rows(x, slots, offsets=None, *, out=None):
    """Rows of x [tokens, cols] to the places of their choices: out [tokens * k, cols].  With the router's `offsets`, rows behind the last
    place are set to 0; without, they stay as they are, in an `out` allocated here whatever stood in that memory."""
    if x.dim() != 2:
        _refuse("x must be [tokens, cols]")
    dev = _here()
    rows, cols = x.shape
    act, ps = x.dtype, _slots_of(slots, rows, dev)
    k = slots.shape[1]
    if out is None:
        out = torch.empty(rows * k, cols, dtype=act, device=x.device)
    px, ld = _rows(x, dev, rows, cols, act, "x")
    po, ld_o = _rows(out, dev, rows * k, cols, act, "out")
    _check(_L.sl_rows_dispatch(_rows_bytes(rows, cols, k, _dtype(act), ld, 0, 0, ld_o, 0), px, ps, _used_of(offsets, dev), po, _queue(dev)))
    return out


def combine_rows(y, slots, *, weights=None, residual=None, out=None):
    """Rows of y [tokens * k, cols] summed back into their tokens: residual + sum of weights * y over a token's choices; out [tokens, cols].
    Without weights, the gradient of `dispatch_rows`."""
    if y.dim() != 2:
        _refuse("y must be [tokens * k, cols]")
    dev = _here()
    ps = _slots_of(slots, None, dev)
    (rows, k), cols, act = slots.shape, y.shape[1], y.dtype
    if weights is not None and weights.shape != slots.shape:
        _refuse(f"weights must be fp32 {tuple(slots.shape)}, got {weights.dtype} {tuple(weights.shape)}")
    if out is None:
        out = torch.empty(rows, cols, dtype=act, device=y.device)
    py, ld = _rows(y, dev, rows * k, cols, act, "y")
    pr, ld_r = _rows(residual, dev, rows, cols, act, "residual")
    po, ld_o = _rows(out, dev, rows, cols, act, "out")
    _check(_L.sl_rows_combine(_rows_bytes(rows, cols, k, _dtype(act), 0, ld_o, ld_r, ld, 0), py, ps, _ptr(weights, dev, rows * k, torch.float32, "weights"), pr, po, _queue(dev)))
    return out


def combine_backward(dout, y, slots, weights=None, offsets=None, *, need_rows: bool = True, need_weights: bool = True, dy=None, dweights=None):
    """Gradients of `combine_rows`: (dy [tokens * k, cols], dweights fp32 [tokens, k]), None for one that is not needed.  With the router's
    `offsets`, rows of dy behind the last place are set to 0; without, they stay as they are, as in `dispatch_rows`."""
    if dout.dim() != 2:
        _refuse("dout must be [tokens, cols]")
    dev = _here()
    rows, cols = dout.shape
    act, ps = dout.dtype, _slots_of(slots, rows, dev)
    k = slots.shape[1]
    if need_rows and dy is None:
        dy = torch.empty(rows * k, cols, dtype=act, device=dout.device)
    if need_weights and dweights is None:
        dweights = torch.empty(rows, k, dtype=torch.float32, device=dout.device)
    pd, ld = _rows(dout, dev, rows, cols, act, "dout")
    py, ld_y = _rows(y, dev, rows * k, cols, act, "y")
    pg, ld_g = _rows(dy, dev, rows * k, cols, act, "dy")
    _check(_L.sl_rows_combine_backward(_rows_bytes(rows, cols, k, _dtype(act), ld, 0, 0, ld_y, ld_g), pd, py, ps, _ptr(weights, dev, rows * k, torch.float32, "weights"), _used_of(offsets, dev), pg,
                                       _ptr(dweights, dev, rows * k, torch.float32, "dweights"), _queue(dev)))
    return dy, dweights


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, mask, renormalize):
        r = route_forward(logits, k, mask=mask, renormalize=renormalize)
        ctx.save_for_backward(logits, r.experts, r.weights, r.counts, r.lse)
        ctx.renormalize = renormalize
        ctx.mark_non_differentiable(r.experts, r.slots, r.counts, r.offsets, r.lse)
        ctx.set_materialize_grads(False)
        return tuple(r)

    @staticmethod
    @once_differentiable
    def backward(ctx, dweights, _e, _s, _c, _o, dbalance, dz, _l):
        logits, experts, weights, counts, lse = ctx.saved_tensors
        dweights, dbalance, dz = (None if g is None else g.contiguous() for g in (dweights, dbalance, dz))
        return route_backward(logits, experts, weights, counts, lse, dweights=dweights, dbalance=dbalance, dz=dz, renormalize=ctx.renormalize), None, None, None


def route(logits, k: int, *, mask=None, renormalize: bool = True) -> Routing:
    """`route_forward` under autograd, on [..., experts] logits of any strides: weights, balance and z carry gradients."""
    mask = None if mask is None else mask.reshape(-1).contiguous()
    return Routing(*_Route.apply(_laid_out(logits.reshape(-1, logits.shape[-1])), k, mask, renormalize))


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, slots, offsets):
        ctx.save_for_backward(slots)
        return dispatch_rows(x, slots, offsets)

    @staticmethod
    @once_differentiable
    def backward(ctx, d):
        return combine_rows(_laid_out(d), ctx.saved_tensors[0]), None, None


def dispatch(x, routing: Routing):
    """Rows of [..., cols] activations in expert order, [tokens * k, cols], under autograd: expert e's are offsets[e] .. offsets[e + 1] - 1, those
    behind the last one 0."""
    return _Dispatch.apply(_laid_out(x.reshape(-1, x.shape[-1])), routing.slots, routing.offsets)


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, weights, residual, slots, offsets):
        ctx.save_for_backward(y, weights, slots, offsets)
        return combine_rows(y, slots, weights=weights, residual=residual)

    @staticmethod
    @once_differentiable
    def backward(ctx, d):
        y, weights, slots, offsets = ctx.saved_tensors
        rows, scales = ctx.needs_input_grad[:2]
        dy, dw = combine_backward(_laid_out(d), y, slots, weights, offsets, need_rows=rows, need_weights=scales) if rows or scales else (None, None)
        return dy, dw, d if ctx.needs_input_grad[2] else None, None, None


def combine(y, routing: Routing, *, residual=None):
    """Experts' outputs [tokens * k, cols] back in their tokens' rows, weighted by the router, on top of `residual` ([..., cols]), under autograd.
    The result has the residual's shape ([tokens, cols] without one)."""
    flat = None if residual is None else _laid_out(residual.reshape(-1, residual.shape[-1]))
    out = _Combine.apply(_laid_out(y), routing.weights, flat, routing.slots, routing.offsets)
    return out if residual is None else out.view(residual.shape)


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
