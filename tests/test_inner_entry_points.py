"""CPU-side checks of the inner phase's entry points: what is refused before any device call, and the closed forms."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__ as g
    g.build()
    from paper_2508_15706_b200 import inner  # declares the argument types
    return inner._L


def test_null_arguments(lib):
    from paper_2508_15706_b200 import binding as B
    N = None
    assert lib.sl_adamw_create(N, N, N, 0, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_adamw_destroy(N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_adamw_sizes(N, N, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_adamw_step(N, N, N, N, N, N, N, N, 1, 1e-3, 1.0, 0, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_adamw_read_state(N, N, N, N, N, N, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_adamw_write_state(N, N, N, N, N, N, 0, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_norm_forward(*[N] * 11) == B.SL_ERR_INVALID_ARG
    assert lib.sl_norm_backward(*[N] * 16, 0, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_norm_workspace_bytes(N, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_rotary_create(N, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_rotary_destroy(N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_rotary_apply(*[N] * 6) == B.SL_ERR_INVALID_ARG
    assert lib.sl_token_loss(*[N] * 8, 0, N) == B.SL_ERR_INVALID_ARG
    assert lib.sl_loss_workspace_bytes() >= 16


def test_adamw_tables_and_settings(lib):
    from paper_2508_15706_b200 import binding as B, inner

    def create(descs, decay=None, **k):
        v = {"param_dtype": 0, "grad_dtype": 0, "state_bits": 32, "skip_nonfinite": 1, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "max_norm": 1.0, **k}
        cfg = inner._AdamWConfig(*[v[n] for n, _ in inner._AdamWConfig._fields_])
        arr = (B._TensorDesc * len(descs))(*[B._TensorDesc(*d) for d in descs])
        out = C.c_void_p()
        st = lib.sl_adamw_create(C.byref(cfg), arr, (C.c_float * len(descs))(*(decay or [0.0] * len(descs))), len(descs), C.byref(out))
        assert out.value is None
        return st

    ok = [(4, 4, 0)]
    assert create([(64, 64, 0), (64, 64, 4092)]) == B.SL_ERR_INVALID_ARG
    assert create([(4, 4, 2)]) == B.SL_ERR_ALIGNMENT
    assert create([(0, 4, 0)]) == B.SL_ERR_INVALID_ARG and create([(4, 4, -4)]) == B.SL_ERR_INVALID_ARG
    assert create([(1 << 41, 1 << 30, 0)]) == B.SL_ERR_TOO_LARGE
    assert create(ok, decay=[-0.1]) == B.SL_ERR_INVALID_ARG and create(ok, decay=[float("nan")]) == B.SL_ERR_INVALID_ARG
    assert create(ok, state_bits=4) == B.SL_ERR_UNSUPPORTED and create(ok, param_dtype=7) == B.SL_ERR_UNSUPPORTED
    for bad in ({"beta1": 1.0}, {"beta2": -0.1}, {"eps": -1.0}, {"max_norm": float("inf")}, {"skip_nonfinite": 2}, {"beta1": float("nan")}):
        assert create(ok, **bad) == B.SL_ERR_INVALID_ARG


def test_norm_and_loss_descriptions(lib):
    from paper_2508_15706_b200 import binding as B, inner

    def norm(**k):
        d = inner._NormDesc(rows=0, cols=64, dtype=0, weight_dtype=0, gate_kind=0, alpha=1.0, eps=1e-6)
        for n, v in k.items():
            setattr(d, n, v)
        return lib.sl_norm_forward(C.byref(d), *[None] * 10)

    assert norm() == B.SL_OK  # no rows: nothing to do, nothing to check
    assert norm(cols=0) == B.SL_ERR_INVALID_ARG and norm(rows=-1) == B.SL_ERR_INVALID_ARG
    assert norm(eps=-1.0) == B.SL_ERR_INVALID_ARG and norm(alpha=float("inf")) == B.SL_ERR_INVALID_ARG
    assert norm(gate_kind=9) == B.SL_ERR_INVALID_ARG and norm(ld_x=63) == B.SL_ERR_INVALID_ARG
    assert norm(dtype=3) == B.SL_ERR_UNSUPPORTED and norm(dtype=0, weight_dtype=1) == B.SL_ERR_UNSUPPORTED
    assert norm(cols=16385) == B.SL_ERR_TOO_LARGE

    def loss(**k):
        d = inner._LossDesc(rows=0, vocab=8, dtype=0, target_bits=64, ignore_index=-100, smoothing=0.0, z=0.0, scale=1.0, mean=1)
        for n, v in k.items():
            setattr(d, n, v)
        return lib.sl_token_loss(C.byref(d), *[None] * 7, 0, None)

    assert loss() == B.SL_ERR_NOMEM  # (the workspace is asked for last)
    assert loss(vocab=0) == B.SL_ERR_INVALID_ARG and loss(rows=3) == B.SL_ERR_INVALID_ARG and loss(smoothing=-0.1) == B.SL_ERR_INVALID_ARG
    assert loss(target_bits=16) == B.SL_ERR_UNSUPPORTED and loss(vocab=(1 << 30) + 1) == B.SL_ERR_TOO_LARGE and loss(ld_grad=7) == B.SL_ERR_INVALID_ARG


def test_rotary_settings(lib):
    from paper_2508_15706_b200 import binding as B, inner

    def create(**k):
        v = {"rot_dim": 64, "layout": 0, "scaling": 0, "base": 1e4, "factor": 1.0, "original_length": 0.0, "low_turns": 1.0, "high_turns": 32.0, "magnitude": 1.0, **k}
        cfg, out = inner._RotaryConfig(*[v[n] for n, _ in inner._RotaryConfig._fields_]), C.c_void_p()
        return lib.sl_rotary_create(C.byref(cfg), C.byref(out))

    for bad in ({"rot_dim": 7}, {"rot_dim": 1026}, {"layout": 2}, {"scaling": 5}, {"base": 1.0}, {"magnitude": float("nan")}, {"scaling": 1, "factor": 0.0}, {"scaling": 2, "factor": 2.0, "rot_dim": 2},
                {"scaling": 3, "factor": 2.0}, {"scaling": 3, "factor": 2.0, "original_length": 100.0, "high_turns": 1.0}):
        assert create(**bad) == B.SL_ERR_INVALID_ARG, bad


def test_tensor_checks_refuse_with_a_message(lib):
    """The compiled checks: None passes through, everything that is not a fitting CUDA tensor raises SlError, nothing aborts."""
    import torch
    from paper_2508_15706_b200 import binding as B, inner
    f32 = torch.float32
    assert inner._ptr(None, 0, 4, f32, "x") is None and inner._rows(None, 0, 2, 2, f32, "x") == (None, 0)
    q = torch.zeros(1, 2, 3, 4)
    for bad in (torch.zeros(2, 2), torch.zeros(2, 2).to_sparse(), torch.zeros(2, 2, device="meta"), 7, "x", [1.0]):
        for call in (lambda: inner._ptr(bad, 0, 4, f32, "x"), lambda: inner._rows(bad, 0, 2, 2, f32, "x"), lambda: inner._heads(bad, q, 0, 1, 2, 4, f32, "x"),
                     lambda: inner._ptr(bad, -1, 4, f32, "x"), lambda: inner._rows(bad, -1, 2, 2, f32, "x"), lambda: inner._ptr(bad, 0, 4, "float", "x")):
            with pytest.raises(B.SlError) as e:
                call()
            assert e.value.status == B.SL_ERR_INVALID_ARG and "x must be a" in str(e.value)
    with pytest.raises(TypeError):
        inner._ptr(None, 0)
    with pytest.raises(TypeError):
        inner._rows(torch.zeros(2, 2), "0", 2, 2, f32, "x")
