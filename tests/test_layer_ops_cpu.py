"""CPU-only checks of the norm, dropout and attention entry points: what they refuse before anything is launched."""
import ctypes

import pytest
import torch

import paper_2605_16184_amd as ast
from paper_2605_16184_amd import binding as B

WS = ctypes.c_void_p(0x10000)


def _make(cls, base, kw):
    s = cls()
    for k, v in {**base, **kw}.items():
        setattr(s, k, v)
    return ctypes.byref(s)


def _rng(**kw):
    return _make(B._Rng, {"p": 0.25, "seed": 1}, kw)


def _drop(**kw):
    return _make(B._Drop, {"X": 0x1000, "Y": 0x2000, "rows": 4, "cols": 8, "ldx": 8, "ldy": 8}, kw)


@pytest.mark.parametrize("bad", [{"X": None}, {"Y": None}, {"rows": 0}, {"rows": -1}, {"cols": 0}, {"ldx": 7}, {"ldy": 7}, {"dtype": 2},
                                 {"dtype": -1}, {"Y": 0x1000, "ldy": 16}])
def test_dropout_refuses_bad_matrices(bad):
    assert ast.lib().asteria_dropout(_drop(**bad), _rng(), None) == B.INVALID_ARG


@pytest.mark.parametrize("p", [-0.1, 1.0, 1.5, float("nan"), float("inf"), 65535.6 / 65536])
def test_probabilities_that_leave_nothing_are_refused(p):
    lib = ast.lib()
    assert lib.asteria_dropout(_drop(), _rng(p=p), None) == B.INVALID_ARG
    assert lib.asteria_rms_norm(_norm(), 1e-6, _rng(p=p), None) == B.INVALID_ARG
    assert lib.asteria_rms_norm_backward(_norm_grad(), 1e-6, _rng(p=p), WS, 1 << 20, None) == B.INVALID_ARG


def test_dropout_refuses_missing_structs_and_too_many_elements():
    lib = ast.lib()
    assert lib.asteria_dropout(None, _rng(), None) == B.INVALID_ARG
    assert lib.asteria_dropout(_drop(), None, None) == B.INVALID_ARG
    assert lib.asteria_dropout(_drop(rows=1 << 30, cols=1 << 10, ldx=1 << 10, ldy=1 << 10), _rng(), None) == B.UNSUPPORTED


def _norm(**kw):
    return _make(B._Norm, {"X": 0x1000, "R": 0x2000, "W": 0x3000, "H": 0x4000, "Y": 0x5000, "rows": 4, "cols": 8, "ldx": 8, "ldr": 8,
                           "ldh": 8, "ldy": 8}, kw)


@pytest.mark.parametrize("bad", [
    {"X": None}, {"Y": None}, {"rows": 0}, {"cols": 0}, {"ldx": 7}, {"ldr": 7}, {"ldh": 7}, {"ldy": 7}, {"x_dtype": 2}, {"h_dtype": 2},
    {"w_dtype": 3}, {"y_dtype": 3}, {"y_dtype": 2}, {"y_dtype": 2, "Scale": 0x6000, "group": 64}, {"group": 128},
    {"H": 0x2000, "ldh": 16}, {"H": 0x1000, "h_dtype": 1}, {"H": 0x1000, "ldh": 16}, {"Y": 0x4000}, {"Y": 0x2000}, {"Y": 0x1000, "y_dtype": 1},
    {"Y": 0x1000, "ldy": 16}])
def test_norm_refuses_bad_arguments(bad):
    assert ast.lib().asteria_rms_norm(_norm(**bad), 1e-6, None, None) == B.INVALID_ARG


@pytest.mark.parametrize("eps", [-1e-6, float("nan"), float("inf")])
def test_norm_refuses_bad_eps(eps):
    assert ast.lib().asteria_rms_norm(_norm(), eps, None, None) == B.INVALID_ARG
    assert ast.lib().asteria_rms_norm_backward(_norm_grad(), eps, None, WS, 1 << 20, None) == B.INVALID_ARG


def test_norm_sizes_beyond_its_kernels_are_unsupported():
    lib = ast.lib()
    wide = dict(cols=16385, ldx=16385, ldr=16385, ldh=16385, ldy=16385)
    assert lib.asteria_rms_norm(_norm(**wide), 1e-6, None, None) == B.UNSUPPORTED
    assert lib.asteria_rms_norm(_norm(rows=1 << 22), 1e-6, None, None) == B.UNSUPPORTED
    wide = dict(cols=16385, ldh=16385, lddy=16385, lddh=16385, lddx=16385, lddr=16385)
    assert lib.asteria_rms_norm_backward(_norm_grad(**wide), 1e-6, None, WS, 1 << 30, None) == B.UNSUPPORTED


def _norm_grad(**kw):
    return _make(B._NormGrad, {"H": 0x1000, "dY": 0x2000, "W": 0x3000, "dH": 0x4000, "dX": 0x5000, "dR": 0x6000, "dW": 0x7000, "rows": 4,
                               "cols": 8, "ldh": 8, "lddy": 8, "lddh": 8, "lddx": 8, "lddr": 8}, kw)


@pytest.mark.parametrize("bad", [
    {"H": None}, {"dY": None}, {"rows": 0}, {"cols": 0}, {"ldh": 7}, {"lddy": 7}, {"lddh": 7}, {"lddx": 7}, {"lddr": 7}, {"x_dtype": 2},
    {"h_dtype": 2}, {"y_dtype": 2}, {"w_dtype": 2}, {"dR": 0x1000}, {"dR": 0x2000}, {"dR": 0x4000, "lddr": 16}, {"dX": 0x1000},
    {"dX": 0x4000}, {"dX": 0x6000}, {"dX": 0x2000, "x_dtype": 1}, {"dX": 0x2000, "lddx": 16}])
def test_norm_backward_refuses_bad_arguments(bad):
    assert ast.lib().asteria_rms_norm_backward(_norm_grad(**bad), 1e-6, None, WS, 1 << 20, None) == B.INVALID_ARG


def test_norm_backward_workspace():
    lib = ast.lib()
    f = lib.asteria_rms_norm_backward
    need = lib.asteria_rms_norm_backward_workspace_bytes(_norm_grad())
    assert need > 0 and lib.asteria_rms_norm_backward_workspace_bytes(_norm_grad(dW=None)) == 0
    assert f(_norm_grad(), 1e-6, None, None, 0, None) == B.WORKSPACE_TOO_SMALL
    assert f(_norm_grad(), 1e-6, None, WS, need - 1, None) == B.WORKSPACE_TOO_SMALL
    assert f(_norm_grad(), 1e-6, None, ctypes.c_void_p(0x10010), need, None) == B.INVALID_ARG


ATTN = {"Q": 0x1000, "K": 0x2000, "V": 0x3000, "O": 0x4000, "lse": 0x5000, "cu": 0x6000, "total": 6, "nseq": 2, "heads": 4, "kv_heads": 2,
        "dim": 8, "ldq": 32, "hq": 8, "ldk": 16, "hk": 8, "ldv": 16, "hv": 8, "ldo": 32, "ho": 8, "scale": 0.3}
GRAD = {"dO": 0x7000, "dQ": 0x8000, "dK": 0x9000, "dV": 0xa000, "lddo": 32, "hdo": 8, "lddq": 32, "hdq": 8, "lddk": 16, "hdk": 8, "lddv": 16,
        "hdv": 8}


@pytest.mark.parametrize("bad", [
    {"Q": None}, {"K": None}, {"V": None}, {"O": None}, {"total": 0}, {"nseq": 0}, {"heads": 0}, {"kv_heads": 0}, {"dim": 0}, {"kv_heads": 3},
    {"cu": None}, {"dtype": 2}, {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"scale": 2.0 ** -101}, {"scale": 2.0 ** 101}, {"ldq": -1}, {"hk": -8}])
def test_attention_refuses_bad_arguments(bad):
    lib = ast.lib()
    assert lib.asteria_attention(_make(B._Attn, ATTN, bad), None) == B.INVALID_ARG
    assert lib.asteria_attention_backward(_make(B._Attn, ATTN, bad), _make(B._AttnGrad, GRAD, {}), WS, 1 << 20, None) == B.INVALID_ARG


@pytest.mark.parametrize("bad", [{"ldo": 31}, {"ho": 7}, {"ldo": 0}, {"ho": 0}, {"ldo": 8, "ho": 47}])
def test_attention_refuses_outputs_that_overlap_themselves(bad):
    assert ast.lib().asteria_attention(_make(B._Attn, ATTN, bad), None) == B.INVALID_ARG


@pytest.mark.parametrize("bad", [{"dO": None}, {"dQ": None}, {"dK": None}, {"dV": None}, {"lddo": -1}, {"lddq": 31}, {"hdk": 7}, {"lddv": 15},
                                 {"lddk": 0}])
def test_attention_backward_refuses_bad_gradients(bad):
    lib = ast.lib()
    assert lib.asteria_attention_backward(_make(B._Attn, ATTN, {}), _make(B._AttnGrad, GRAD, bad), WS, 1 << 20, None) == B.INVALID_ARG
    assert lib.asteria_attention_backward(_make(B._Attn, ATTN, {"lse": None}), _make(B._AttnGrad, GRAD, {}), WS, 1 << 20, None) == B.INVALID_ARG


def test_attention_refuses_outputs_that_begin_where_another_array_does():
    lib = ast.lib()
    for name in ("Q", "K", "V"):
        assert lib.asteria_attention(_make(B._Attn, ATTN, {"O": ATTN[name]}), None) == B.INVALID_ARG
    read = [ATTN[name] for name in ("Q", "K", "V", "O")] + [GRAD["dO"]]
    for out in ("dQ", "dK", "dV"):
        for place in read + [GRAD[other] for other in ("dQ", "dK", "dV") if other != out]:
            bad = _make(B._AttnGrad, GRAD, {out: place})
            assert lib.asteria_attention_backward(_make(B._Attn, ATTN, {}), bad, WS, 1 << 20, None) == B.INVALID_ARG


def test_attention_sizes_beyond_its_kernels_are_unsupported():
    lib = ast.lib()
    wide = dict(dim=129, ldq=129 * 4, hq=129, ldo=129 * 4, ho=129)
    assert lib.asteria_attention(_make(B._Attn, ATTN, wide), None) == B.UNSUPPORTED
    assert lib.asteria_attention(_make(B._Attn, ATTN, {"nseq": 1 << 23}), None) == B.UNSUPPORTED


def test_attention_backward_workspace():
    lib = ast.lib()
    a, g = _make(B._Attn, ATTN, {}), _make(B._AttnGrad, GRAD, {})
    need = lib.asteria_attention_backward_workspace_bytes(a)
    assert need >= 6 * 4 * 4
    assert lib.asteria_attention_backward(a, g, None, 0, None) == B.WORKSPACE_TOO_SMALL
    assert lib.asteria_attention_backward(a, g, WS, need - 1, None) == B.WORKSPACE_TOO_SMALL
    assert lib.asteria_attention_backward(a, g, ctypes.c_void_p(0x10010), need, None) == B.INVALID_ARG


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(4, 8)
    q = torch.zeros(4, 2, 8)
    with pytest.raises(ValueError):
        ast.dropout(x, x, 0.1)
    with pytest.raises(ValueError):
        ast.rms_norm(x, x)
    with pytest.raises(ValueError):
        ast.rms_norm_backward(x, x)
    with pytest.raises(ValueError):
        ast.attention(q, q, q, q)
