"""CPU checks of the mixture-of-experts layer's refusals: everything is decided before a kernel is launched."""
import ctypes as C

import pytest
import torch

from paper_1712_01670_amd import binding


def _moe(**kw):
    f = dict(experts=8, top_k=2, cin=64, hidden=96, cout=64, act=1, renormalize=1, wtype=0)
    f.update(kw)
    return binding.Moe(*[f[n] for n, _ in binding.Moe._fields_])


def _layer(x=16, out=32, n=4, dtype=0, ws=256, nbytes=1 << 40, moe=None, drop=(), **kw):
    w = binding.MoeWeights(*[None if name in drop else 16 for name, _ in binding.MoeWeights._fields_])       # never dereferenced
    p = lambda v: None if v is None else C.c_void_p(v)
    return binding.lib().dc_moe_layer(C.byref(moe or _moe(**kw)), C.byref(w), p(x), p(out), None, None, n, dtype, p(ws), nbytes, None)


def test_refusals_of_the_layer():
    assert binding.lib().dc_moe_layer(None, None, None, None, None, None, 1, 0, None, 0, None) == -2
    assert _layer(x=None) == -2 and _layer(out=None) == -2 and _layer(ws=None) == -2
    for name in ("router", "up", "down"):
        assert _layer(drop=(name,)) == -2
    for name in ("up_scale", "down_scale"):
        assert _layer(drop=(name,), wtype=2) == -2
    for bad in (dict(n=0), dict(experts=0), dict(top_k=0), dict(top_k=9), dict(cin=0), dict(hidden=0), dict(cout=-1), dict(act=2), dict(act=-1),
                dict(renormalize=2), dict(wtype=3), dict(wtype=1), dict(dtype=1), dict(dtype=2), dict(out=16), dict(ws=300)):
        assert _layer(**bad) == -1, bad
    for bad in (dict(experts=257), dict(experts=64, top_k=17), dict(n=513), dict(cin=1 << 25)):
        assert _layer(**bad) == -4, bad
    need = C.c_size_t()
    assert binding.lib().dc_moe_workspace_bytes(C.byref(_moe()), 4, C.byref(need)) == 0 and need.value >= 4 * 2 * 96 * 4
    assert _layer(nbytes=need.value - 1) == -5


def test_refusals_of_the_workspace_query():
    f, need = binding.lib().dc_moe_workspace_bytes, C.c_size_t()
    assert f(None, 4, C.byref(need)) == -2 and f(C.byref(_moe()), 4, None) == -2
    assert f(C.byref(_moe()), 0, C.byref(need)) == -1 and f(C.byref(_moe(experts=300)), 4, C.byref(need)) == -4


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    moe = dict(experts=2, top_k=1, cin=8, hidden=8, cout=8, act=0, renormalize=0)
    with pytest.raises(ValueError):
        binding.dc_moe_layer(moe, torch.zeros(1, 8), torch.zeros(2, 8), torch.zeros(2, 8, 8), torch.zeros(2, 8, 8))
