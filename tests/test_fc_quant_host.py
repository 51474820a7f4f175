"""CPU checks of the 8-bit fully-connected layer's refusals: everything is decided before a kernel is launched."""
import ctypes as C

import pytest
import torch

from paper_1712_01670_amd import binding


def _layer(x=16, w=16, s=16, b=None, out=32, n=40, k=100, cout=8, relu=0, dtype=0, ws=256, nbytes=1 << 30):
    p = lambda v: None if v is None else C.c_void_p(v)       # never dereferenced: validation fails first
    return binding.lib().dc_fc_quant_layer(p(x), p(w), p(s), p(b), p(out), n, k, cout, relu, dtype, p(ws), nbytes, None)


def test_refusals_of_the_layer():
    for name in ("x", "w", "s", "out"):
        assert _layer(**{name: None}) == -2
    assert _layer(ws=None) == -2
    for bad in (dict(n=0), dict(n=-1), dict(k=0), dict(cout=0), dict(cout=-3), dict(relu=2), dict(relu=-1), dict(dtype=2), dict(dtype=-1)):
        assert _layer(**bad) == -1, bad
    assert _layer(k=131073) == -4                            # a sum could leave 32 bits
    assert _layer(out=16) == -1                              # in place
    assert _layer(ws=264) == -1                              # a workspace that is not aligned
    need = C.c_size_t()
    assert binding.lib().dc_fc_quant_workspace_bytes(40, 100, 8, C.byref(need)) == 0 and need.value >= 40 * 100
    assert _layer(nbytes=need.value - 1) == -5


def test_refusals_of_the_workspace_query():
    f, need = binding.lib().dc_fc_quant_workspace_bytes, C.c_size_t()
    assert f(4, 100, 8, None) == -2
    assert f(0, 100, 8, C.byref(need)) == -1 and f(4, 0, 8, C.byref(need)) == -1 and f(4, 100, 0, C.byref(need)) == -1
    assert f(4, 131073, 8, C.byref(need)) == -4
    assert f(2 ** 24, 131072, 8, C.byref(need)) == 0 and need.value >= 2 ** 41          # sizes are counted in 64 bits
    assert f(2 ** 24 + 1, 16, 8, C.byref(need)) == -4 and f(4, 16, 2 ** 20 + 1, C.byref(need)) == -4 and f(2 ** 24, 16, 2 ** 11, C.byref(need)) == -4


def test_refusals_of_the_rounding():
    f, one = binding.lib().dc_quantize_rows, C.c_void_p(16)
    assert f(None, 1, 1, 0, one, one, None) == -2 and f(one, 1, 1, 0, None, one, None) == -2 and f(one, 1, 1, 0, one, None, None) == -2
    assert f(one, 0, 1, 0, one, one, None) == -1 and f(one, 1, 0, 0, one, one, None) == -1 and f(one, 1, 1, 2, one, one, None) == -1
    assert f(one, 1, 131073, 0, C.c_void_p(32), one, None) == -4 and f(one, 1 << 31, 8, 0, C.c_void_p(32), one, None) == -4
    assert f(one, 1, 8, 0, one, C.c_void_p(64), None) == -1                              # in place


def test_refusals_of_the_packed_block():
    f, g, one, n = binding.lib().dc_packed_fc_bytes, binding.lib().dc_pack_fc_weights, C.c_void_p(16), C.c_size_t()
    assert f(100, 7, C.byref(n)) == 0 and n.value == 704 + 28                            # 700 bytes, the scales from 704 on
    assert f(100, 7, None) == -2 and f(0, 7, C.byref(n)) == -1 and f(8, 0, C.byref(n)) == -1 and f(131073, 7, C.byref(n)) == -4
    assert g(None, 8, 8, 0, one, None) == -2 and g(one, 8, 8, 0, None, None) == -2 and g(one, 8, 8, 0, C.c_void_p(24), None) == -1
    assert g(one, 8, 8, 5, C.c_void_p(32), None) == -1 and g(one, 0, 8, 0, C.c_void_p(32), None) == -1


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    x, w, s = torch.zeros(2, 8), torch.zeros(3, 8, dtype=torch.int8), torch.zeros(3)
    with pytest.raises(ValueError):
        binding.dc_fc_quant_layer(x, w, s, None, False)
    with pytest.raises(ValueError):
        binding.dc_quantize_rows(x)
