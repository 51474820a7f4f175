"""CPU checks of the 8-bit fully-connected layer's refusals: everything is decided before a kernel is launched."""
import ctypes as C
import os
import subprocess

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


# What the launches of one call write, from the kernels' indexing: (area, bytes from its start on).
_PLAN_CHECK = r"""
#include <cstdio>
#include <cstdlib>
#include "dc_fc_quant_plan.h"
using namespace dc;
static int check(int n, int K, int cout, bool vectors, size_t room) {
    const I8Plan p = i8_plan(n, K, cout, vectors, room);
    const size_t width = ((size_t)K + 127) / 128 * 128;
    auto fail = [&](const char* why) { printf("%s: %d rows, %d -> %d, vectors %d\n", why, n, K, cout, vectors); return 1; };
    if (p.bytes > room) return fail("more than the query says");
    if (p.width != width) return fail("row width");
    if (n == 1) return p.bytes || p.splits != 1 ? fail("one row needs nothing") : 0;
    if (!p.few && !vectors && !p.copy) return fail("the GEMM takes rows of whole vectors");
    if (p.few && (n > 64 || p.splits != 1 || p.copy)) return fail("few rows");
    struct Write { const I8Plan::Area* area; size_t bytes; } w[5] = {
        // tiles of 16 rows in the one form (what is not a row is read, too), rows in the other
        {&p.rows, p.few ? ((size_t)n + 15) / 16 * 16 * width : (size_t)n * width},
        {&p.scales, (size_t)n * 4},
        {&p.weights, p.copy ? (size_t)cout * width : 0},
        {&p.part, p.splits > 1 ? ((size_t)n + 63) / 64 * (((size_t)cout + 63) / 64) * p.splits * 64 * 64 * 4 : 0},
        {&p.done, p.splits > 1 ? ((size_t)n + 63) / 64 * (((size_t)cout + 63) / 64) * 4 : 0}};
    size_t end = 0;
    for (const Write& v : w) {
        if (!v.bytes) continue;
        if (v.area->at % 256) return fail("alignment");
        if (v.area->at < end) return fail("areas overlap");
        end = v.area->at + v.bytes;
        if (v.bytes > v.area->bytes || end > p.bytes) return fail("written behind the end");
    }
    return 0;
}
int main(int argc, char** argv) {
    if (argc == 4) { printf("%zu\n", i8_workspace(atoi(argv[1]), atoi(argv[2]), atoi(argv[3]))); return 0; }
    if (i8_rows(5, 131072, 8, true, 100000) || i8_rows(1, 131072, 8, true, 0) != 1) return 2;
    const int Ks[] = {1, 15, 16, 17, 100, 128, 1000, 1024, 3968, 3969, 4096, 4097, 4112, 8064, 8065, 8080, 8192, 9216, 9217, 16400, 25088, 50000, 65536, 100001,
                      131056, 131071, 131072};
    const int Cs[] = {1, 5, 63, 64, 65, 129, 500, 1000, 2048, 3000, 4096, 5000, 8000, 8192, 8193, 16384, 16448, 40000, 65535, 1 << 20};
    int bad = 0;
    for (int i = 0; i < 320; ++i) {
        const int n = i < 300 ? i + 1 : 300 << (i - 299 < 15 ? i - 299 : 15);
        for (int K : Ks)
            for (int c : Cs) {
                if (((long)n * c) >> 34) continue;
                const size_t room = i8_workspace(n, K, c);
                bad += check(n, K, c, false, room);
                if (K % 16 == 0) bad += check(n, K, c, true, room);
                // the 32 MiB that a layer of a stack has, whatever its size: all rows at once, or parts
                for (int vectors = 0; vectors <= (K % 16 == 0); ++vectors) {
                    const int part = i8_rows(n, K, c, vectors, 32 << 20);
                    if (part != n && part != 64) { printf("%d rows at once: %d, %d -> %d\n", part, n, K, c); ++bad; }
                    else bad += check(part, K, c, vectors, 32 << 20) + (n % part ? check(n % part, K, c, vectors, 32 << 20) : 0);
                }
                if (bad > 10) return 1;
            }
    }
    return bad ? 1 : 0;
}
"""


def test_every_area_of_a_call_lies_in_its_workspace(tmp_path):
    """One to 300 rows and many more, lengths and channels up to the limits, weights in whole vectors and not: what the rounding, the
    copy of the weights and the shared sums write lies apart, and inside what dc_fc_quant_workspace_bytes asks for."""
    source, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    source.write_text(_PLAN_CHECK)
    csrc = os.path.join(os.path.dirname(os.path.abspath(binding.__file__)), "csrc")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", csrc, str(source), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    need = C.c_size_t()
    for shape in ((1, 100, 8), (40, 100, 8), (64, 50000, 8000), (64, 131056, 3000), (32, 131056, 8000), (17, 8080, 65), (65, 9216, 4096), (300, 4099, 1000)):
        assert binding.lib().dc_fc_quant_workspace_bytes(*shape, C.byref(need)) == 0
        assert need.value == int(subprocess.run([str(exe), *map(str, shape)], capture_output=True, text=True, check=True).stdout)
