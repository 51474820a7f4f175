"""GPU parity of the 8-bit fully-connected layer and of dc_quantize_rows against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_1712_01670_amd import binding, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16]


def _rows(n, k, dtype, seed, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, k, generator=g)
    if kind == "relu":
        x = x.clamp(min=0)
    if kind == "spread":                             # rows of very different size, an outlier in some
        x *= torch.logspace(-20, 20, n)[:, None]
        x[::3, k // 2] *= 50
    return x.to(dtype)


def _quantized(x):
    """(q, scales) of the definition: 64-bit quotients, 32-bit scales."""
    x = x.double().numpy()
    s = np.abs(x).max(axis=1).astype(np.float32) / np.float32(127)
    q = np.rint(x / np.where(s > 0, s, 1).astype(np.float64)[:, None])
    return q, s


def _expected(x, w, ws, bias, relu):
    q, s = _quantized(x)
    y = (q @ w.double().numpy().T) * s.astype(np.float64)[:, None] * ws.double().numpy()
    if bias is not None:
        y = y + bias.double().numpy()
    return np.maximum(y, 0) if relu else y


def _weights(cout, k, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.randint(-127, 128, (cout, k), generator=g, dtype=torch.int8)
    return w, (torch.rand(cout, generator=g) + 0.5) / (127 * math.sqrt(k)), torch.randn(cout, generator=g)


def _check(got, want, dtype, terms):
    """Roundings: the sum to fp32, two products, the bias; then the storage type's.  Each is half a step of the value it
    rounds, and no value is larger than the largest of the terms (the product, the bias, their sum)."""
    got = got.double().cpu().numpy().reshape(want.shape)
    step = torch.finfo(dtype).eps / 2
    tol = 4 * 2.0 ** -24 * terms + step * (np.abs(want) + 4 * 2.0 ** -24 * terms)
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / np.maximum(tol, 1e-300)).max())


SHAPES = [  # rows, K, cout
    (1, 1, 1), (1, 15, 3), (2, 16, 16), (1, 17, 50), (3, 63, 17), (1, 64, 10), (5, 65, 33), (16, 100, 50), (17, 127, 15),
    (1, 1152, 100), (2, 1151, 100), (4, 1153, 129), (1, 9216, 512), (8, 4096, 1000), (15, 1024, 1000), (16, 2048, 256), (31, 1000, 77),
    (33, 129, 257), (64, 576, 128), (65, 64, 64), (63, 4100, 40), (100, 333, 111), (127, 250, 130), (128, 512, 128), (129, 515, 127),
    (200, 2048, 64), (257, 192, 300), (512, 768, 260), (1000, 36, 24), (1023, 517, 131), (2049, 256, 256), (777, 4099, 255), (3, 25088, 48),
    (1, 131072, 5), (18, 70000, 9), (300, 17000, 20), (40, 5000, 4096),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_layer_matches_the_definition(shape, dtype):
    n, k, cout = shape
    print(f"[fc quant] {shape} {dtype}", flush=True)
    x = _rows(n, k, dtype, n + k + cout, "relu" if cout % 2 else "normal")
    w, ws, bias = _weights(cout, k, n * 3 + k)
    for b, relu in ((bias, True), (None, False)):
        got = binding.dc_fc_quant_layer(x.to(DEV), w.to(DEV), ws.to(DEV), None if b is None else b.to(DEV), relu)
        assert got.shape == (n, 1, 1, cout) and got.dtype == dtype
        plain = _expected(x, w, ws, None, False)
        want = _expected(x, w, ws, b, relu)
        _check(got, want, dtype, np.abs(plain) + (0 if b is None else np.abs(b.double().numpy())) + np.abs(want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (5, 16), (9, 250), (64, 256), (33, 1000), (7, 1024), (18, 1025), (5, 4096), (3, 4111),
                                   (2, 16384), (2, 16400), (1, 65536), (2, 70001), (1, 131072), (3000, 64), (1, 200)])
def test_quantized_rows_are_exact(shape, dtype):
    print(f"[quantize] {shape} {dtype}", flush=True)
    x = _rows(*shape, dtype, sum(shape), "spread" if dtype == torch.float32 else "normal")
    q, s = binding.dc_quantize_rows(x.to(DEV))
    want_q, want_s = _quantized(x)
    assert (s.cpu().numpy() == want_s).all()
    assert (q.cpu().numpy() == want_q).all()


def test_ties_go_to_the_even_integer():
    """Rows of half-integers times a power of two and 127 of them: every quotient but the largest is a tie."""
    x = torch.arange(-126.5, 127, 1.0).repeat(3, 1) * torch.tensor([1.0, 2.0 ** -40, 2.0 ** 90])[:, None]
    x = torch.cat([x, 127.0 * torch.tensor([[1.0], [2.0 ** -40], [2.0 ** 90]])], dim=1)
    q, s = binding.dc_quantize_rows(x.to(DEV))
    assert s.cpu().tolist() == [1.0, 2.0 ** -40, 2.0 ** 90]
    assert (q.cpu().double() == torch.round(torch.cat([torch.arange(-126.5, 127, 1.0), torch.tensor([127.0])]).double())).all()


def test_borders_of_a_rounding():
    """Values next to the borders between two integers, a step of fp32 to either side: decided as in 64 bits."""
    g = torch.Generator().manual_seed(5)
    top = torch.rand(64, generator=g) + 0.5
    s = top / 127
    near = ((torch.randint(0, 126, (64, 500), generator=g) + 0.5).double() * s.double()[:, None]).float()
    x = torch.cat([near, torch.nextafter(near, torch.tensor(0.0)), -torch.nextafter(near, torch.tensor(9.0)), top[:, None]], dim=1)
    for scale in (1.0, 2.0 ** -110, 2.0 ** 100):
        y = x * scale
        q, s = binding.dc_quantize_rows(y.to(DEV))
        want_q, want_s = _quantized(y)
        assert (s.cpu().numpy() == want_s).all() and (q.cpu().numpy() == want_q).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 3, 40, 300])
def test_rows_without_a_number(dtype, n):
    """Zeros give the bias, NaN and infinities NaN, in their row alone; tiny rows saturate and stay finite."""
    k, cout = 333, 70
    x = _rows(n, k, dtype, 3)
    w, ws, bias = _weights(cout, k, 4)
    clean = binding.dc_fc_quant_layer(x.to(DEV), w.to(DEV), ws.to(DEV), bias.to(DEV), False).cpu()
    for value in (float("nan"), float("inf"), float("-inf"), 0.0, 1e-44):
        y = x.clone()
        at = n // 2
        if value == 0.0 or value == 1e-44:
            y[at] = value
        else:
            y[at, k - 1] = value
        got = binding.dc_fc_quant_layer(y.to(DEV), w.to(DEV), ws.to(DEV), bias.to(DEV), False).cpu()
        if value == 0.0 or (value == 1e-44):
            assert torch.isfinite(got[at]).all()
            assert torch.equal(got[at].flatten(), bias.to(dtype)) or value != 0.0
        else:
            assert torch.isnan(got[at]).all()
            assert torch.isnan(binding.dc_fc_quant_layer(y.to(DEV), w.to(DEV), ws.to(DEV), bias.to(DEV), True).cpu()[at]).all()
        keep = [r for r in range(n) if r != at]
        assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_do_not_depend_on_each_other(dtype):
    """The sums are exact: a row alone, among a few and among many gives the same bits."""
    k, cout = 1000, 300
    x = _rows(600, k, dtype, 9)
    w, ws, bias = (t.to(DEV) for t in _weights(cout, k, 10))
    x = x.to(DEV)
    whole = binding.dc_fc_quant_layer(x, w, ws, bias, True)
    for n in (1, 2, 4, 8, 16, 17, 33, 64, 65, 130, 300):
        assert torch.equal(binding.dc_fc_quant_layer(x[:n].contiguous(), w, ws, bias, True), whole[:n]), n


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 7, 40, 200])
def test_any_alignment(dtype, n):
    """Rows, weights, scales, bias and output that start anywhere their element type allows; nothing is written outside."""
    k, cout = 256, 96
    es = torch.finfo(dtype).bits // 8
    x = _rows(n, k, dtype, 1)
    w, ws, bias = _weights(cout, k, 2)
    want = binding.dc_fc_quant_layer(x.to(DEV), w.to(DEV), ws.to(DEV), bias.to(DEV), False)

    def shifted(t, by):
        buf = torch.zeros(t.numel() + 64, dtype=t.dtype, device=DEV)
        buf[by:by + t.numel()] = t.flatten().to(DEV)
        return buf[by:by + t.numel()].view(t.shape)

    L = binding.lib()
    for xo, wo, so in ((1, 1, 1), (3, 7, 2), (16 // es, 8, 3)):
        xs, wsh, ss, bs = shifted(x, xo), shifted(w, wo), shifted(ws, so), shifted(bias, so)
        out = torch.full((n * cout + 64,), 7.0, dtype=dtype, device=DEV)
        o = out[xo:xo + n * cout]
        need = binding.C.c_size_t()
        assert L.dc_fc_quant_workspace_bytes(n, k, cout, binding.C.byref(need)) == 0
        space = torch.empty(max(need.value, 256), dtype=torch.uint8, device=DEV)
        assert L.dc_fc_quant_layer(xs.data_ptr(), wsh.data_ptr(), ss.data_ptr(), bs.data_ptr(), o.data_ptr(), n, k, cout, 0,
                                   1 if dtype == torch.bfloat16 else 0, space.data_ptr(), need.value, binding._stream()) == 0
        torch.cuda.synchronize()
        assert torch.equal(o.view(want.shape), want)
        assert (out[:xo] == 7).all() and (out[xo + n * cout:] == 7).all()


@pytest.mark.parametrize("n", [1, 20, 300])
def test_captured_calls(n):
    """Two layers recorded into two graphs, replayed in turn with new inputs and eager work between: as the eager calls."""
    k, mid, cout = 500, 200, 60
    w1, s1, b1 = (t.to(DEV) for t in _weights(mid, k, 1))
    w2, s2, b2 = (t.to(DEV) for t in _weights(cout, mid, 2))
    xs = [_rows(n, k, torch.bfloat16, 20 + i).to(DEV) for i in range(4)]

    def net(x):
        return binding.dc_fc_quant_layer(binding.dc_fc_quant_layer(x, w1, s1, b1, True), w2, s2, b2, False)

    want = [net(x) for x in xs]
    torch.cuda.synchronize()
    static = [torch.empty_like(xs[0]) for _ in range(2)]
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(net(static[i]))
        graphs.append(g)
    for rep in range(4):
        for i in range(2):
            static[i].copy_(xs[(rep + i) % 4])
            graphs[i].replay()
        eager = net(xs[rep])
        torch.cuda.synchronize()
        assert torch.equal(eager, want[rep])
        for i in range(2):
            assert torch.equal(outs[i], want[(rep + i) % 4])


def test_two_streams_at_once():
    k, cout = 2048, 512
    w, s, b = (t.to(DEV) for t in _weights(cout, k, 1))
    xs = [_rows(n, k, torch.float32, n).to(DEV) for n in (5, 90)]
    want = [binding.dc_fc_quant_layer(x, w, s, b, True) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(binding.dc_fc_quant_layer(xs[i], w, s, b, True))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


@pytest.mark.parametrize("dtype", TYPES)
def test_a_head_as_it_is_used(dtype):
    """Weights rounded once by dc_quantize_rows, then three layers and a softmax over the maps of eight streams: near the
    fp32 layers of the same weights (an 8-bit step is 1/254 of a row's largest value either side)."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(8, 6, 6, 256, generator=g).clamp(min=0).to(dtype).to(DEV)
    sizes = [6 * 6 * 256, 512, 512, 100]
    q, full = x, x.float()
    for i in range(3):
        w = (torch.randn(sizes[i + 1], sizes[i], generator=g) * math.sqrt(2 / sizes[i])).to(DEV)
        b = (torch.randn(sizes[i + 1], generator=g) * 0.1).to(DEV)
        wq, ws = binding.dc_quantize_rows(w)
        q = binding.dc_fc_quant_layer(q, wq, ws, b, i < 2)
        full = binding.dc_fc_layer(full, w, b, i < 2)
    # two roundings a layer, each uniform in +-1/2 step of a row whose largest value is a few times its deviation: under 2 % of
    # the outputs' norm a layer
    err = (q.float() - full).norm() / full.norm()
    assert err < 0.06, float(err)
    p = binding.dc_softmax_layer(q)
    assert (p.float().sum(-1) - 1).abs().max() < 100 * 2.0 ** -9


@pytest.mark.parametrize("mode", ["host", "maps", "replayed", "plain"])
@pytest.mark.parametrize("dtype", [binding.DC_F32, binding.DC_BF16])
@pytest.mark.parametrize("n", [1, 3])
def test_a_stack_whose_head_is_in_8_bits(n, dtype, mode):
    """StackRunner(fc_quant=True): every frame's fully-connected outputs are dc_fc_quant_layer's of their inputs, bit for bit, the
    layers in front of them are those of the plain runner, and so is a runner made without it."""
    layers = synth.alexnet(n_classes=40, width=0.25)
    H = W = 227
    ws, bs = synth.he_weights(layers, 5, bias_scale=0.05, input_shape=(H, W, 3))
    kw = dict(dtype=dtype)
    if mode in ("maps", "replayed"):
        kw.update(device_plan=True, exact_masks=True)
    if mode == "plain":
        kw.update(overlap=False)
    runner = binding.StackRunner(layers, ws, bs, n, H, W, 3, fc_quant=True, **kw)
    plain = binding.StackRunner(layers, ws, bs, n, H, W, 3, **kw)
    if mode == "replayed":
        runner.set_replay(1)
    blocks = {i: binding.dc_quantize_rows(runner.w[i].reshape(runner.w[i].shape[0], -1)) for i, L in enumerate(layers) if L["type"] == synth.FC}
    rng = np.random.default_rng(0)
    base = rng.integers(0, 256, (n, H + 16, W + 16, 3), dtype=np.uint8)
    frames = [torch.from_numpy(np.ascontiguousarray(base[:, f:f + H, f:f + W])).to(DEV) for f in range(6)]
    for f in frames * (4 if mode == "replayed" else 1):      # (a recording is replayed when its buffers and plan area come round again)
        got = runner.step(f)
        torch.cuda.synchronize()
        want = plain.step(f)
        torch.cuda.synchronize()
        for i, L in enumerate(layers):
            x, y = got[L["in0"]], got[i + 1]
            if L["type"] == synth.FC:
                q, s = blocks[i]
                assert torch.equal(y.view(n, 1, 1, -1), binding.dc_fc_quant_layer(x, q, s, runner.b[i], bool(L["relu"]))), i
            elif i < min(blocks):
                assert torch.equal(y, want[i + 1]), i
        assert torch.isfinite(got[-1].float()).all()
    if mode == "replayed":
        assert runner.overlap_counters().replayed > 0


def test_a_stack_needs_no_plain_weights_behind_a_packed_block():
    """The plain weights of a layer in 8-bit integers may be gone: NULL entries give the same bits; without a block they are refused."""
    layers = synth.alexnet(n_classes=24, width=0.25)
    H = W = 227
    ws, bs = synth.he_weights(layers, 7, bias_scale=0.05, input_shape=(H, W, 3))
    frame = torch.randint(0, 256, (2, H, W, 3), dtype=torch.uint8, generator=torch.Generator().manual_seed(3)).to(DEV)
    fc = [i for i, L in enumerate(layers) if L["type"] == synth.FC]
    outs = []
    for gone in (False, True):
        runner = binding.StackRunner(layers, ws, bs, 2, H, W, 3, fc_quant=True, overlap=False)
        for i in fc if gone else ():
            runner._wp[i] = None
        outs.append(runner.step(frame)[-1].clone())
        torch.cuda.synchronize()
    assert fc and torch.equal(*outs)
    runner = binding.StackRunner(layers, ws, bs, 2, H, W, 3, overlap=False)
    runner._wp[fc[0]] = None
    with pytest.raises(binding.DcError):
        runner.step(frame)


def test_a_block_of_no_channels_is_refused():
    with pytest.raises(binding.DcError):
        binding.dc_pack_fc_weights(torch.zeros(0, 8, device=DEV))


LONG = [(17, 8208, 65), (33, 131072, 20), (64, 9216, 1000), (65, 4096, 1), (66, 4101, 70), (130, 4112, 100), (250, 8191, 64), (1000, 5000, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", LONG)
def test_long_rows_shared_by_workgroups(shape, dtype):
    """Tiles whose K several workgroups share: as the definition, the same bits call after call in one workspace, and those of single rows."""
    n, k, cout = shape
    x = _rows(n, k, dtype, n, "relu")
    w, s, b = _weights(cout, k, n)
    dev = [t.to(DEV) for t in (x, w, s, b)]
    got = binding.dc_fc_quant_layer(*dev, True)
    want = _expected(x, w, s, b, True)
    q, sc = _quantized(x)
    terms = np.abs((q @ w.double().numpy().T) * sc.astype(np.float64)[:, None] * s.double().numpy()) + b.double().abs().numpy()
    _check(got, want, dtype, terms)
    for _ in range(5):
        assert torch.equal(binding.dc_fc_quant_layer(*dev, True), got)
    for r in (0, n - 1):
        assert torch.equal(binding.dc_fc_quant_layer(dev[0][r:r + 1].contiguous(), *dev[1:], True)[0], got[r])


def test_long_rows_on_two_streams_and_in_graphs():
    """Workspaces and counters of calls that overlap are their own; a replayed graph clears its counters each time."""
    k, cout = 8192, 300
    w, s, b = (t.to(DEV) for t in _weights(cout, k, 4))
    xs = [_rows(n, k, torch.bfloat16, n).to(DEV) for n in (40, 150)]
    want = [binding.dc_fc_quant_layer(x, w, s, b, False) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(binding.dc_fc_quant_layer(xs[i], w, s, b, False))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i]) for i in range(2) for g in got[i])
    static = torch.zeros_like(xs[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = binding.dc_fc_quant_layer(static, w, s, b, False)
    for rep in range(4):
        static.copy_(xs[1] if rep % 2 == 0 else -xs[1])
        g.replay()
        eager = binding.dc_fc_quant_layer(xs[0], w, s, b, False)
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0])
        assert torch.equal(out, binding.dc_fc_quant_layer(xs[1] if rep % 2 == 0 else -xs[1], w, s, b, False))
    assert torch.equal(binding.dc_fc_quant_layer(xs[1], w, s, b, False), want[1])


@pytest.mark.parametrize("shape", [(6300, 2064, 2000), (6300, 2060, 2000), (4100, 2064, 2000)])
def test_large_products_of_any_row_length(shape):
    """Rows of many cache lines that begin inside one: as 64 rows at a time, bit for bit."""
    n, k, cout = shape
    x = _rows(n, k, torch.bfloat16, 1).to(DEV)
    w, s, b = (t.to(DEV) for t in _weights(cout, k, 2))
    got = binding.dc_fc_quant_layer(x, w, s, b, False)
    for r in (0, 1000, n - 64):
        assert torch.equal(got[r:r + 64], binding.dc_fc_quant_layer(x[r:r + 64], w, s, b, False)), r


@pytest.mark.parametrize("shape", [(64, 50000, 8000), (33, 131056, 3000)])
def test_few_rows_of_very_long_weights(shape):
    """Whole vectors that end inside a cache line, 2.6e10 and 1.3e10 products, at most 64 rows: nothing is written behind the
    workspace that the query asks for, and the bits are those of 16 rows at a time."""
    n, k, cout = shape
    print(f"[fc quant long] {shape}", flush=True)
    x = _rows(n, k, torch.bfloat16, 1, "relu").to(DEV)
    w = torch.randint(-127, 128, (cout, k), generator=torch.Generator(device=DEV).manual_seed(2), dtype=torch.int8, device=DEV)
    s, b = torch.rand(cout, device=DEV) + 0.5, torch.randn(cout, device=DEV)
    need = binding.C.c_size_t()
    L = binding.lib()
    assert L.dc_fc_quant_workspace_bytes(n, k, cout, binding.C.byref(need)) == 0
    space = torch.full((need.value + (1 << 20),), 77, dtype=torch.uint8, device=DEV)
    out = torch.empty(n, cout, dtype=torch.bfloat16, device=DEV)
    assert L.dc_fc_quant_layer(x.data_ptr(), w.data_ptr(), s.data_ptr(), b.data_ptr(), out.data_ptr(), n, k, cout, 0, binding.DC_BF16, space.data_ptr(),
                               need.value, binding._stream()) == 0
    torch.cuda.synchronize()
    assert (space[need.value:] == 77).all()
    for r in range(0, n, 16):
        assert torch.equal(out[r:r + 16], binding.dc_fc_quant_layer(x[r:r + 16], w, s, b, False).view(-1, cout)), r


@pytest.mark.parametrize("dtype", [binding.DC_F32, binding.DC_BF16])
@pytest.mark.parametrize("size,channels,n", [(32, 16, 70), (31, 17, 130)])
def test_a_stack_of_many_streams(size, channels, n, dtype):
    """More than 64 streams, and a head whose weights are more than a stage's scratch memory: rows of whole vectors, which need no copy of
    them, and rows of an odd length, which are taken 64 streams at a time.  Bits of the single call."""
    print(f"[stack of many streams] {size} {channels} {n} {dtype}", flush=True)
    layers = synth._chain([("c", channels, 3, 1, 1)], 3)
    layers += [synth._fc(channels, 2200, True, 1), synth._fc(2200, 30, False, 2)]
    ws, bs = synth.he_weights(layers, 5, bias_scale=0.05, input_shape=(size, size, 3))
    assert ws[1].size > 33 << 20
    runner = binding.StackRunner(layers, ws, bs, n, size, size, 3, dtype=dtype, fc_quant=True)
    frame = torch.randint(0, 256, (n, size, size, 3), dtype=torch.uint8, generator=torch.Generator().manual_seed(3)).to(DEV)
    for _ in range(2):
        got = runner.step(frame)
        torch.cuda.synchronize()
        for i in (1, 2):
            q, s = binding.dc_quantize_rows(runner.w[i].reshape(runner.w[i].shape[0], -1))
            assert torch.equal(got[i + 1].view(n, 1, 1, -1), binding.dc_fc_quant_layer(got[i], q, s, runner.b[i], i == 1)), i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 5, 64, 70, 300])
def test_scales_at_opposite_ends_of_the_range(n, dtype):
    """Large weights for small rows and the other way round: the product of the sum and one scale leaves fp32, the result does not."""
    k, cout = 5000, 130
    x = _rows(n, k, dtype, n, "relu")
    w, s, b = _weights(cout, k, 2)
    w[5] = 0
    for row, weight in ((1e-30, 1e41), (1e-25, 1e38), (2.0 ** -95, 2.0 ** 135), (1e30, 1e-34), (1e20, 1e-40), (2.0 ** 110, 2.0 ** -100)):
        xs, ss = (x.double() * row).to(dtype), (s.double() * weight).float()
        ss[::7] = s[::7]                             # ordinary channels beside them,
        ss[3] = 0                                    # and one without weights
        got = binding.dc_fc_quant_layer(xs.to(DEV), w.to(DEV), ss.to(DEV), b.to(DEV), False)
        terms = np.abs(_expected(xs, w, ss, None, False)) + b.double().abs().numpy()
        assert np.isfinite(terms).all() and terms.max() < 1e38
        _check(got, _expected(xs, w, ss, b, False), dtype, terms)
    # both large: the outputs are infinite where there is anything, and a sum of zero gives the bias
    xs, ss = (x.double() * 1e30).to(dtype), (s.double() * 1e41).float()
    got = binding.dc_fc_quant_layer(xs.to(DEV), w.to(DEV), ss.to(DEV), b.to(DEV), False).cpu().view(n, cout)
    q, _ = _quantized(xs)
    sums = q @ w.double().numpy().T
    assert torch.equal(got[:, 5], b[5].to(dtype).expand(n))
    assert (got.double().numpy()[sums != 0] == np.sign(sums[sums != 0]) * np.inf).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(8300, 200, 50), (8200, 208, 64), (3100, 528, 1000), (3137, 515, 900), (12400, 272, 4090), (12300, 259, 4100),
                                   (4100, 272, 1300), (70, 33, 70000), ((1 << 20) + 30, 17, 5)])
def test_products_of_many_tiles(shape, dtype):
    """The GEMM's other tiles, with ragged rows and channels and rows of weights in whole vectors and not: 128 x 64 (up to 64
    channels), 128 x 128 in three stages (as many tiles as CUs) and in two, 256 x 256 (many); more channels than a launch of the
    copy has, and more rows than a launch of the rounding.  Rows from every part, the last tile's among them."""
    n, k, cout = shape
    print(f"[fc quant tiles] {shape} {dtype}", flush=True)
    x = _rows(n, k, dtype, n, "relu")
    w, s, b = _weights(cout, k, 3)
    rows = torch.unique(torch.cat([torch.arange(0, n, n // 40), torch.arange(n - 20, n)]))
    for bias, relu in ((b, True), (None, False)):
        got = binding.dc_fc_quant_layer(x.to(DEV), w.to(DEV), s.to(DEV), None if bias is None else bias.to(DEV), relu).cpu()[rows]
        assert got.shape == (len(rows), 1, 1, cout)
        plain = _expected(x[rows], w, s, None, False)
        want = _expected(x[rows], w, s, bias, relu)
        _check(got, want, dtype, np.abs(plain) + (0 if bias is None else np.abs(bias.double().numpy())) + np.abs(want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [300, 1000, 2001, 4090, 8191, 20000])
def test_many_quantized_rows_are_exact(k, dtype):
    """Every number of lanes that share a row of many, and rows that are read in two passes of a workgroup."""
    print(f"[quantize many] {k} {dtype}", flush=True)
    x = _rows(2051, k, dtype, k)
    q, s = binding.dc_quantize_rows(x.to(DEV))
    want_q, want_s = _quantized(x)
    assert (s.cpu().numpy() == want_s).all() and (q.cpu().numpy() == want_q).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(3, 131072, 5), (16, 70001, 9), (40, 100001, 7), (60, 70001, 37), (70, 70001, 33), (70, 131072, 3)])
def test_rows_that_are_read_twice(shape, dtype):
    """Rows too long for a workgroup's registers, behind either kernel."""
    n, k, cout = shape
    print(f"[fc quant long rows] {shape} {dtype}", flush=True)
    x = _rows(n, k, dtype, n)
    w, s, b = _weights(cout, k, 3)
    got = binding.dc_fc_quant_layer(x.to(DEV), w.to(DEV), s.to(DEV), b.to(DEV), False)
    want = _expected(x, w, s, b, False)
    _check(got, want, dtype, np.abs(_expected(x, w, s, None, False)) + np.abs(b.double().numpy()) + np.abs(want))
