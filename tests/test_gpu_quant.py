"""The output layer in 4 bits against its definition in 64 bits (needs a B200)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fef():
    import paper_2605_14305_b200 as lib

    lib.load(build_if_missing=True)
    return lib


def _values(weight, group, zero_points):
    """(values [V, d], scales [V, d / group]) of the quantised layer in 64 bits, on the host."""
    V, d = weight.shape
    w = weight.double().cpu().view(V, d // group, group)
    if zero_points:
        lo, hi = w.amin(-1).clamp(max=0.0), w.amax(-1).clamp(min=0.0)
        s = ((hi - lo) / 15).to(torch.bfloat16).double()
        z = torch.where(s > 0, (-lo / s).round().clamp(0, 15), torch.zeros_like(s))
    else:
        s = (w.abs().amax(-1) / 7).to(torch.bfloat16).double()
        z = torch.full_like(s, 8.0)
    q = torch.where(s[..., None] > 0, (w / s[..., None]).round() + z[..., None], z[..., None]).clamp(0, 15)
    return ((q - z[..., None]) * s[..., None]).view(V, d), s


SHAPES = [(1, 32, 32), (3, 64, 32), (33, 96, 32), (31, 128, 128), (65, 192, 64), (257, 1056, 32), (1000, 1152, 128), (100, 4096, 64)]


@pytest.mark.parametrize("V,d,group", SHAPES)
@pytest.mark.parametrize("zero_points", [False, True])
def test_quantized_values(fef, V, d, group, zero_points):
    g = torch.Generator(device="cuda").manual_seed(V + d)
    w = torch.randn((V, d), generator=g, device="cuda") + 0.3
    w = torch.where(torch.rand((V, d), generator=g, device="cuda") < 0.3, w.mul(4).round().div(4), w).to(torch.bfloat16)  # (ties)
    layer = fef.fef_lmhead_quantize(w, group, zero_points)
    got = fef.fef_lmhead_dequantize(layer)
    torch.cuda.synchronize()
    ref, s = _values(w, group, zero_points)
    assert torch.equal(got.cpu().double(), ref)              # bit for bit: (q - z) s is exact in binary32
    # half a step of the scale, and what rounding the scale to bfloat16 moves the largest weight by (15 steps at most)
    off = (ref.view(V, -1, group) - w.cpu().double().view(V, -1, group)).abs()
    assert (off <= s[..., None] * (0.5 + 15 * 2.0 ** -8 + (0.5 if zero_points else 0.0))).all()
    blocks, Vp = (d + 127) // 128, (V + 31) // 32 * 32
    flat = layer.scale.float().cpu().transpose(0, 1).reshape(Vp, -1)
    assert torch.equal(flat[:V, :d // group].double(), s) and (flat[V:] == 0).all() and (flat[:, d // group:] == 0).all()
    assert int(layer.device_status.item()) == 0 and (layer.zero is None) == (not zero_points)


@pytest.mark.parametrize("zero_points", [False, True])
def test_weights_at_the_borders(fef, zero_points):
    w = torch.zeros((12, 64), dtype=torch.bfloat16, device="cuda")
    w[1] = 5.0                                               # one sign only
    w[2] = -5.0
    w[3, 7] = 1e-40                                          # a scale below the normal numbers, or zero
    w[4] = torch.linspace(-7.5, 7.5, 64, device="cuda").to(torch.bfloat16)
    w[5] = torch.arange(64, device="cuda").to(torch.bfloat16) * 0.25 - 7          # quotients on ties
    w[6, 0], w[6, 1] = 3e38, -3e38
    w[7, 40] = math.nan
    w[8, 3] = math.inf
    w[9, 33] = -math.inf
    w[10] = torch.finfo(torch.bfloat16).tiny
    layer = fef.fef_lmhead_quantize(w, 32, zero_points)
    got = fef.fef_lmhead_dequantize(layer).cpu()
    ref, _ = _values(w, 32, zero_points)
    fine = torch.ones((12, 2), dtype=torch.bool)
    for r, c in ((7, 1), (8, 0), (9, 1)) + (((6, 0),) if zero_points else ()):    # 6e38 is no binary32 number
        fine[r, c] = False
    fine = fine.repeat_interleave(32, 1)
    assert torch.equal(got[fine].double(), ref[fine]) and torch.isnan(got[~fine]).all()
    assert int(layer.device_status.item()) == fef.FEF_ERR_NONFINITE


def _layer(fef, V, d, group, zero_points, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn((V, d), generator=g, device="cuda") + (0.2 if zero_points else 0.0)) * (2.0 / math.sqrt(d))
    return fef.fef_lmhead_quantize(w.to(torch.bfloat16), group, zero_points), g


def _check_product(fef, layer, hidden, dtype, out=None):
    got, status = fef.fef_lmhead_logits_quantized(hidden, layer, dtype=dtype, out=out)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    V, d = layer.packed.shape[0], layer.d
    w = fef.fef_lmhead_dequantize(layer).double()
    h = hidden.double()
    ref, scale = h @ w.T, h.abs() @ w.abs().T
    # A group's sum of at most 128 exact products, its scaling and the sum over the groups: every addition rounds, or in a
    # matrix instruction cuts off, at most one step 2^-23 of what has been added up so far; d / 8 + d / 32 additions bound
    # the length of the chain (no product is added alone: eight at least are added together), and a chain's partial sums
    # are below sum |h w|.  The errors are independent enough for the square root of the length with a factor of 4.
    bound = 4 * 2.0 ** -23 * math.sqrt(d / 8 + d / 32) * scale + 1e-37
    if dtype == torch.bfloat16:
        bound = bound + torch.finfo(dtype).eps / 2 * (ref.abs() + bound)
    err = (got[:, :V].double() - ref).abs()
    assert (err <= bound).all(), float((err / bound).max())
    return got


PRODUCTS = [
    # rows, V, d, group, zero points, dtype
    (1, 1, 32, 32, True, torch.float32),
    (1, 5, 96, 32, False, torch.bfloat16),
    (2, 33, 64, 64, True, torch.float32),
    (3, 31, 160, 32, True, torch.bfloat16),
    (5, 257, 192, 64, False, torch.float32),
    (7, 300, 384, 128, True, torch.float32),
    (8, 1000, 1056, 32, True, torch.bfloat16),
    (9, 1001, 1152, 128, False, torch.float32),
    (15, 511, 4096, 128, True, torch.float32),
    (16, 513, 4096, 64, False, torch.bfloat16),
    (17, 700, 256, 32, False, torch.float32),
    (31, 129, 576, 64, True, torch.float32),
    (33, 2049, 1280, 128, True, torch.bfloat16),
    (64, 5003, 1024, 128, False, torch.float32),
    (65, 130, 3584, 64, True, torch.float32),
    (100, 385, 8192, 128, True, torch.bfloat16),
    (128, 4099, 512, 32, True, torch.float32),
    (257, 1027, 1152, 128, False, torch.float32),
    (600, 900, 320, 64, True, torch.bfloat16),
    (1, 20000, 4096, 128, False, torch.float32),
    (4, 40001, 2048, 64, True, torch.bfloat16),
    (12, 126464, 1024, 128, False, torch.float32),
    (16, 600, 16384, 128, True, torch.float32),
]


@pytest.mark.parametrize("rows,V,d,group,zero_points,dtype", PRODUCTS)
def test_product(fef, rows, V, d, group, zero_points, dtype):
    layer, g = _layer(fef, V, d, group, zero_points, seed=rows + V + d)
    hidden = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16)
    _check_product(fef, layer, hidden, dtype)


def test_product_leaves_the_padding_and_repeats_itself(fef):
    for rows in (3, 40, 300):
        layer, g = _layer(fef, 1003, 640, 64, True, seed=rows)
        hidden = torch.randn((rows, 640), generator=g, device="cuda").to(torch.bfloat16)
        out = torch.full((rows, 1064), 55.0, device="cuda")
        first = _check_product(fef, layer, hidden, torch.float32, out=out).clone()
        assert (out[:, 1003:] == 55).all()
        again, _ = fef.fef_lmhead_logits_quantized(hidden, layer, out=out)
        assert torch.equal(first, again)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        other, _ = fef.fef_lmhead_logits_quantized(hidden, layer, stream=s)
        s.synchronize()
        assert torch.equal(first[:, :1003], other[:, :1003])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fef.fef_lmhead_logits_quantized(hidden, layer, out=out)
        hidden.mul_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:, :1003], first[:, :1003] * 2)


@pytest.mark.parametrize("rows", [2, 24, 200])
def test_values_that_are_not_numbers_stay_in_their_rows(fef, rows):
    layer, g = _layer(fef, 700, 256, 128, False, seed=1)
    hidden = torch.randn((rows, 256), generator=g, device="cuda").to(torch.bfloat16)
    clean = _check_product(fef, layer, hidden, torch.float32).clone()
    hidden[1, 77] = math.nan
    dirty, _ = fef.fef_lmhead_logits_quantized(hidden, layer)
    keep = torch.arange(rows, device="cuda") != 1
    assert torch.equal(dirty[keep][:, :700], clean[keep][:, :700]) and torch.isnan(dirty[1, :700]).all()
    scale = layer.scale.clone()
    scale[1, 5, 0] = math.nan
    hidden[1, 77] = 0.5
    dirty, _ = fef.fef_lmhead_logits_quantized(hidden, layer._replace(scale=scale))
    other = torch.arange(700, device="cuda") != 5
    base, _ = fef.fef_lmhead_logits_quantized(hidden, layer)
    assert torch.equal(dirty[:, :700][:, other], base[:, :700][:, other]) and torch.isnan(dirty[:, 5]).all()


@pytest.mark.parametrize("rows", [8, 16, 40, 150])
def test_rows_of_any_magnitude(fef, rows):
    """A row's power of two passes through exactly: products and sums are binary32 numbers far from its limits."""
    layer, g = _layer(fef, 333, 384, 64, True, seed=3)
    hidden = torch.randn((rows, 384), generator=g, device="cuda").to(torch.bfloat16)
    base, _ = fef.fef_lmhead_logits_quantized(hidden, layer)
    powers = torch.tensor([0, 90, -60, 26, 30, -81, 60, -100], dtype=torch.float64, device="cuda").repeat((rows + 7) // 8)[:rows]
    scaled = (hidden.double() * torch.exp2(powers)[:, None]).to(torch.bfloat16)
    scaled[rows - 1] = 0.0
    got, _ = fef.fef_lmhead_logits_quantized(scaled, layer)
    want = base.double() * torch.exp2(powers)[:, None]
    want[rows - 1] = 0.0
    torch.cuda.synchronize()
    V = 333
    assert torch.equal(got[:, :V].double(), want[:, :V].float().double())
    # one value of another order of magnitude, an infinity in a row of its own
    scaled[2, 5], scaled[3, 7] = 1e20, math.inf
    got, _ = fef.fef_lmhead_logits_quantized(scaled, layer)
    ref = scaled[2].double() @ fef.fef_lmhead_dequantize(layer).double().T
    assert torch.allclose(got[2, :V].double(), ref, rtol=2e-6, atol=float(ref.abs().max()) * 2e-6)
    assert not torch.isfinite(got[3, :V]).any()
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[2:4] = False
    assert torch.equal(got[keep][:, :V].double(), want[keep][:, :V].float().double())


@pytest.mark.parametrize("rows", [1, 8, 16, 17, 65])
@pytest.mark.parametrize("d,group,zero_points", [(384, 64, True), (256, 32, False), (4096, 128, True), (4096, 128, False)])
def test_outlier_channels_over_weights_of_zero(fef, rows, d, group, zero_points):
    """Hidden channels far larger than the rest, over columns whose weights are zero (q = z): (q - z) h is exactly zero there, however
    large h is, so the logits are as exact as without those channels."""
    V = 700
    g = torch.Generator(device="cuda").manual_seed(d + rows)
    w = (torch.randn((V, d), generator=g, device="cuda") + (0.2 if zero_points else 0.0)) * (2.0 / math.sqrt(d))
    columns = torch.tensor([3, 100, 101, 180, d - 1], device="cuda")
    w[:, columns] = 0.0
    layer = fef.fef_lmhead_quantize(w.to(torch.bfloat16), group, zero_points)
    assert not fef.fef_lmhead_dequantize(layer)[:, columns].any()
    hidden = torch.randn((rows, d), generator=g, device="cuda")
    hidden[:, columns] *= torch.tensor([1e3, 1e4, 1e5, 3e6, 1e8], device="cuda")
    hidden = hidden.to(torch.bfloat16)
    got = _check_product(fef, layer, hidden, torch.float32)         # (the bound counts |w h|: the outliers add nothing to it)
    clean = hidden.clone()
    clean[:, columns] = 0.0
    assert torch.equal(got[:, :V], _check_product(fef, layer, clean, torch.float32)[:, :V])
    # nothing but outliers: exact zeros
    alone = torch.zeros_like(hidden)
    alone[:, columns] = hidden[:, columns]
    got, _ = fef.fef_lmhead_logits_quantized(alone, layer)
    assert not got[:, :V].any()


@pytest.mark.parametrize("rows", [1, 8, 16, 17])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_single_columns_give_the_values_themselves(fef, rows, group):
    """One hidden value per row: the logits are one column of the layer times it, exactly, for every nibble and zero point."""
    V, d = 300, 384
    g = torch.Generator(device="cuda").manual_seed(rows)
    packed = torch.randint(0, 256, (V, d // 2), generator=g, device="cuda").to(torch.uint8)
    shape = (d // 128, (V + 31) // 32 * 32, 128 // group)
    scale = (torch.rand(shape, generator=g, device="cuda") + 0.5).to(torch.bfloat16)
    zero = torch.randint(0, 16, shape, generator=g, device="cuda").to(torch.uint8)
    for z in (zero, None):
        layer = fef.QuantizedLayer(packed, scale, z, d, group)
        w = fef.fef_lmhead_dequantize(layer).double()
        for at in range(0, d, rows):
            hidden = torch.zeros((rows, d), dtype=torch.bfloat16, device="cuda")
            row = torch.arange(min(rows, d - at), device="cuda")
            value = torch.exp2((row * 37 + at * 11).double() % 180 - 90)
            hidden[row, at + row] = value.to(torch.bfloat16)
            got, _ = fef.fef_lmhead_logits_quantized(hidden, layer)
            assert torch.equal(got[row, :V].double(), w[:, at + row].T * value[:, None])


@pytest.mark.parametrize("rows,d", [(8, 13440), (8, 13568), (1, 13440), (16, 6144), (16, 6272), (9, 6144)])
def test_product_where_the_hidden_rows_just_fit_shared_memory(fef, rows, d):
    """... and where they do not."""
    layer, g = _layer(fef, 100, d, 128, True, seed=d)
    _check_product(fef, layer, torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16), torch.float32)


@pytest.mark.parametrize("rows", [1, 20])
def test_offsets_beyond_32_bits(fef, rows):
    V, d = 300000, 16384                                     # 2.5 GB of nibbles, 9.8 GB of weights
    row = torch.randn((1, d), device="cuda").to(torch.bfloat16)
    last = fef.fef_lmhead_quantize(row, 128)
    Vp = (V + 31) // 32 * 32
    packed = torch.zeros((V, d // 2), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((d // 128, Vp, 1), dtype=torch.bfloat16, device="cuda")
    packed[-1], scale[:, V - 1] = last.packed[0], last.scale[:, 0]
    hidden = torch.randn((rows, d), device="cuda").to(torch.bfloat16)
    got, _ = fef.fef_lmhead_logits_quantized(hidden, fef.QuantizedLayer(packed, scale, None, d, 128))
    ref, _ = fef.fef_lmhead_logits_quantized(hidden, last)
    torch.cuda.synchronize()
    assert torch.allclose(got[:, V - 1], ref[:, 0], rtol=1e-4, atol=1e-3) and (got[:, :V - 1] == 0).all()


def test_two_streams_and_graphs_at_once(fef):
    """Calls that overlap, each with scratch of its own: eager ones on two streams, two captured ones replayed together."""
    layer, g = _layer(fef, 20011, 1024, 128, False, seed=12)
    inputs = [torch.randn((rows, 1024), generator=g, device="cuda").to(torch.bfloat16) for rows in (12, 90, 70, 16)]
    alone = [fef.fef_lmhead_logits_quantized(h, layer)[0].clone() for h in inputs]
    outs = [torch.zeros_like(a) for a in alone]
    graphs = []
    for h, out in zip(inputs, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fef.fef_lmhead_logits_quantized(h, layer, out=out)
        graphs.append(graph)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in inputs]
    for _ in range(5):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        eager = [fef.fef_lmhead_logits_quantized(h, layer, stream=s)[0] for h, s in zip(inputs, streams)]
        torch.cuda.synchronize()
        for a, out, e in zip(alone, outs, eager):
            assert torch.equal(a[:, :20011], out[:, :20011]) and torch.equal(a[:, :20011], e[:, :20011])


def test_refusals(fef):
    w = torch.randn((40, 128), device="cuda").to(torch.bfloat16)
    for args in ((w.float(),), (w[:, ::2],), (w[0],), (w, 16), (w, 256), (w[:, :96].contiguous(), 64), (w[:0],)):
        with pytest.raises(fef.FefError):
            fef.fef_lmhead_quantize(*args)
    layer = fef.fef_lmhead_quantize(w, 64, True)
    hidden = torch.zeros((3, 128), dtype=torch.bfloat16, device="cuda")
    changes = [dict(packed=layer.packed[:, :32].contiguous()), dict(packed=layer.packed.int()), dict(scale=layer.scale.float()),
               dict(scale=layer.scale[:, :40].contiguous()), dict(zero=layer.zero.int()), dict(zero=layer.zero[:, :32].contiguous()),
               dict(d=256), dict(group=32), dict(group=128), dict(packed=layer.packed[:3])]
    for change in changes:
        broken = layer._replace(**change)
        with pytest.raises(fef.FefError):
            fef.fef_lmhead_dequantize(broken)
        with pytest.raises(fef.FefError):
            fef.fef_lmhead_logits_quantized(hidden, broken)
    for h, kw in ((hidden.float(), {}), (hidden[:, :64].contiguous(), {}), (hidden[:0], {}), (hidden, dict(dtype=torch.float16)),
                  (hidden, dict(out=torch.zeros((2, 40), device="cuda"))), (hidden, dict(out=torch.zeros((3, 36), device="cuda"))),
                  (hidden, dict(out=torch.zeros((3, 42), device="cuda"))), (hidden, dict(out=torch.zeros((3, 40), device="cuda").half()))):
        with pytest.raises(fef.FefError):
            fef.fef_lmhead_logits_quantized(h, layer, **kw)
    with pytest.raises(fef.FefError):
        fef.fef_lmhead_dequantize(layer, out=torch.zeros((40, 64), device="cuda"))
    many = torch.zeros((40, 128), dtype=torch.bfloat16, device="cuda")
    need = fef.fef_lmhead_logits_quantized_workspace_bytes(40, 40, 128, 64)
    with pytest.raises(fef.FefError):
        fef.fef_lmhead_logits_quantized(many, layer, workspace=torch.zeros(need - 1, dtype=torch.uint8, device="cuda"))
    fef.fef_lmhead_logits_quantized(many, layer, workspace=torch.zeros(need, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        fef.fef_lmhead_logits_quantized(hidden, layer._replace(packed=layer.packed.cpu()))


@pytest.mark.parametrize("rows,V,d,group", [
    (8, 100, 12544, 128), (8, 100, 12672, 128),              # the hidden rows just fit one SM's shared memory, and do not
    (16, 100, 5760, 64), (16, 100, 5888, 64),
    (1, 33, 1 << 20, 32), (20, 33, 1 << 20, 128),            # the longest rows
    (70001, 40, 32, 32),                                     # many
])
def test_product_at_the_ends_of_its_ranges(fef, rows, V, d, group):
    layer, g = _layer(fef, V, d, group, True, seed=rows)
    hidden = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16)
    _check_product(fef, layer, hidden, torch.float32)


def test_quantize_beyond_32_bits(fef):
    V, d = 300001, 16384                                     # 9.8 GB of weights, 19.7 GB of values
    w = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    w[-1] = torch.randn(d, device="cuda").to(torch.bfloat16)
    alone = fef.fef_lmhead_quantize(w[-1:].contiguous(), 64, True)
    layer = fef.fef_lmhead_quantize(w, 64, True)
    del w
    assert int(layer.device_status.item()) == 0
    assert torch.equal(layer.packed[-1], alone.packed[0]) and torch.equal(layer.scale[:, V - 1], alone.scale[:, 0])
    values = fef.fef_lmhead_dequantize(layer)
    assert torch.equal(values[-1], fef.fef_lmhead_dequantize(alone)[0]) and not values[:-1].any()


FIRST_CALLS = """
import torch
import paper_2605_14305_b200 as fef

fef.load()
g = torch.Generator(device="cuda").manual_seed(1)
w = torch.randn((1003, 256), generator=g, device="cuda").to(torch.bfloat16)
hidden = [torch.randn((rows, 256), generator=g, device="cuda").to(torch.bfloat16) for rows in (4, 40, 140)]
bias = torch.randn(1003, generator=g, device="cuda")

def chain():
    layer = fef.fef_lmhead_quantize(w, 64, True)
    out = [fef.fef_lmhead_dequantize(layer)]
    for h in hidden:
        logits = fef.fef_lmhead_logits_quantized(h, layer)[0]
        out += list(fef.fef_logits_adjust(logits.view(4, -1, logits.shape[-1]), bias=bias, V=1003, with_norm=True))
    return out

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    captured = chain()
graph.replay()
eager = chain()
torch.cuda.synchronize()
for a, b in zip(captured, eager):
    a, b = (x[..., :1003] if x.dim() == 3 else x for x in (a, b))
    assert torch.equal(a, b) and torch.isfinite(a).all()
"""


def test_first_calls_of_a_process_captured(fef):
    """Nothing has to have run before a capture."""
    import subprocess
    import sys

    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
