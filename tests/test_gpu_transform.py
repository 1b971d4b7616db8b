"""fef_hidden_transform against its definition in 64 bits (needs a B200)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


@pytest.fixture(scope="module")
def fef():
    import paper_2605_14305_b200 as lib

    lib.load(build_if_missing=True)
    return lib


def _act(y, act):
    if act == "relu":
        return y.clamp(min=0)
    if act == "silu":
        return y * torch.sigmoid(y)
    if act == "gelu":
        return y * torch.special.ndtr(y)
    if act == "gelu_tanh":
        return y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
    return y


def _want(hidden, weight, bias, residual, act):
    """(value, bound of the error before the last rounding), in 64 bits."""
    h, w = hidden.double(), weight.double()
    y, size = h @ w.T, h.abs() @ w.abs().T
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    # the products are exact; however they are added, d + 8 additions in binary32 that may round towards zero (2^-23 each) cost
    # that share of the sum of the magnitudes at most
    err = (hidden.shape[1] + 8) * 2.0 ** -23 * size
    z = _act(y, act)
    # the activations' slopes are at most 1.13; the functions themselves: an exponential within 2^-22, its argument's rounding
    # (|y| log2(e) 2^-23, and three operations more for gelu_tanh's cubic, whose effect y z' sigmoid' stays below 4), erfc and
    # a division: less than 2^-19 of |y|
    err = 1.13 * err + (0 if act in ("none", "relu") else 2.0 ** -19 * y.abs())
    if residual is not None:
        z = z + residual.double()
        err = err + 2.0 ** -24 * z.abs()
    return z, err + 1e-37


def _check(fef, rows, n, d, act="none", bias=False, residual=False, dtype=torch.bfloat16, seed=0, scale=None, out=None):
    g = torch.Generator(device="cuda").manual_seed(seed + rows + 31 * n + 7 * d)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    h, w = normal(rows, d), (normal(n, d).float() * (d ** -0.5 if scale is None else scale)).to(torch.bfloat16)
    b, r = normal(n) if bias else None, normal(rows, n) if residual else None
    got, status = fef.fef_hidden_transform(h, w, bias=b, residual=r, activation=act, dtype=dtype, out=out)
    torch.cuda.synchronize()
    assert int(status) == 0 and got.shape == (rows, n) and got.dtype == dtype
    want, err = _want(h, w, b, r, act)
    half = torch.finfo(dtype).eps / 2
    bound = err + half * (want.abs() + err)
    worst = float(((got.double() - want).abs() / bound).max())
    assert worst <= 1, worst
    return h, w, b, r, got


SIZES = [(1, 1, 8), (1, 128, 64), (2, 7, 16), (3, 130, 72), (5, 1000, 1056), (8, 257, 520), (9, 5003, 1056), (16, 4096, 4096),
         (17, 333, 248), (31, 64, 4096), (33, 1024, 1000), (64, 3584, 3584), (65, 129, 64), (100, 700, 2048), (128, 512, 512),
         (129, 300, 136), (200, 2000, 1024), (257, 1111, 328), (300, 4096, 1024), (515, 640, 4096), (1000, 513, 200), (2048, 256, 64),
         (257, 5003, 72), (520, 4000, 264), (1030, 2500, 1000), (2048, 1300, 136), (2048, 4096, 512), (5000, 1111, 520)]


@pytest.mark.parametrize("rows,n,d", SIZES)
def test_sizes(fef, rows, n, d):
    _check(fef, rows, n, d, "silu", True, True)
    _check(fef, rows, n, d, "none", False, False, torch.float32)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_activations_and_epilogues(fef, act, dtype):
    for rows in (3, 70, 300, 7000):
        for bias in (False, True):
            for residual in (False, True):
                _check(fef, rows, 390, 264, act, bias, residual, dtype, seed=5)
        _check(fef, rows, 390, 264, act, True, False, dtype, scale=4.0)     # arguments of 60 and more, both signs
        _check(fef, rows, 390, 264, act, True, False, dtype, scale=1e-6)


@pytest.mark.parametrize("rows,n,d", [(1, 512, 8192), (20, 300, 16384), (64, 4096, 8192), (300, 700, 5000), (700, 5003, 4104),
                                      (1000, 4096, 8192)])
def test_binary32_sums_of_many_products(fef, rows, n, d):
    """Products of one sign, so that the sums grow and roundings towards zero add up."""
    g = torch.Generator(device="cuda").manual_seed(d)
    h, w = (torch.rand(s, generator=g, device="cuda").bfloat16() for s in ((rows, d), (n, d)))
    got, status = fef.fef_hidden_transform(h, w, dtype=torch.float32)
    assert int(status) == 0
    want = h.double() @ w.double().T
    # 512 products go to one sum, sixteen at a time: 32 additions, each within two roundings towards zero (2^-23 of the sum each: the
    # addition's and the products'); the sums of at most d / 512 + 8 parts are added with rounding to nearest, 2^-24 each.  8192 products
    # in one sum lose 512 x 2^-24 x half of the final sum on average, 1.5 10^-5, twice what is allowed
    allowed = 64 * 2.0 ** -23 + (d / 512 + 9) * 2.0 ** -24
    assert float(((got.double() - want).abs() / want).max()) <= allowed


def test_every_row_count_up_to_a_tile(fef):
    for rows in range(1, 70):
        _check(fef, rows, 200, 128, "gelu", True, False)


def test_strided_operands_and_what_is_left_alone(fef):
    g = torch.Generator(device="cuda").manual_seed(1)
    for rows, n, d in ((5, 37, 40), (70, 301, 200), (260, 129, 64), (2600, 1025, 72)):
        big = torch.randn((rows, 2 * d + 8), generator=g, device="cuda").to(torch.bfloat16)
        res = torch.randn((rows, n + 3), generator=g, device="cuda").to(torch.bfloat16)
        w = torch.randn((n, d), generator=g, device="cuda").to(torch.bfloat16)
        hidden, residual = big[:, 8:8 + d], res[:, 1:1 + n]
        for dtype in (torch.float32, torch.bfloat16):
            buf = torch.full((rows + 2, n + 5), 77.0, dtype=dtype, device="cuda")
            out = buf[1:-1, 3:3 + n]
            got, _ = fef.fef_hidden_transform(hidden, w, residual=residual, activation="relu", out=out)
            want, _ = fef.fef_hidden_transform(hidden.contiguous(), w, residual=residual.contiguous(), activation="relu", dtype=dtype)
            torch.cuda.synchronize()
            assert got is out and torch.equal(out, want)
            rest = buf.clone()
            rest[1:-1, 3:3 + n] = 77.0
            assert (rest == 77.0).all()


def test_in_place_on_the_residual(fef):
    for rows, n, d in ((1, 512, 512), (40, 1024, 1024), (300, 520, 520), (1500, 2056, 2056)):
        h, w, b, r, want = _check(fef, rows, n, d, "silu", True, True)
        got, _ = fef.fef_hidden_transform(h, w, bias=b, residual=r, activation="silu", out=r)
        torch.cuda.synchronize()
        assert got is r and torch.equal(r, want)


def test_columns_of_one_buffer(fef):
    g = torch.Generator(device="cuda").manual_seed(3)
    for rows, n, d in ((3, 40, 64), (90, 520, 512), (700, 1032, 264)):
        buf = torch.randn((rows, d + 2 * n), generator=g, device="cuda").bfloat16()
        w = torch.randn((n, d), generator=g, device="cuda").bfloat16()
        before = buf.clone()
        want, _ = fef.fef_hidden_transform(before[:, :d].contiguous(), w, residual=before[:, d + n:].contiguous(), activation="gelu")
        fef.fef_hidden_transform(buf[:, :d], w, residual=buf[:, d + n:], activation="gelu", out=buf[:, d:d + n])
        assert torch.equal(buf[:, d:d + n], want) and torch.equal(buf[:, :d], before[:, :d]) and torch.equal(buf[:, d + n:], before[:, d + n:])


def test_a_bad_row_stays_alone(fef):
    for rows, n, d in ((4, 300, 256), (50, 300, 256), (300, 300, 256), (9000, 300, 256)):
        h, w, b, r, want = _check(fef, rows, n, d, "gelu_tanh", True, True)
        bad = rows // 2
        for value in (math.nan, math.inf):
            x = h.clone()
            x[bad, d - 1] = value
            got, _ = fef.fef_hidden_transform(x, w, bias=b, residual=r, activation="gelu_tanh")
            torch.cuda.synchronize()
            others = torch.arange(rows, device="cuda") != bad
            assert torch.equal(got[others], want[others])
            assert not torch.isfinite(got[bad]).all()


def test_large_weights_and_infinities_of_the_bias(fef):
    h = torch.ones((3, 8), dtype=torch.bfloat16, device="cuda")
    w = torch.full((5, 8), 1e38, dtype=torch.bfloat16, device="cuda")
    w[1] = -1e38
    b = torch.tensor([0, 0, math.inf, -math.inf, 0], dtype=torch.bfloat16, device="cuda")
    w[2:] = 1.0
    got, _ = fef.fef_hidden_transform(h, w, bias=b, activation="relu", dtype=torch.float32)
    assert got[0].tolist() == [math.inf, 0.0, math.inf, 0.0, 8.0]
    got, _ = fef.fef_hidden_transform(h, w, bias=b, activation="gelu", dtype=torch.float32)
    assert got[0, 0] == math.inf and got[0, 2] == math.inf and got[0, 4] == 8.0


def test_rows_do_not_depend_on_their_neighbours(fef):
    """The same row gives the same bits in any place of any call with as many rows; twice the same call, the same bits."""
    for rows in (300, 4000):
        _same_rows(fef, rows)


def _same_rows(fef, rows):
    h, w, b, r, first = _check(fef, rows, 640, 1024, "silu", True, True)
    again, _ = fef.fef_hidden_transform(h, w, bias=b, residual=r, activation="silu")
    assert torch.equal(first, again)
    turned, _ = fef.fef_hidden_transform(h.flip(0).contiguous(), w, bias=b, residual=r.flip(0).contiguous(), activation="silu")
    assert torch.equal(turned.flip(0), first)


def test_streams_and_graphs(fef):
    for rows in (2, 100, 600, 3000):
        h, w, b, r, want = _check(fef, rows, 1000, 512, "gelu", True, True)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got, _ = fef.fef_hidden_transform(h, w, bias=b, residual=r, activation="gelu", stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        out, graph = torch.empty_like(want), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fef.fef_hidden_transform(h, w, bias=b, residual=r, activation="gelu", out=out)
        h2 = torch.randn_like(h)
        h.copy_(h2)
        graph.replay()
        graph.replay()
        want, _ = fef.fef_hidden_transform(h2, w, bias=b, residual=r, activation="gelu")
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_calls_at_once(fef):
    streams = [torch.cuda.Stream() for _ in range(3)]
    work = [_check(fef, rows, 2000, 1024, "silu", True, False, seed=rows) for rows in (1, 64, 1700)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, (h, w, b, _, _) in zip(streams, work):
            got.append(fef.fef_hidden_transform(h, w, bias=b, activation="silu", stream=s)[0])
    torch.cuda.synchronize()
    for i, t in enumerate(got):
        assert torch.equal(t, work[i % 3][4])


def test_offsets_beyond_32_bits(fef):
    """An output whose last rows lie more than 2^32 bytes behind its first."""
    rows, n, d = 40, 64, 64
    pitch = (1 << 32) // 2 // 32
    buf = torch.empty((rows - 1) * pitch + n, dtype=torch.bfloat16, device="cuda")
    out = buf.as_strided((rows, n), (pitch, 1))
    _, _, _, _, got = _check(fef, rows, n, d, "silu", True, False, out=out)
    assert got.data_ptr() == buf.data_ptr()


def test_refusals(fef):
    mk = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    h, w = mk(4, 64), mk(32, 64)
    f = fef.fef_hidden_transform
    square = mk(4, 64)
    calls = [lambda: f(h, mk(32, 72)), lambda: f(h.float(), w), lambda: f(h, w.float()), lambda: f(h[0], w),
             lambda: f(mk(4, 12), mk(32, 12)), lambda: f(h, mk(64, 32).T), lambda: f(h, w, bias=mk(31)), lambda: f(h, w, bias=mk(32).float()),
             lambda: f(h, w, residual=mk(4, 31)), lambda: f(h, w, residual=mk(4, 32).float()), lambda: f(h, w, activation="tanh"),
             lambda: f(h, w, dtype=torch.float16), lambda: f(h, w, out=mk(4, 31)), lambda: f(h, w, out=mk(32, 4).T),
             lambda: f(mk(0, 64), w), lambda: f(mk(1, 64).expand(4, 64), w), lambda: f(h, w, out=mk(1, 32).expand(4, 32)),
             lambda: f(mk(4, 65)[:, 1:], w), lambda: f(mk(4, 68)[:, :64], w),            # a pitch or an address off 16 bytes
             lambda: f(square, mk(64, 64), out=square),                                  # the output over the input
             lambda: f(h, w, residual=mk(5, 32)[:4], out=mk(5, 32)[:4].float()[:, :31])]
    shared = mk(5, 32)
    calls.append(lambda: f(h, w, residual=shared[:4], out=shared[1:]))                   # ... over another part of the residual
    for i, call in enumerate(calls):
        with pytest.raises(fef.FefError):
            call()
    with pytest.raises(ValueError):
        f(h, w.cpu())
    torch.cuda.synchronize()
