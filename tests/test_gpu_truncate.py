"""Laws cut to top-k, top-p and min-p sets, and draws from them, against their definition in 64 bits (needs a B200)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LOG2E = math.log2(math.e)
NORM_TOL = 1.9e-6   # relative error of a law's normaliser that the verification's intervals allow for (2e-6)


@pytest.fixture(scope="module")
def fef():
    import paper_2605_14305_b200 as lib

    lib.load(build_if_missing=True)
    return lib


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _f32(*v):
    return torch.tensor(v, dtype=torch.float32, device="cuda")


def _philox_word(seed, counter):
    """Output word 0 of Philox4x32-10."""
    c, k = list(counter), [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        a, d = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(d >> 32) ^ c[1] ^ k[0], d & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c[0]


def _row(l, T, k, p, m, u):
    """(token, conf, log2_norm, cut_logit, cut_id, kept) of one row of float64 logits; None for a row that is an error."""
    if np.isnan(l).any() or (l == np.inf).any() or not np.isfinite(l).any() or any(v != v for v in (p, m, u)):
        return None
    V = len(l)
    order = np.lexsort((np.arange(V), -l))
    order = order[l[order] > -np.inf]
    w = np.exp((l[order] - l[order[0]]) / T)
    n = min(k, len(order)) if 0 < k < V else len(order)
    if p < 1:
        upto = np.cumsum(w[:n])
        n = min(n, int(np.searchsorted(upto, p * upto[-1])) + 1)
    if m > 0:   # w >= m, without the rounding of w: at T = 1e30 every w is 1 in 64 bits, and none but the largest entry's is 1
        n = min(n, int((l[order] - l[order[0]] >= T * math.log(min(m, 1.0))).sum()))
    weights = np.zeros(V)
    weights[order[:n]] = w[:n]
    upto = np.cumsum(weights)
    unit = 2.0 ** -(62 - max(V - 1, 0).bit_length())   # the draw's unit: what rounds to none of it is never drawn, by u = 0 neither
    drawn = np.cumsum(np.where(weights <= unit / 2, 0.0, weights))
    x = int(np.searchsorted(drawn, min(max(u, 0.0), 1 - 2.0 ** -24) * drawn[-1], side="right"))
    cut = (l[order[n - 1]], order[n - 1]) if 0 < k < V or p < 1 or m > 0 else (-np.inf, -1)
    return x, weights[x] / upto[-1], l[order[0]] * (LOG2E / T) + math.log2(upto[-1]), *cut, n


def _check(fef, logits, T=1.0, top_k=None, top_p=None, min_p=None, uniforms=None, row_len=None, V=None, seed=0, step=0, **more):
    B, K, ld = logits.shape
    V = ld if V is None else V
    if more.get("device_round") is not None:
        assert uniforms is None
    d = fef.fef_draft_sample_truncated(logits, T, seed, step, top_k, top_p, min_p, uniforms, row_len, V, **more)
    law = fef.fef_law_truncate(logits, T, top_k, top_p, min_p, row_len, V)
    torch.cuda.synchronize()
    for a, b in zip(law[:4], d.law[:4]):   # the law does not depend on whether something is drawn
        assert torch.equal(torch.nan_to_num(a, nan=7.25), torch.nan_to_num(b, nan=7.25))
    T = float(np.float32(T))
    l = logits[..., :V].double().cpu().numpy()
    at = lambda t, b, off: off if t is None else float(t[b])  # noqa: E731
    got = [t.cpu().numpy() for t in (d.tokens, d.conf, d.law.log2_norm, d.law.cut_logit, d.law.cut_id, d.law.kept)]
    errors = False
    for b in range(B):
        for i in range(K):
            tok, conf, norm, cut, cut_id, kept = (g[b, i] for g in got)
            if row_len is not None and i >= int(row_len[b]):
                assert (tok, conf, norm, cut, cut_id, kept) == (-1, -1.0, 0.0, 0.0, -1, 0)
                continue
            if uniforms is not None:
                u = float(uniforms[b, i])
            else:
                rnd = 0 if more.get("device_round") is None else int(more["device_round"])
                u = ((_philox_word(seed, (2 << 30, b, i, (step + rnd) & 0xFFFFFFFF)) >> 9) + 0.5) * 2.0 ** -23
            want = _row(l[b, i], T, int(at(top_k, b, 0)), at(top_p, b, 1.0), at(min_p, b, 0.0), u)
            if want is None:
                errors = True
                assert (tok, conf, cut_id, kept) == (-1, -1.0, -1, 0) and math.isnan(norm) and math.isnan(cut)
                continue
            assert (kept, cut_id, cut) == (want[5], want[4], want[3]), (b, i, kept, cut_id, cut, want)
            assert tok == want[0], (b, i, tok, want)
            assert abs(norm - want[2]) <= NORM_TOL / math.log(2) + 2.0 ** -50 * abs(want[2])
            assert abs(conf - want[1]) <= want[1] * (NORM_TOL + 2.0 ** -24)
    for s in (d.law.device_status, law.device_status):
        assert int(s.item()) == (fef.FEF_ERR_NONFINITE if errors else 0)
    return d


def _logits(B, K, V, dtype, seed, pad=0, std=2.0, boost=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    per_vec = 8 if dtype == torch.bfloat16 else 4
    ld = (V + pad + per_vec - 1) // per_vec * per_vec
    x = torch.randn((B, K, ld), generator=g, device="cuda") * std
    if boost:
        x += 8 * (torch.rand((B, K, ld), generator=g, device="cuda") < 0.01)
    x[..., V:] = float("nan")   # never looked at
    return x.to(dtype), torch.rand((B, K), generator=g, device="cuda")


RULES = {
    "none": dict(),
    "k": dict(top_k=(1, 7, 50, 1000)),
    "p": dict(top_p=(0.9, 0.5, 0.999, 0.05)),
    "m": dict(min_p=(0.05, 0.5, 0.001, 1.0)),
    "kp": dict(top_k=(20, 3, 900, 0), top_p=(0.8, 0.95, 0.3, 0.99)),
    "kpm": dict(top_k=(40, 0, 5, 100000000), top_p=(0.9, 0.7, 1.0, 0.6), min_p=(0.01, 0.02, 0.0, 0.3)),
    "off": dict(top_k=(0, -3, 0, 2147483647), top_p=(1.0, 2.0, 1.0, math.inf), min_p=(0.0, -1.0, 0.0, -math.inf)),
    "edges": dict(top_p=(0.0, -1.0, 1e-30, 1 - 2.0 ** -24), min_p=(0.0, 1e-38, 2.0, 1e-30)),
}


def _rules(kind, B):
    r = {}
    for name, values in RULES[kind].items():
        t = (_i32 if name == "top_k" else _f32)(*values)
        r[name] = t[torch.arange(B, device="cuda") % 4].contiguous()
    return r


@pytest.mark.parametrize("kind", list(RULES))
@pytest.mark.parametrize("B,K,V,dtype,T,pad", [
    (4, 2, 1, torch.float32, 1.0, 0), (4, 1, 7, torch.bfloat16, 0.5, 0), (5, 3, 33, torch.float32, 1.3, 7),
    (4, 2, 1000, torch.bfloat16, 0.7, 24), (4, 1, 5003, torch.float32, 1.0, 0), (4, 2, 50257, torch.bfloat16, 1.0, 7),
    (4, 1, 126464, torch.bfloat16, 1.0, 0), (4, 1, 126464, torch.float32, 0.8, 8)])
def test_rules_and_sizes(fef, B, K, V, dtype, T, pad, kind):
    x, u = _logits(B, K, V, dtype, 17 * V + K, pad)
    _check(fef, x, T, uniforms=u, V=V, **_rules(kind, B))


@pytest.mark.parametrize("kind", ["p", "kpm", "none"])
@pytest.mark.parametrize("std", [0.01, 2.0, 40.0])
def test_flat_and_steep_laws(fef, std, kind):
    for dtype in (torch.float32, torch.bfloat16):
        x, u = _logits(4, 1, 40000, dtype, 5, std=std, boost=False)
        _check(fef, x, uniforms=u, **_rules(kind, 4))


@pytest.mark.parametrize("rows", [1, 3, 40, 200, 700])
def test_numbers_of_rows(fef, rows):
    B, K = (rows, 1) if rows < 64 else (rows // 4, 4)
    x, u = _logits(B, K, 20011, torch.bfloat16, rows)
    _check(fef, x, 0.9, uniforms=u, **_rules("kpm", B))
    x, u = _logits(B, K, 20011, torch.float32, rows + 1)
    _check(fef, x, 0.9, uniforms=u, V=20005, **_rules("p", B))


def test_ragged_windows_and_random_numbers_of_their_own(fef):
    x, _ = _logits(5, 7, 3000, torch.bfloat16, 3, pad=9)
    row_len = _i32(0, 7, 3, 1, 9)   # (more than K counts as K)
    rnd = torch.tensor([5], dtype=torch.int32, device="cuda")
    rules = _rules("kp", 5)
    _check(fef, x, 0.7, row_len=row_len, V=3000, seed=(7 << 40) + 9, step=4, **rules)
    d = _check(fef, x, 0.7, row_len=row_len, V=3000, seed=(7 << 40) + 9, step=4, device_round=rnd, **rules)
    e = fef.fef_draft_sample_truncated(x, 0.7, (7 << 40) + 9, 9, row_len=row_len, V=3000, **rules)
    assert torch.equal(d.tokens, e.tokens)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties(fef, dtype):
    """Equal logits: the lowest ids stay, and a border in the middle of them falls where the definition says."""
    x = torch.zeros((4, 2, 4096), dtype=dtype, device="cuda")
    x[:, 1, ::2] = -0.0           # equal to 0
    u = torch.tensor([[0.0, 0.999], [0.5, 0.25], [0.125, 0.75], [1.0, -3.0]], device="cuda")
    for rules in (dict(top_k=_i32(1, 100, 4095, 4096)), dict(top_p=_f32(0.25, 0.5, 0.75, 0.1)), dict(min_p=_f32(1.0, 1.0, 0.5, 0.1)),
                  dict(top_k=_i32(10, 1000, 0, 64), top_p=_f32(0.5, 0.5, 0.5, 0.5))):
        _check(fef, x, uniforms=u, **rules)
    y = torch.randint(0, 3, (4, 2, 30000), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype)
    for kind in ("k", "p", "m", "kp", "kpm", "none"):
        _check(fef, y, uniforms=u, **_rules(kind, 4))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_entries(fef, dtype):
    """Rows that a mask leaves little of, with -inf or the type's lowest value in the masked places."""
    low = torch.finfo(dtype).min
    x, u = _logits(4, 3, 9001, dtype, 8, pad=7)
    x = x[..., :9008].contiguous()
    for value in (-math.inf, low):
        y = x.clone()
        y[:, 0, 5:8990] = value
        y[:, 1, :9001] = value
        y[:, 1, 4567] = 3.0
        y[:, 2, 1:9001:2] = value
        for kind in ("k", "p", "m", "kpm", "none"):
            _check(fef, y, uniforms=u, V=9001, **_rules(kind, 4))
    y = torch.full((4, 1, 1024), low, dtype=dtype, device="cuda")   # nothing but the lowest value: a law like any other
    for kind in ("k", "p", "none"):
        _check(fef, y, uniforms=u[:, :1].contiguous(), **_rules(kind, 4))
    top = torch.finfo(dtype).max
    y[:, :, 77] = top                                               # the whole range in one row
    for kind in ("k", "p", "m", "none"):
        _check(fef, y, uniforms=u[:, :1].contiguous(), **_rules(kind, 4))


@pytest.mark.parametrize("where", [0, 5000, 9000])
def test_errors_stay_in_their_rows(fef, where):
    for dtype in (torch.float32, torch.bfloat16):
        for bad in (math.nan, math.inf):
            for kind in ("k", "p", "m", "none"):
                x, u = _logits(4, 3, 9001, dtype, 8, pad=7)
                x[1, 1, where] = bad
                x[2, 0, :] = -math.inf
                _check(fef, x, uniforms=u, V=9001, **_rules(kind, 4))
    x, u = _logits(4, 3, 9001, torch.float32, 8, pad=7)
    u[3, 1] = math.nan
    d = fef.fef_draft_sample_truncated(x, 1.0, uniforms=u, V=9001, top_p=_f32(0.5, math.nan, 0.5, 0.5), min_p=_f32(math.nan, 0, 0, 0))
    torch.cuda.synchronize()
    assert (d.tokens[:2] == -1).all() and (d.tokens[2] >= 0).all() and d.tokens[3].ge(0).tolist() == [True, False, True]
    assert torch.isnan(d.law.log2_norm[:2]).all() and int(d.law.device_status) == fef.FEF_ERR_NONFINITE


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_orders_of_the_vocabulary(fef, dtype):
    """Likely entries together at one end, in the middle, or in every 32nd place: what a sample of the row would miss."""
    V = 126464
    g = torch.Generator(device="cuda").manual_seed(4)
    base = torch.randn(V, generator=g, device="cuda") * 2
    u = torch.rand((4, 1), generator=g, device="cuda")
    for n in (1, 40, 3000, 30000):
        for place in ("front", "back", "middle", "comb", "sorted", "reversed"):
            x = base.clone()
            if place == "front":
                x[:n] += 9
            elif place == "back":
                x[-n:] += 9
            elif place == "middle":
                x[60000:60000 + n] += 9
            elif place == "comb":
                x[5::max(V // n, 2)] += 9
            else:
                x[:n] += 9
                x = x.sort(descending=place == "sorted").values
            for kind in ("k", "p", "kpm") if n != 40 else ("p", "m", "none"):
                _check(fef, x.to(dtype).expand(4, 1, V).contiguous(), uniforms=u, **_rules(kind, 4))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_unusual_numbers(fef, dtype):
    """Many zeros (of both signs), numbers too small to tell apart, small or shifted laws with masked entries, few different values,
    steep laws: what the counting of values has to leave to another path, or to treat with care."""
    V = 20000
    g = torch.Generator(device="cuda").manual_seed(6)
    normal = torch.randn(V, generator=g, device="cuda")
    rnd = torch.rand(V, generator=g, device="cuda")
    u = torch.tensor([[0.0], [0.3], [0.71], [0.9999999]], device="cuda")
    low = torch.finfo(dtype).min
    rows = {
        "zeros": torch.where(rnd < 0.5, torch.zeros_like(normal), normal),
        "signed zeros": torch.where(rnd < 0.3, -torch.zeros_like(normal), torch.where(rnd < 0.6, torch.zeros_like(normal), -normal.abs())),
        "relu": normal.clamp(min=0) * 3,
        "tiny": torch.where(rnd < 0.5, normal * 1e-12, normal),
        "all tiny": normal * 1e-30,
        "denormal": torch.where(rnd < 0.2, normal * 1e-39, normal),
        "small and masked": torch.where(rnd < 0.6, torch.full_like(normal, -math.inf), normal * 0.02),
        "small and lowest": torch.where(rnd < 0.6, torch.full_like(normal, low), normal * 0.02),
        "shifted up": normal * 2 + 300,
        "shifted down and masked": torch.where(rnd < 0.6, torch.full_like(normal, -math.inf), normal * 2 - 900),
        "few values": (normal * 2).round(),
        "two values": torch.where(rnd < 0.5, torch.zeros_like(normal) + 1, torch.zeros_like(normal) + 2),
        "one far above": torch.where(rnd == rnd.max(), torch.full_like(normal, 80.0), normal * 2),
        "far below": torch.where(rnd < 0.5, normal * 2 - 70, normal * 2),
        "huge": normal * 1e30,
        "ladder": -torch.arange(V, device="cuda") * 0.01,
    }
    for name, x in rows.items():
        x = x.to(dtype).expand(4, 1, V).contiguous()
        for kind in ("k", "p", "m", "kpm", "none", "edges"):
            for T in ((1.0, 0.05) if kind in ("p", "none") else (1.0,)):
                _check(fef, x, T, uniforms=u, **_rules(kind, 4))
        # limits that reach far into the row
        _check(fef, x, uniforms=u, top_k=_i32(9000, 15000, 19990, 6000))
        _check(fef, x, uniforms=u, top_k=_i32(9000, 15000, 19990, 6000), top_p=_f32(0.99, 0.6, 0.9, 0.999), min_p=_f32(0, 1e-3, 1e-6, 0.2))
        _check(fef, x, uniforms=u, min_p=_f32(1e-3, 1e-8, 1e-20, 1e-37))
        _check(fef, x, uniforms=u, top_p=_f32(0.99, 0.9999, 0.999999, 0.3), min_p=_f32(1e-3, 1e-8, 1e-3, 1e-37))


@pytest.mark.parametrize("T", [0.6, 30.0])
@pytest.mark.parametrize("k,p,m", [(0, 0.9, 0.0), (100, 1.0, 0.0), (0, 1.0, 0.001), (15000, 0.99, 0.0), (0, 1.0, 0.0)])
def test_tiny_numbers_among_bfloat16(fef, k, p, m, T):
    x, u = _logits(4, 1, 20000, torch.bfloat16, 31)
    tiny = torch.tensor([1e-30, -1e-30, 2e-38, -9e-41, 0.0, -0.0], device="cuda").bfloat16()
    x[0, 0, 5::4000] = tiny[:5]                       # a few among ordinary ones
    x[1, 0, 30:] = tiny.repeat(4000)[30:20000]        # thirty ordinary ones among them
    x[2, 0] = tiny.repeat(4000)[:20000]               # nothing else
    x[3, 0, ::2] = tiny.repeat(4000)[:10000]
    _check(fef, x, T, top_k=_i32(k, k, k, k), top_p=_f32(p, p, p, p), min_p=_f32(m, m, m, m), uniforms=u)


@pytest.mark.parametrize("rows", [2, 200, 400])    # (as many threads to a row as there are for it)
def test_every_share_of_threads(fef, rows):
    for V in (4097, 8193, 16385, 40961):
        for dtype in (torch.float32, torch.bfloat16):
            x, u = _logits(rows // 2, 2, V, dtype, V, std=1.5, boost=V % 3 == 0)
            few = slice(0, 6)
            for kind in ("p", "kp", "m", "none"):
                rules = _rules(kind, rows // 2)
                d = fef.fef_draft_sample_truncated(x, 1.0, uniforms=u, V=V, **rules)
                sub = _check(fef, x[few].contiguous(), uniforms=u[few].contiguous(), V=V, **{n: t[few].contiguous() for n, t in rules.items()})
                for a, b in zip((*d[:2], *d.law[:4]), (*sub[:2], *sub.law[:4])):
                    if a.dtype == torch.int32 or a is d.law.cut_logit:
                        assert torch.equal(a[few], b)
                    else:
                        assert ((a[few] - b).abs() <= 2 * NORM_TOL * (1 + b.abs())).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V", [(40, 1000), (200, 5000), (40, 9000)])    # (256, 512 and 1024 threads to a row)
def test_rows_of_so_many_finite_entries(fef, B, V, dtype):
    g = torch.Generator(device="cuda").manual_seed(51)
    x, u = _logits(B, 1, V, dtype, 52)
    for finite in (1, 2, 31, 127, 128, 129, 255, 256, 257, 300):
        y = torch.full_like(x, -math.inf)
        for b in range(B):
            ids = torch.randperm(V, generator=g, device="cuda")[:finite]
            y[b, 0, ids] = x[b, 0, ids]
        for kind in ("kpm", "p", "m", "edges"):
            _check(fef, y, 0.9, uniforms=u, **_rules(kind, B))


def test_a_single_row_leaves_no_status_behind(fef):
    x, u = _logits(1, 1, 20000, torch.float32, 61)
    bad = x.clone()
    bad[0, 0, 777] = math.nan
    k = _i32(9)
    d = fef.fef_draft_sample_truncated(bad, 1.0, top_k=k, uniforms=u)
    assert int(d.law.device_status) == fef.FEF_ERR_NONFINITE
    for logits, lens, status in ((x, 1, 0), (bad, 1, fef.FEF_ERR_NONFINITE), (bad, 0, 0), (bad, 1, fef.FEF_ERR_NONFINITE), (x, 1, 0)):
        fef.fef_draft_sample_truncated(logits, 1.0, top_k=k, uniforms=u, row_len=_i32(lens), out=d)
        assert int(d.law.device_status) == status
        assert (int(d.tokens) >= 0) == (logits is x)


def test_largest_vocabulary_and_temperatures(fef):
    V = fef.FEF_MAX_TRUNCATE_V
    x, u = _logits(1, 1, V, torch.bfloat16, 2)
    for rules in (dict(top_p=_f32(0.95)), dict(top_k=_i32(70000)), dict(min_p=_f32(1e-4)), dict()):
        _check(fef, x, uniforms=u, **rules)
    x, u = _logits(4, 1, 3000, torch.float32, 2)
    for T in (1e-3, 0.05, 50.0, 1e30):
        for kind in ("k", "p", "m", "none"):
            _check(fef, x, T, uniforms=u, **_rules(kind, 4))


def test_offsets_beyond_32_bits(fef):
    x, u = _logits(5, 16, 3000, torch.bfloat16, 41)
    far = torch.empty((5, 16, 1 << 26), dtype=torch.bfloat16, device="cuda")   # 2^32 entries before the last window's rows
    far[..., :3000] = x[..., :3000]
    k, p = _i32(40, 0, 40, 0, 40), _f32(0.9, 0.9, 1.0, 0.9, 0.7)
    a = fef.fef_draft_sample_truncated(x, 0.8, top_k=k, top_p=p, uniforms=u, V=3000)
    b = fef.fef_draft_sample_truncated(far, 0.8, top_k=k, top_p=p, uniforms=u, V=3000)
    law = fef.fef_law_truncate(far, 0.8, top_k=k, V=3000)
    for s, t in zip((a.tokens, a.conf, *a.law), (b.tokens, b.conf, *b.law)):
        assert torch.equal(s, t)
    near = fef.fef_law_truncate(x, 0.8, top_k=k, V=3000)
    tokens = a.tokens.clone()
    tokens[:, 3] = 7
    for s, t in zip(fef.fef_spec_verify_truncated(x, x, tokens, 0.8, 1, 2, a.law, near, V=3000),
                    fef.fef_spec_verify_truncated(far, far, tokens, 0.8, 1, 2, b.law, law, V=3000)):
        assert torch.equal(s, t)


def test_frequencies_follow_the_cut_law(fef):
    """A chi-square test of draws with Philox's numbers (99.99 % point of its law)."""
    from scipy.stats import chi2

    V, rounds = 400, 500
    x = (torch.randn(V, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda") * 1.5).expand(64, 32, V).contiguous()
    k = torch.full((64,), 12, dtype=torch.int32, device="cuda")
    law = fef.fef_law_truncate(x[:1, :1].contiguous(), 1.0, k[:1])
    counts = torch.zeros(V, dtype=torch.int64, device="cuda")
    for t in range(rounds // 50):
        counts += torch.bincount(fef.fef_draft_sample_truncated(x, 1.0, 77, t, k).tokens.flatten().long(), minlength=V)
    pi = torch.exp2(x[0, 0].double() * LOG2E - law.log2_norm[0, 0])
    inside = (x[0, 0] > law.cut_logit[0, 0]) | ((x[0, 0] == law.cut_logit[0, 0]) & (torch.arange(V, device="cuda") <= law.cut_id[0, 0]))
    assert int(inside.sum()) == 12 and int(counts[~inside].sum()) == 0
    n = int(counts.sum())
    stat = float((((counts[inside] - n * pi[inside]) ** 2) / (n * pi[inside])).sum())
    assert stat < chi2.ppf(0.9999, 11), stat


def test_given_outputs_streams_and_graphs(fef):
    x, u = _logits(3, 4, 20000, torch.bfloat16, 6)
    rules = _rules("kp", 3)
    want = fef.fef_draft_sample_truncated(x, 0.8, uniforms=u, **rules)
    law = fef.TruncatedLaw(*(torch.full_like(t, 77) for t in want.law))
    out = fef.TruncatedDraft(torch.full_like(want.tokens, 77), torch.full_like(want.conf, 77), law)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = fef.fef_draft_sample_truncated(x, 0.8, uniforms=u, out=out, stream=side, **rules)
    assert got is out
    side.synchronize()
    same = lambda a, b: all(torch.equal(s, t) for s, t in zip((*a[:2], *a.law), (*b[:2], *b.law)))  # noqa: E731
    assert same(got, want)
    bare = fef.TruncatedLaw(law.log2_norm, law.cut_logit, law.cut_id, None, None)   # no counts, no status, no confidences
    out.tokens.fill_(77)
    fef.fef_draft_sample_truncated(x, 0.8, uniforms=u, out=fef.TruncatedDraft(out.tokens, None, bare), **rules)
    assert torch.equal(out.tokens, want.tokens)
    graph, rnd = torch.cuda.CUDAGraph(), torch.zeros(1, dtype=torch.int32, device="cuda")
    fef.fef_draft_sample_truncated(x, 0.8, 5, 3, device_round=rnd, **rules)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        d = fef.fef_draft_sample_truncated(x, 0.8, 5, 3, device_round=rnd, **rules)
    for r in range(3):
        rnd.fill_(r)
        graph.replay()
        assert same(d, fef.fef_draft_sample_truncated(x, 0.8, 5, 3 + r, **rules))


def test_results_do_not_change_from_call_to_call(fef):
    x, u = _logits(16, 32, 126464, torch.bfloat16, 12)
    rules = _rules("p", 16)
    first = fef.fef_draft_sample_truncated(x, 1.0, uniforms=u, **rules)
    for _ in range(3):
        again = fef.fef_draft_sample_truncated(x, 1.0, uniforms=u, **rules)
        for a, b in zip((*first[:2], *first.law), (*again[:2], *again.law)):
            assert torch.equal(a, b)
    part = fef.fef_draft_sample_truncated(x[:1, :2].contiguous(), 1.0, uniforms=u[:1, :2].contiguous(), top_p=rules["top_p"][:1])
    assert torch.equal(part.tokens[0], first.tokens[0, :2])   # (few rows take another path)
    assert torch.equal(part.law.cut_id[0], first.law.cut_id[0, :2]) and torch.equal(part.law.kept[0], first.law.kept[0, :2])


# -------------------------------------------------------------- verification against cut laws ----
def _mask(x, law, V):
    ids = torch.arange(x.shape[-1], device="cuda")
    f = x.float()
    inside = (f > law.cut_logit[..., None]) | ((f == law.cut_logit[..., None]) & (ids <= law.cut_id[..., None]))
    return torch.where(inside & (ids < V), x, torch.full_like(x, -math.inf))


@pytest.mark.parametrize("B,K,V,dtype,T,kind", [
    (3, 8, 50257, torch.bfloat16, 0.7, "kp"), (2, 32, 126464, torch.bfloat16, 1.0, "p"), (5, 5, 1003, torch.float32, 1.0, "kpm"),
    (64, 4, 8000, torch.float32, 0.8, "m"), (1, 1, 9, torch.float32, 1.0, "k"), (4, 6, 40000, torch.float32, 1.2, "none"),
    (300, 3, 2000, torch.bfloat16, 1.0, "kpm")])
def test_verification_equals_the_oracle_on_masked_rows(fef, B, K, V, dtype, T, kind):
    import oracle
    from oracle.compare import compare_verify

    q, u = _logits(B, K, V, dtype, 31, pad=5)
    g = torch.Generator(device="cuda").manual_seed(32)
    rules = _rules(kind, B)
    for noise in (0.0, 0.3, 1.5):
        p = (q.float() + noise * torch.randn(q.shape, generator=g, device="cuda")).to(dtype)
        row_len = torch.randint(0, K + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        row_len[0] = K
        d = fef.fef_draft_sample_truncated(q, T, uniforms=u, row_len=row_len, V=V, **rules)
        tokens = d.tokens.clone()
        stray = torch.rand((B, K), generator=g, device="cuda") < 0.1      # drafts from elsewhere: outside their law as a rule
        tokens[stray] = torch.randint(0, V, (int(stray.sum()),), generator=g, device="cuda", dtype=torch.int32)
        other = {n: t.flip(0).contiguous() for n, t in rules.items()}     # the target's limits need not be the draft's
        law = fef.fef_law_truncate(p, T, row_len=row_len, V=V, **other)
        got = fef.fef_spec_verify_truncated(q, p, tokens, T, 99, 7, d.law, law, row_len=row_len, V=V)
        torch.cuda.synchronize()
        assert int(got.device_status) == 0
        ref = oracle.spec_verify(_mask(q, d.law, V)[..., :V].contiguous().cpu(), _mask(p, law, V)[..., :V].contiguous().cpu(),
                                 tokens.cpu(), T, 99, 7, row_len=row_len.cpu())
        rep = compare_verify(got.accept_len.cpu().numpy(), got.tokens.cpu().numpy(), got.conf.cpu().numpy(), ref)
        assert rep.ok, rep.mismatches


def test_verification_with_laws_that_are_not_cut(fef):
    q, u = _logits(4, 6, 30000, torch.float32, 3)
    p = q + 0.5 * torch.randn_like(q)
    d, law = fef.fef_draft_sample_truncated(q, 1.0, uniforms=u), fef.fef_law_truncate(p, 1.0)
    a = fef.fef_spec_verify_truncated(q, p, d.tokens, 1.0, 5, 6, d.law, law)
    b = fef.fef_spec_verify(q, p, d.tokens, 1.0, 5, 6, draft_log2_norm=d.law.log2_norm, target_log2_norm=law.log2_norm)
    for s, t in zip(a, b):
        assert torch.equal(s, t)


def test_verification_reports_bad_laws_and_rows(fef):
    q, u = _logits(4, 6, 3000, torch.float32, 3)
    p = q.clone()
    p[1, 2, 7] = math.nan
    k = _i32(30, 30, 30, 30)
    d, law = fef.fef_draft_sample_truncated(q, 1.0, uniforms=u, top_k=k), fef.fef_law_truncate(p, 1.0, top_k=k)
    r = fef.fef_spec_verify_truncated(q, p, d.tokens, 1.0, 5, 6, d.law, law)
    torch.cuda.synchronize()
    assert int(r.device_status) == fef.FEF_ERR_NONFINITE and r.accept_len.lt(0).tolist() == [False, True, False, False]
    assert (r.tokens[1] == -1).all() and (r.conf[1] == -1).all()


# ------------------------------------------------------------------------------------ refusals ----
def test_refusals(fef):
    x, u = _logits(2, 3, 64, torch.float32, 1)
    k, p = _i32(1, 2), _f32(0.5, 0.5)
    d = fef.fef_draft_sample_truncated(x, 1.0, uniforms=u, top_k=k)
    law = d.law
    calls = [lambda: fef.fef_law_truncate(x, 0.0), lambda: fef.fef_law_truncate(x, -1.0), lambda: fef.fef_law_truncate(x, math.nan),
             lambda: fef.fef_law_truncate(x, 1e-40), lambda: fef.fef_law_truncate(x[0], 1.0), lambda: fef.fef_law_truncate(x.half(), 1.0),
             lambda: fef.fef_law_truncate(x.transpose(0, 1), 1.0), lambda: fef.fef_law_truncate(x, 1.0, V=65),
             lambda: fef.fef_law_truncate(x, 1.0, top_k=p), lambda: fef.fef_law_truncate(x, 1.0, top_k=k[:1]),
             lambda: fef.fef_law_truncate(x, 1.0, top_p=k), lambda: fef.fef_law_truncate(x, 1.0, min_p=p.double()),
             lambda: fef.fef_law_truncate(x, 1.0, top_p=p[:1].expand(2)), lambda: fef.fef_law_truncate(x, 1.0, row_len=p),
             lambda: fef.fef_draft_sample_truncated(x, 1.0, uniforms=u[:1]), lambda: fef.fef_draft_sample_truncated(x, 1.0, uniforms=u.double()),
             lambda: fef.fef_draft_sample_truncated(x, 1.0, out=fef.TruncatedDraft(d.tokens[:1], d.conf, law)),
             lambda: fef.fef_law_truncate(x, 1.0, out=law._replace(cut_id=law.cut_logit)),
             lambda: fef.fef_law_truncate(x, 1.0, out=law._replace(log2_norm=None)),
             lambda: fef.fef_spec_verify_truncated(x, x, d.tokens, 0.0, 1, 1, law, law),
             lambda: fef.fef_spec_verify_truncated(x, x[:1], d.tokens, 1.0, 1, 1, law, law),
             lambda: fef.fef_spec_verify_truncated(x, x, d.tokens[:1], 1.0, 1, 1, law, law),
             lambda: fef.fef_spec_verify_truncated(x, x, d.tokens, 1.0, 1, 1, law, law._replace(cut_id=None)),
             lambda: fef.fef_spec_verify_truncated(x, x, d.tokens, 1.0, 1, 1, law, law._replace(log2_norm=law.cut_logit)),
             lambda: fef.fef_spec_verify_truncated(x, x, d.tokens, 1.0, 1, 1, law, law,
                                                   workspace=torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 24))]
    for call in calls:
        with pytest.raises(fef.FefError):
            call()
    with pytest.raises(ValueError):
        fef.fef_law_truncate(x, 1.0, top_k=k.cpu())
    torch.cuda.synchronize()
