"""fef_logits_adjust against the operation's definition in 64 bits (needs a B200)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

LOG2E = math.log2(math.e)


@pytest.fixture(scope="module")
def fef():
    import paper_2605_14305_b200 as lib

    lib.load(build_if_missing=True)
    return lib


def _case(B, K, V, L, dtype, seed, pad=0, drafts=True, bias="window", masks="position", ragged=False):
    """Everything a call takes, on the device."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    per_vec = 8 if dtype == torch.bfloat16 else 4
    ld = (V + pad + per_vec - 1) // per_vec * per_vec
    rnd = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    c = dict(logits=(torch.randn((B, K, ld), generator=g, device="cuda") * 3).to(dtype), V=V)
    # few different ids, so that there are repetitions; unresolved entries among them
    ids = lambda *s: (torch.randint(0, max(V // 2, 1), s, generator=g, device="cuda")).to(torch.int32)  # noqa: E731
    c["tokens"] = torch.where(rnd(B, L) < 0.15, torch.full((B, L), -1, dtype=torch.int32, device="cuda"), ids(B, L))
    c["prompt_len"] = torch.randint(0, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    c["penalties"] = rnd(B, 3) * torch.tensor([1.0, 0.8, 0.8], device="cuda") + torch.tensor([0.6, -0.1, -0.1], device="cuda")
    c["draft_tokens"] = ids(B, K) if drafts else None
    c["bias"] = None if bias is None else torch.randn((V,) if bias == "shared" else (B, V), generator=g, device="cuda")
    words = (V + 31) // 32
    shape = {None: None, "all": (words,), "window": (B, words), "position": (B, K, words)}[masks]
    c["allowed"] = None if shape is None else torch.randint(-(1 << 31), 1 << 31, shape, generator=g, device="cuda").to(torch.int32)
    c["row_len"] = torch.randint(0, K + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if ragged else None
    return c


def _reference(c):
    """(adjusted rows in 64 bits, bound of the error of the binary32 arithmetic), [B, K, V] each, on the host."""
    V = c["V"]
    l = c["logits"][..., :V].double().cpu()
    B, K = l.shape[:2]
    y, slack = l.clone(), torch.zeros_like(l)
    for b in range(B):
        rep, freq, pres = (1.0, 0.0, 0.0) if c["penalties"] is None else c["penalties"][b].double().tolist()
        text = [] if c["tokens"] is None else c["tokens"][b].tolist()
        prompt = 0 if c["prompt_len"] is None else int(c["prompt_len"][b])
        h, a = torch.zeros(V, dtype=torch.int64), torch.zeros(V, dtype=torch.float64)
        for t, x in enumerate(text):
            if 0 <= x < V:
                h[x] += 1
                a[x] += t >= prompt
        for i in range(K):
            v = l[b, i]
            if c["penalties"] is not None:
                v = torch.where(h > 0, torch.where(v > 0, v / rep, v * rep), v)
            base = v.abs()
            down = (freq * a + pres * (a > 0)) if c["penalties"] is not None else torch.zeros(V, dtype=torch.float64)
            up = torch.zeros(V, dtype=torch.float64)
            if c["bias"] is not None:
                up = (c["bias"] if c["bias"].dim() == 1 else c["bias"][b])[:V].double().cpu()
            y[b, i] = v + (up - down)
            # one rounding each of the quotient, of freq a + pres, of bias - that, and of the sum
            slack[b, i] = 2.0 ** -24 * 1.001 * (base + (abs(freq) * a + abs(pres) * (a > 0)) + (up - down).abs() + y[b, i].abs())
            if c["allowed"] is not None:
                w = c["allowed"].cpu()
                w = w if w.dim() == 1 else w[b] if w.dim() == 2 else w[b, i]
                x = torch.arange(V)
                y[b, i][(w.long()[x // 32] >> (x % 32)) & 1 == 0] = -math.inf
            if c["draft_tokens"] is not None:
                x = int(c["draft_tokens"][b, i])
                if 0 <= x < V:
                    h[x] += 1
                    a[x] += 1
    return y, slack


def _norm_reference(stored, T):
    """log2-normalisers of the stored rows in 64 bits, and the bound of the kernel's error.  A term 2^((l - m) c) carries three
    roundings of its argument (the difference, c, the product: relative 2^-24 each), whose weighted mean is at most log2 V;
    ex2 is within 2^-22, and it is applied twice (the warps' sums are joined); a term passes 22 additions in binary32."""
    T = float(torch.tensor(T or 1.0, dtype=torch.float32))   # the call takes T in binary32: 0.05 is 1.5e-8 larger there
    z = stored.double() * (LOG2E / T)
    top = z.amax(-1, keepdim=True)
    ref = top[..., 0] + torch.log2(torch.exp2(z - top).sum(-1))
    V = stored.shape[-1]
    tol = (2 * 2.0 ** -22 + 24 * 2.0 ** -24) / math.log(2.0) + 3 * 2.0 ** -24 * math.log2(V) + 2.0 ** -50 * ref.abs()
    return ref, tol


def _check(fef, c, T=1.0, in_place=False, expect_out=None):
    dtype, V = c["logits"].dtype, c["V"]
    B, K = c["logits"].shape[:2]
    y, slack = _reference(c)
    args = {k: v for k, v in c.items() if k != "logits"}
    if in_place:
        out = c["logits"].clone()
        before = out.clone()
        r = fef.fef_logits_adjust(out, out=out, temperature=T, with_norm=True, **args)
    else:
        out = torch.full_like(c["logits"], 77.0)
        before = out.clone()
        r = fef.fef_logits_adjust(c["logits"], out=out, temperature=T, with_norm=True, **args)
    torch.cuda.synchronize()
    assert r.logits is out
    n = torch.full((B,), K) if c["row_len"] is None else c["row_len"].cpu()
    used = torch.arange(K) < n[:, None]
    got = out[..., :V].cpu().double()
    # rows behind row_len and the padding are left as they were
    assert torch.equal(out.cpu()[~used].view(torch.int16 if dtype == torch.bfloat16 else torch.int32),
                       before.cpu()[~used].view(torch.int16 if dtype == torch.bfloat16 else torch.int32))
    assert torch.equal(out[..., V:], before[..., V:])
    got, y, slack = got[used], y[used], slack[used]
    fine = torch.isfinite(y)
    assert torch.equal(torch.isnan(got), torch.isnan(y))
    rest = ~fine & ~torch.isnan(y)
    assert torch.equal(got[rest], y[rest])
    half = torch.finfo(dtype).eps / 2 if dtype == torch.bfloat16 else 0.0   # (binary32: the last rounding is in `slack`)
    bound = slack + half * (y.abs() + slack) + 1e-38
    err = (got - y).abs()[fine]
    assert (err <= bound[fine]).all(), float((err / bound[fine]).max())
    norm = r.log2_norm.cpu()
    assert (norm[~used] == 0).all()
    ref, tol = _norm_reference(out[..., :V].cpu()[used], T)
    ok = torch.isfinite(ref)
    assert torch.isnan(norm[used][~ok]).all()
    assert ((norm[used] - ref).abs()[ok] <= tol[ok]).all(), float(((norm[used] - ref).abs()[ok] / tol[ok]).max())
    return r


CASES = [
    # B, K, V, L, dtype, options
    (1, 1, 1, 0, torch.float32, dict(bias=None, masks=None, drafts=False)),
    (1, 1, 1, 1, torch.bfloat16, dict(masks=None)),
    (2, 3, 7, 1, torch.float32, dict(pad=3)),
    (2, 4, 8, 5, torch.bfloat16, dict(bias="shared", masks="all")),
    (3, 5, 33, 100, torch.bfloat16, dict(pad=9, ragged=True)),
    (3, 9, 31, 50, torch.float32, dict(ragged=True, masks="window")),
    (1, 64, 2047, 300, torch.bfloat16, dict()),
    (2, 6, 2048, 1000, torch.float32, dict(bias="shared")),
    (2, 6, 2049, 1003, torch.bfloat16, dict(ragged=True)),
    (5, 8, 4099, 257, torch.float32, dict(ragged=True, drafts=False)),
    (2, 32, 5003, 9001, torch.bfloat16, dict(pad=40)),
    (1, 2, 50257, 40000, torch.bfloat16, dict()),
    (1, 5, 152064, 700, torch.float32, dict(masks="window")),
    (40, 3, 1000, 33, torch.bfloat16, dict(ragged=True, bias=None)),
]


@pytest.mark.parametrize("B,K,V,L,dtype,options", CASES)
def test_against_the_definition(fef, B, K, V, L, dtype, options):
    _check(fef, _case(B, K, V, L, dtype, seed=V + L, **options), T=0.7)


@pytest.mark.parametrize("T", [0.0, 0.05, 1.0, 20.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_temperatures_and_in_place(fef, T, dtype):
    _check(fef, _case(3, 7, 3001, 64, dtype, seed=4), T=T, in_place=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_each_rule_alone(fef, dtype):
    full = _case(2, 5, 2500, 80, dtype, seed=9)
    none = dict.fromkeys(("tokens", "prompt_len", "draft_tokens", "penalties", "bias", "allowed", "row_len"))
    r = _check(fef, dict(none, logits=full["logits"], V=2500))
    assert torch.equal(r.logits[..., :2500], full["logits"][..., :2500])            # nothing asked for: a copy
    for keep in (("bias",), ("allowed",), ("tokens", "penalties"), ("draft_tokens", "penalties"),
                 ("tokens", "prompt_len", "penalties")):
        _check(fef, dict(none, logits=full["logits"], V=2500, **{k: full[k] for k in keep}))
    # a text without penalties changes nothing
    r = _check(fef, dict(none, logits=full["logits"], V=2500, tokens=full["tokens"], draft_tokens=full["draft_tokens"]))
    assert torch.equal(r.logits[..., :2500], full["logits"][..., :2500])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_that_are_not_numbers(fef, dtype):
    c = _case(2, 6, 700, 40, dtype, seed=2)
    l, low = c["logits"], torch.finfo(dtype).min
    c["penalties"][:, 0] = 1.25
    c["allowed"].fill_(-1)
    c["allowed"][0, 0] = 0                                  # row (0, 0): nothing is left
    for x, bad in ((3, math.nan), (40, math.inf), (77, -math.inf), (100, low), (200, -low)):
        l[0, 1, x] = bad                                    # row (0, 1): all of it masked away
        c["allowed"][0, 1, x // 32] &= ~(1 << x % 32) if x % 32 != 31 else 0x7FFFFFFF
    l[0, 2, 5] = math.nan                                   # rows (0, 2), (0, 3): not masked
    l[0, 3, 5] = math.inf
    l[0, 4] = -math.inf                                     # nothing finite
    l[0, 5, ::2] = -math.inf
    l[1, 0] = low                                           # a row of the type's lowest value
    c["bias"][0, 9] = -math.inf                             # a ban by bias
    c["bias"][1, :] = 0.0
    c["penalties"][1] = torch.tensor([1.0, 0.0, 0.0], device="cuda")
    r = _check(fef, c)
    norm = r.log2_norm.cpu()
    assert torch.isnan(norm[0, [0, 2, 3, 4]]).all() and torch.isfinite(norm[0, [1, 5]]).all()
    assert float(norm[1, 0]) < -1e38                        # as finite as any other


def test_ids_outside_the_vocabulary_and_repeated_drafts(fef):
    c = _case(3, 64, 2100, 30, torch.float32, seed=3)
    c["tokens"][:, ::3] = torch.tensor([-1, -(1 << 31), (1 << 31) - 1, 2100, 2099, 0, 2048, 2047, -2, 5],
                                       dtype=torch.int32, device="cuda")
    c["draft_tokens"][0] = 17                               # the same draft at every position
    c["draft_tokens"][1, ::2] = -1
    c["draft_tokens"][1, 1::4] = 2100
    c["draft_tokens"][2] = (torch.arange(64, device="cuda") % 2 * 2099).to(torch.int32)
    _check(fef, c)


def test_strides_of_biases_and_masks(fef):
    c = _case(4, 5, 1001, 60, torch.bfloat16, seed=8)
    wide = torch.randn((4, 2100), device="cuda")
    words = torch.randint(-(1 << 31), 1 << 31, (4, 5, 100), device="cuda").to(torch.int32)
    for bias, allowed in ((wide[:, 3:1004], words[:, :, 7:39]), (wide[1, :1500].expand(4, -1), words[:1, :, :40].expand(4, 5, 40)),
                          (wide[0], words[:, :1, 1:33].expand(4, 5, 32)), (wide[:, 50:1051], words[2, 3])):
        _check(fef, dict(c, bias=bias, allowed=allowed))


def test_offsets_beyond_32_bits(fef):
    B, K, V = 9, 64, 2 ** 22 + 8                            # 4.8 GB of bfloat16
    logits = torch.zeros((B, K, V), dtype=torch.bfloat16, device="cuda")
    logits[-1, -1] = 1.0
    tokens = torch.full((B, 1), V - 1, dtype=torch.int32, device="cuda")
    pen = torch.tensor([[2.0, 0.0, 0.0]], device="cuda").repeat(B, 1)
    r = fef.fef_logits_adjust(logits, tokens=tokens, penalties=pen, out=logits, with_norm=True)
    torch.cuda.synchronize()
    assert float(logits[-1, -1, -1]) == 0.5 and float(logits[-1, -1, -2]) == 1.0 and float(logits[-1, -1, :-1].float().min()) == 1.0
    assert abs(float(r.log2_norm[-1, -1]) - (22 + LOG2E)) < 1e-5 and abs(float(r.log2_norm[0, 0]) - 22) < 1e-5


def test_streams_graphs_and_repeats(fef):
    c = _case(4, 16, 20001, 500, torch.bfloat16, seed=6)
    args = {k: v for k, v in c.items() if k != "logits"}
    first = fef.fef_logits_adjust(c["logits"], with_norm=True, **args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    other = fef.fef_logits_adjust(c["logits"], with_norm=True, stream=s, **args)
    s.synchronize()
    assert torch.equal(first.logits[..., :20001], other.logits[..., :20001]) and torch.equal(first.log2_norm, other.log2_norm)
    # two captured calls with scratch of their own, replayed on new contents of the same buffers
    outs = [(torch.zeros_like(c["logits"]), torch.zeros((4, 16), dtype=torch.float64, device="cuda")) for _ in range(2)]
    graphs = []
    for out, norm in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fef.fef_logits_adjust(c["logits"], out=out, log2_norm=norm, **args)
        graphs.append(graph)
    c["logits"].mul_(0.5)
    c["draft_tokens"].add_(1)
    for graph in graphs:
        graph.replay()
    again = fef.fef_logits_adjust(c["logits"], with_norm=True, **args)
    torch.cuda.synchronize()
    for out, norm in outs:
        assert torch.equal(out[..., :20001], again.logits[..., :20001]) and torch.equal(norm, again.log2_norm)
    assert not torch.equal(first.logits[..., :20001], again.logits[..., :20001])


def test_refusals(fef):
    c = _case(2, 4, 96, 10, torch.float32, seed=1)
    args = {k: v for k, v in c.items() if k not in ("logits", "V")}
    bad = [
        dict(tokens=c["tokens"].long()), dict(tokens=c["tokens"][:1]), dict(tokens=c["tokens"][:, ::2]),
        dict(prompt_len=c["prompt_len"][:1]), dict(draft_tokens=c["draft_tokens"][:, :3]), dict(row_len=torch.zeros(2, device="cuda")),
        dict(penalties=c["penalties"][:, :2]), dict(penalties=c["penalties"].double()), dict(bias=c["bias"][:, :95]),
        dict(bias=c["bias"].half()), dict(bias=c["bias"][:1]), dict(bias=c["bias"].T.contiguous().T),
        dict(allowed=c["allowed"][..., :2]), dict(allowed=c["allowed"].long()), dict(allowed=c["allowed"][:, :3]),
        dict(out=torch.empty_like(c["logits"])[:1]), dict(out=c["logits"].bfloat16()), dict(temperature=-1.0),
        dict(temperature=math.nan), dict(V=97), dict(V=0), dict(log2_norm=torch.zeros((2, 4), device="cuda")),
        dict(with_norm=True, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")),
    ]
    for change in bad:
        with pytest.raises(fef.FefError):
            fef.fef_logits_adjust(c["logits"], **{**args, **change})
    for logits in (c["logits"].half(), c["logits"][0], c["logits"][:, ::2], c["logits"][..., :50].contiguous()):
        with pytest.raises(fef.FefError):
            fef.fef_logits_adjust(logits)
    with pytest.raises(ValueError):
        fef.fef_logits_adjust(c["logits"], tokens=c["tokens"].cpu())
    fef.fef_logits_adjust(c["logits"], **args)              # and the call itself is fine


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [2048, 5003, 126464])
def test_normalisers_within_what_the_residual_draw_counts_on(fef, dtype, V):
    """2e-6 relative (fef_residual.cuh).  A term 2^((l - m) c) carries a rounding of the difference, of the product and, in binary32, of c
    (2^-24 each, relative to its argument e; bfloat16 laws have c itself in binary32), in two steps that add up to e: to its warp's
    largest and from there to the largest of 2048 ids; ex2 is within 2^-22 and applied twice, and the term passes eight additions
    in its warp and one rounding of the joined sum (the rest is in double precision).  The weighted mean of |e| over 2048 ids is
    largest when one id stands at 0 and all others together at one x."""
    x = torch.linspace(0.0, 20.0, 10001, dtype=torch.float64)
    mean = float((2047 * x * torch.exp2(-x) / (1 + 2047 * torch.exp2(-x))).max())
    roundings = 2 if dtype == torch.bfloat16 else 3
    bound = 1.01 * (roundings * 2.0 ** -24 * mean * math.log(2.0) + 2 * 2.0 ** -22 + 9 * 2.0 ** -24)
    assert bound < 2e-6
    g = torch.Generator(device="cuda").manual_seed(V)
    for T in (0.3, 1.0, 2.7):
        T = float(torch.tensor(T, dtype=torch.float32))
        rows = []
        for down in (1.0, 3.3, 4.9, 6.0, 8.0, 8.6, 11.0, 14.0, 20.0, 0.0):
            row = torch.full((V,), 7.0 - down * T * math.log(2.0), device="cuda")
            row[int(down * 100) % V] = 7.0
            rows.append(row)
        rows += [torch.randn(V, generator=g, device="cuda") * s for s in (0.1, 1.0, 3.0, 10.0)]
        ld = (V + 7) // 8 * 8
        logits = torch.zeros((2, 7, ld), device="cuda")
        logits[..., :V] = torch.stack(rows).view(2, 7, V)
        logits = logits.to(dtype)
        norm = fef.fef_logits_adjust(logits, V=V, temperature=T, with_norm=True).log2_norm
        c = LOG2E / T
        law = c if dtype == torch.float32 else float(torch.tensor(c, dtype=torch.float64).float())
        z = logits[..., :V].double() * law
        top = z.amax(-1, keepdim=True)
        ref = top[..., 0] + torch.log2(torch.exp2(z - top).sum(-1))
        off = (norm * (law / c) - ref).abs() * math.log(2.0)
        assert float(off.max()) <= bound, float(off.max())


@pytest.mark.parametrize("dtype,ld", [(torch.float32, 4), (torch.bfloat16, 8)])
def test_the_largest_batch(fef, dtype, ld):
    B, V = 65535, 3
    logits = torch.randn((B, 1, ld), device="cuda").to(dtype)
    bias = torch.randint(-8, 9, (B, V), device="cuda").float()
    allowed = (torch.arange(B, device="cuda", dtype=torch.int32) % 7 + 1)[:, None]
    r = fef.fef_logits_adjust(logits, bias=bias, allowed=allowed, V=V, with_norm=True)
    want = (logits[:, 0, :V].float() + bias).to(dtype)
    want[(allowed >> torch.arange(V, device="cuda")) & 1 == 0] = -math.inf
    assert torch.equal(r.logits[:, 0, :V], want)
    ref, tol = _norm_reference(want.cpu(), 1.0)
    assert ((r.log2_norm[:, 0].cpu() - ref).abs() <= tol).all()


def test_the_longest_text(fef):
    L = 1 << 24
    tokens = torch.full((1, L), 5, dtype=torch.int32, device="cuda")
    tokens[0, 0] = 2
    pen = torch.tensor([[2.0, 2.0 ** -24, 0.5]], device="cuda")
    logits = torch.ones((1, 3, 8), device="cuda")
    r = fef.fef_logits_adjust(logits, tokens=tokens, prompt_len=torch.tensor([L // 2], dtype=torch.int32, device="cuda"),
                              draft_tokens=torch.tensor([[2, 5, 7]], dtype=torch.int32, device="cuda"), penalties=pen)
    want = torch.ones((3, 8))
    want[:, 2], want[:, 5] = 0.5, 0.5 - (0.5 + 0.5)
    want[1:, 2] = 0.5 - (2.0 ** -24 + 0.5)
    # (position 2, id 5: freq a + pres = 1 + 2^-24 lies between two numbers of binary32 and goes to the even one, 1)
    torch.cuda.synchronize()
    assert torch.equal(r.logits[0].cpu(), want)


def test_calls_on_two_streams_at_once(fef):
    cases = [_case(8, 32, 50001, 300, torch.bfloat16, seed=21), _case(8, 16, 50001, 700, torch.float32, seed=22)]
    args = [{k: v for k, v in c.items() if k != "logits"} for c in cases]
    alone = [fef.fef_logits_adjust(c["logits"], with_norm=True, **a) for c, a in zip(cases, args)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        both = [fef.fef_logits_adjust(c["logits"], with_norm=True, stream=s, **a) for c, a, s in zip(cases, args, streams)]
        torch.cuda.synchronize()
        for x, y in zip(alone, both):
            assert torch.equal(x.logits[..., :50001], y.logits[..., :50001]) and torch.equal(x.log2_norm, y.log2_norm)
