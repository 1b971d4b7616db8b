"""The operators on logits and on the 4-bit output layer as they are used together (needs a B200): hidden states through the
quantised product, both laws adjusted, draft draws, verification with both normalisers; and the decoding loop with rules."""
import math

import pytest
import torch

import oracle
from oracle.compare import compare_verify

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fef():
    import paper_2605_14305_b200 as lib

    lib.load(build_if_missing=True)
    return lib


def _rules(B, V, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    words = torch.randint(-(1 << 31), 1 << 31, (B, (V + 31) // 32), generator=g, device="cuda").to(torch.int32)
    words[0] = -1
    return dict(penalties=torch.rand((B, 3), generator=g, device="cuda") * torch.tensor([0.5, 0.3, 0.3], device="cuda")
                + torch.tensor([1.0, 0.0, 0.0], device="cuda"),
                bias=torch.randn((V,), generator=g, device="cuda") * 0.2, allowed=words)


def _verified(got, q, p, tokens, T, seed, step, row_len=None, V=None):
    ref = oracle.spec_verify(q.cpu(), p.cpu(), tokens.cpu(), T, seed, step, row_len=None if row_len is None else row_len.cpu(), V=V)
    rep = compare_verify(got.accept_len.cpu().numpy(), got.tokens.cpu().numpy(), got.conf.cpu().numpy(), ref)
    assert rep.ok, rep.mismatches[:5]
    return rep


@pytest.mark.parametrize("B,K,V,d,group,dtype", [(2, 4, 3001, 256, 64, torch.float32), (3, 8, 5000, 512, 128, torch.bfloat16),
                                                 (4, 16, 4099, 160, 32, torch.float32)])
def test_from_hidden_states_to_verified_tokens(fef, B, K, V, d, group, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    weight = (torch.randn((V, d), generator=g, device="cuda") * (2.0 / math.sqrt(d))).to(torch.bfloat16)
    layer = fef.fef_lmhead_quantize(weight, group, zero_points=group == 64)
    hq = torch.randn((B * K, d), generator=g, device="cuda")
    hp = hq + 0.35 * torch.randn((B * K, d), generator=g, device="cuda")
    q, _ = fef.fef_lmhead_logits_quantized(hq.to(torch.bfloat16), layer, dtype=dtype)
    p, _ = fef.fef_lmhead_logits_quantized(hp.to(torch.bfloat16), layer, dtype=dtype)
    q, p = q.view(B, K, -1), p.view(B, K, -1)
    text = torch.randint(-1, V, (B, 40), generator=g, device="cuda", dtype=torch.int32)
    rules = dict(_rules(B, V, 5), tokens=text, V=V)
    T = 0.8
    q = fef.fef_logits_adjust(q, temperature=T, out=q, **rules).logits
    draft = fef.fef_draft_sample(q, T, 11, 3, V=V)
    p, norm = fef.fef_logits_adjust(p, temperature=T, out=p, draft_tokens=draft.tokens, with_norm=True, **rules)
    got = fef.fef_spec_verify(q, p, draft.tokens, T, 11, 3, V=V, draft_log2_norm=draft.log2_norm, target_log2_norm=norm)
    torch.cuda.synchronize()
    assert int(got.device_status.item()) == 0 and int(draft.device_status.item()) == 0
    _verified(got, q, p, draft.tokens, T, 11, 3, V=V)
    # the verification takes normalisers that are right to 2e-6
    z = p[..., :V].double() * (math.log2(math.e) / float(torch.tensor(T, dtype=torch.float32)))
    top = z.amax(-1, keepdim=True)
    exact = top[..., 0] + torch.log2(torch.exp2(z - top).sum(-1))
    assert float((norm - exact).abs().max()) <= 2e-6 / math.log(2.0)
    # nothing that the mask forbids was drawn or committed
    words = rules["allowed"].cpu()
    for t in (draft.tokens, got.tokens):
        for b, row in enumerate(t.cpu().tolist()):
            assert all(x < 0 or words[b, x // 32].item() >> (x % 32) & 1 for x in row)


@pytest.mark.parametrize("T", [0.05, 0.1, 0.2, 1.0])
@pytest.mark.parametrize("top", [60.0, 25.0, -60.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_normalisers_of_adjusted_rows_belong_to_the_laws_of_the_verification(fef, T, top, dtype):
    """Low temperatures and large logits: a normaliser under another rounding of log2(e) / T than the one the verification
    evaluates the law with is off in proportion to the logits."""
    B, K, V = 6, 16, 3000
    g = torch.Generator(device="cuda").manual_seed(int(top) + 100)
    q = torch.randn((B, K, V), generator=g, device="cuda") * 0.25 + top
    p = (q + 0.1 * torch.randn((B, K, V), generator=g, device="cuda")).to(dtype)
    q = q.to(dtype)
    rules = dict(bias=torch.randn((B, V), generator=g, device="cuda") * 0.1, temperature=T)
    q = fef.fef_logits_adjust(q, **rules).logits
    draft = fef.fef_draft_sample(q, T, 5, 8)
    p, norm = fef.fef_logits_adjust(p, draft_tokens=draft.tokens, with_norm=True, **rules)
    got = fef.fef_spec_verify(q, p, draft.tokens, T, 5, 8, draft_log2_norm=draft.log2_norm, target_log2_norm=norm)
    both = fef.fef_draft_sample(q, T, 5, 8, target_logits=p)
    torch.cuda.synchronize()
    assert int(got.device_status.item()) == 0 and torch.equal(both.tokens, draft.tokens)
    _verified(got, q, p, draft.tokens, T, 5, 8)
    # the two calls that deliver the target rows' normalisers agree within what each may be off by
    assert float((norm - both.target_log2_norm).abs().max()) <= 2 * 2e-6 / math.log(2.0)
    # and each of them is, within that and the law's rounded scale (2^-24 of log2 V at most), what the header says
    z = p.double() * (math.log2(math.e) / float(torch.tensor(T, dtype=torch.float32)))
    peak = z.amax(-1, keepdim=True)
    exact = peak[..., 0] + torch.log2(torch.exp2(z - peak).sum(-1))
    for n in (norm, both.target_log2_norm):
        assert float((n - exact).abs().max()) <= 2e-6 / math.log(2.0) + 2.0 ** -24 * math.log2(V)


def test_a_mask_that_leaves_nothing_is_reported(fef):
    V = 500
    q = torch.randn((2, 3, 504), device="cuda")
    words = torch.full((2, 3, 16), -1, dtype=torch.int32, device="cuda")
    words[1, 1] = 0
    p, norm = fef.fef_logits_adjust(q, allowed=words, V=V, with_norm=True)
    tok = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    draft = fef.fef_draft_sample(q, 1.0, 1, 1, V=V)
    got = fef.fef_spec_verify(q, p, tok, 1.0, 1, 1, V=V, draft_log2_norm=draft.log2_norm, target_log2_norm=norm)
    torch.cuda.synchronize()
    assert int(got.device_status.item()) == fef.FEF_ERR_NONFINITE
    assert int(got.accept_len[1]) == -1 and int(got.accept_len[0]) >= 0


@pytest.mark.parametrize("when", [0, 3])
def test_a_mask_that_leaves_nothing_ends_the_loops(fef, when):
    """... with an error, from the first round on or from a later one, the replayed loop like the eager one."""
    from paper_2605_14305_b200.decode_loop import run_decode_loop_device, run_decode_loop_graph

    B, L, K, V = 2, 40, 4, 300
    words = torch.full((B, K, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    last = torch.full((B, 1, 1), L, dtype=torch.int32, device="cuda")
    last[1] = when * K                                       # sequence 1: nothing is allowed from this position on

    def rules(rnd, window, row_len, drafts):
        return dict(allowed=torch.where(window[:, :, None] < last, words, 0))

    def eager(rnd, window, row_len, inputs):
        return fef.fef_synth_logits(B, K, V, torch.float32, 2.0, 0.7, 4, rnd)

    def captured(rnd, window, row_len):
        return fef.fef_synth_logits(B, K, V, torch.float32, 2.0, 0.7, 4, 0, device_round=rnd)

    with pytest.raises(RuntimeError, match="data error"):
        run_decode_loop_device(fef, B, L, K, 1, 0, eager, 1.0, 3, adjust=rules)
    with pytest.raises(RuntimeError, match="data error"):
        run_decode_loop_graph(fef, B, L, K, 1, 0, captured, 1.0, 3, adjust=rules)
    last[1] = L
    run_decode_loop_graph(fef, B, L, K, 1, 0, captured, 1.0, 3, adjust=rules)


@pytest.mark.parametrize("T", [1.0, 0.0])
def test_decoding_loop_with_rules(fef, T):
    from paper_2605_14305_b200.decode_loop import run_decode_loop_device, run_decode_loop_graph

    B, L, K, V, steps, k = 3, 24, 6, 2000, 2, 4
    rules = _rules(B, V, 9)
    checked = []

    def eager_logits(rnd, window, row_len, inputs):
        return fef.fef_synth_logits(B, K, V, torch.float32, 2.0, 0.7, 4, rnd)

    def hook(rnd, info):
        if rnd is None:
            return
        _verified(info["result"], info["q"], info["p"], info["draft"].tokens, T, 21, rnd, row_len=info["row_len"], V=V)
        raw_q, raw_p = fef.fef_synth_logits(B, K, V, torch.float32, 2.0, 0.7, 4, rnd)
        tokens, row_len = info["before"][0], info["row_len"]
        again_q = fef.fef_logits_adjust(raw_q, tokens=tokens, row_len=row_len, V=V, **rules).logits
        again_p = fef.fef_logits_adjust(raw_p, tokens=tokens, draft_tokens=info["draft"].tokens, row_len=row_len, V=V, **rules).logits
        used = torch.arange(K, device="cuda") < row_len[:, None]
        assert torch.equal(info["q"][used], again_q[used]) and torch.equal(info["p"][used], again_p[used])
        checked.append(rnd)

    one = run_decode_loop_device(fef, B, L, K, steps, k, eager_logits, T, 21, on_round=hook, adjust=rules)
    assert len(checked) == one["rounds"] > 0
    two = run_decode_loop_device(fef, B, L, K, steps, k, eager_logits, T, 21, adjust=lambda *_: rules)
    assert torch.equal(one["tokens"], two["tokens"]) and torch.equal(one["conf"], two["conf"])

    def captured_logits(rnd, window, row_len):
        return fef.fef_synth_logits(B, K, V, torch.float32, 2.0, 0.7, 4, 0, device_round=rnd)

    three = run_decode_loop_graph(fef, B, L, K, steps, k, captured_logits, T, 21, adjust=rules)
    assert torch.equal(one["tokens"], three["tokens"]) and torch.equal(one["conf"], three["conf"])
    words = rules["allowed"].cpu()
    for b, row in enumerate(one["tokens"].cpu().tolist()):
        assert all(words[b, x // 32].item() >> (x % 32) & 1 for x in row)
    plain = run_decode_loop_device(fef, B, L, K, steps, k, eager_logits, T, 21)
    assert not torch.equal(plain["tokens"], one["tokens"])
