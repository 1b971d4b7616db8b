"""The operators between the last hidden states and the verified tokens as they are used together (needs a B200): a prediction
head's layer, the output layer, rules on the logits, cut laws, draws, verification; and the decoding loops with sampling limits."""
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


def _cut(x, law, V):
    """Logits with -inf outside a cut law."""
    x = x[..., :V]
    ids, f = torch.arange(V, device="cuda"), x.float()
    cut = law.cut_logit[..., None]
    return torch.where((f > cut) | ((f == cut) & (ids <= law.cut_id[..., None])), x, torch.full_like(x, -math.inf)).contiguous()


def _verified(got, q, p, q_law, p_law, tokens, T, seed, step, V, row_len=None):
    ref = oracle.spec_verify(_cut(q, q_law, V).cpu(), _cut(p, p_law, V).cpu(), tokens.cpu(), T, seed, step,
                             row_len=None if row_len is None else row_len.cpu())
    rep = compare_verify(got.accept_len.cpu().numpy(), got.tokens.cpu().numpy(), got.conf.cpu().numpy(), ref)
    assert rep.ok, rep.mismatches[:5]


def _limits(B, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda: torch.rand((B,), generator=g, device="cuda")  # noqa: E731
    return dict(top_k=(1 + 60 * rnd()).to(torch.int32), top_p=0.6 + 0.4 * rnd(), min_p=0.05 * rnd())


@pytest.mark.parametrize("B,K,V,d,dtype", [(2, 4, 3001, 256, torch.float32), (3, 8, 20000, 512, torch.bfloat16), (5, 16, 9001, 1024, torch.float32)])
def test_from_hidden_states_to_verified_tokens(fef, B, K, V, d, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    head = (normal(d, d) / math.sqrt(d)).to(torch.bfloat16)
    bias = (0.3 * normal(d)).to(torch.bfloat16)
    output = (normal(V, d) * (2.0 / math.sqrt(d))).to(torch.bfloat16)
    layer = fef.fef_lmhead_quantize(output, 64 if d % 64 == 0 else 32)
    states = normal(B * K, d).to(torch.bfloat16)
    drafts, _ = fef.fef_hidden_transform(states, head, bias=bias, residual=states, activation="silu")      # the draft head's states
    x = states.double() @ head.double().T + bias.double()
    want = x * torch.sigmoid(x) + states.double()
    assert float(((drafts.double() - want).abs() / (1 + want.abs())).max()) < 2.0 ** -8 * 1.01
    targets = (drafts.float() + 0.3 * normal(B * K, d)).to(torch.bfloat16)
    q, _ = fef.fef_lmhead_logits_quantized(drafts, layer, dtype=dtype)
    p, _ = fef.fef_lmhead_logits_quantized(targets, layer, dtype=dtype)
    q, p = q.view(B, K, -1), p.view(B, K, -1)
    text = torch.randint(-1, V, (B, 40), generator=g, device="cuda", dtype=torch.int32)
    rules = dict(tokens=text, V=V, penalties=torch.tensor([[1.2, 0.1, 0.2]], device="cuda").expand(B, 3).contiguous())
    T, limits = 0.8, _limits(B, 3)
    q = fef.fef_logits_adjust(q, out=q, **rules).logits
    draft = fef.fef_draft_sample_truncated(q, T, 11, 3, V=V, **limits)
    p = fef.fef_logits_adjust(p, out=p, draft_tokens=draft.tokens, **rules).logits
    law = fef.fef_law_truncate(p, T, V=V, **limits)
    got = fef.fef_spec_verify_truncated(q, p, draft.tokens, T, 11, 3, draft.law, law, V=V)
    torch.cuda.synchronize()
    assert int(got.device_status) == 0 and int(draft.law.device_status) == 0 and int(law.device_status) == 0
    _verified(got, q, p, draft.law, law, draft.tokens, T, 11, 3, V)
    for b in range(B):      # every committed token is in its position's cut target law
        for i in range(K):
            x = int(got.tokens[b, i])
            if x >= 0:
                l, cut = float(p[b, i, x]), float(law.cut_logit[b, i])
                assert l > cut or (l == cut and x <= int(law.cut_id[b, i]))


def test_first_tokens_follow_the_cut_target_law(fef):
    """Whatever the draft law is cut to: the token that a window commits first has the cut target law (chi-square, 99.99 % point)."""
    from scipy.stats import chi2

    V, B, rounds = 300, 4096, 12
    g = torch.Generator(device="cuda").manual_seed(2)
    q = (torch.randn(V, generator=g, device="cuda") * 1.5).expand(B, 1, V).contiguous()
    p = (q[0, 0] + torch.randn(V, generator=g, device="cuda")).expand(B, 1, V).contiguous()
    k_p = torch.full((B,), 15, dtype=torch.int32, device="cuda")
    law = fef.fef_law_truncate(p, 1.0, k_p)
    pi = torch.exp2(_cut(p[:1], fef.TruncatedLaw(*(t[:1] for t in law[:4]), None), V)[0, 0].double() * math.log2(math.e) - law.log2_norm[0, 0])
    for k_q in (15, 6, 40):
        counts = torch.zeros(V, dtype=torch.int64, device="cuda")
        for t in range(rounds):
            d = fef.fef_draft_sample_truncated(q, 1.0, 5, t, top_k=torch.full_like(k_p, k_q))
            r = fef.fef_spec_verify_truncated(q, p, d.tokens, 1.0, 5, t, d.law, law)
            counts += torch.bincount(r.tokens[:, 0].long(), minlength=V)
        n = int(counts.sum())
        assert n == B * rounds and int(counts[pi == 0].sum()) == 0
        there = pi > 0
        stat = float((((counts[there] - n * pi[there]) ** 2) / (n * pi[there])).sum())
        assert stat < chi2.ppf(0.9999, int(there.sum()) - 1), (k_q, stat)


@pytest.mark.parametrize("with_rules", [False, True])
def test_decoding_loops_with_limits(fef, with_rules):
    from paper_2605_14305_b200.decode_loop import run_decode_loop_device, run_decode_loop_graph

    B, L, K, V, steps, k, T = 3, 24, 6, 2000, 2, 4, 0.9
    limits = _limits(B, 7)
    rules = dict(bias=torch.randn((V,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 0.3,
                 penalties=torch.tensor([[1.3, 0.2, 0.1]], device="cuda").expand(B, 3).contiguous()) if with_rules else None
    checked = []

    def eager_logits(rnd, window, row_len, inputs):
        return fef.fef_synth_logits(B, K, V, torch.float32, 2.0, 0.7, 4, rnd)

    def hook(rnd, info):
        if rnd is None:
            return
        p_law = fef.fef_law_truncate(info["p"], T, row_len=info["row_len"], **limits)
        _verified(info["result"], info["q"], info["p"], info["draft"].law, p_law, info["draft"].tokens, T, 21, rnd, V, info["row_len"])
        checked.append(rnd)

    one = run_decode_loop_device(fef, B, L, K, steps, k, eager_logits, T, 21, on_round=hook, truncate=limits, adjust=rules)
    assert len(checked) == one["rounds"] > 0 and (one["tokens"] >= 0).all()

    def captured_logits(rnd, window, row_len):
        return fef.fef_synth_logits(B, K, V, torch.float32, 2.0, 0.7, 4, 0, device_round=rnd)

    two = run_decode_loop_graph(fef, B, L, K, steps, k, captured_logits, T, 21, truncate=limits, adjust=rules)
    assert torch.equal(one["tokens"], two["tokens"]) and torch.equal(one["conf"], two["conf"])
    whole = run_decode_loop_device(fef, B, L, K, steps, k, eager_logits, T, 21, adjust=rules)
    assert not torch.equal(whole["tokens"], one["tokens"])
    # at temperature 0 no limit removes the arg-max
    greedy = [run_decode_loop_device(fef, B, L, K, 1, 0, eager_logits, 0.0, 21, truncate=t, adjust=rules)["tokens"] for t in (None, limits)]
    assert torch.equal(*greedy)


def test_calls_that_overlap(fef):
    """Draws of several batches at once on streams of their own, while products run on another."""
    streams = [torch.cuda.Stream() for _ in range(3)]
    g = torch.Generator(device="cuda").manual_seed(4)
    work = []
    for V, dtype in ((30000, torch.bfloat16), (126464, torch.float32), (5000, torch.bfloat16)):
        x = (torch.randn((4, 8, V), generator=g, device="cuda") * 2).to(dtype)
        u = torch.rand((4, 8), generator=g, device="cuda")
        limits = _limits(4, V)
        if V == 30000:
            limits = dict(top_p=limits["top_p"])
        work.append((x, u, limits, fef.fef_draft_sample_truncated(x, 1.0, uniforms=u, **limits)))
    h, w = (torch.randn((200, 1024), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    want, _ = fef.fef_hidden_transform(h, w, activation="gelu")
    torch.cuda.synchronize()
    got, outs = [], []
    for _ in range(4):
        for s, (x, u, limits, _) in zip(streams, work):
            got.append(fef.fef_draft_sample_truncated(x, 1.0, uniforms=u, stream=s, **limits))
        outs.append(fef.fef_hidden_transform(h, w, activation="gelu")[0])
    torch.cuda.synchronize()
    for i, d in enumerate(got):
        ref = work[i % 3][3]
        assert torch.equal(d.tokens, ref.tokens) and torch.equal(d.law.kept, ref.law.kept) and torch.equal(d.law.log2_norm, ref.law.log2_norm)
    assert all(torch.equal(o, want) for o in outs)
