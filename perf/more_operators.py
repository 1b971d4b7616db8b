"""Cases and plain forms of the operators on truncated laws and of the transform of hidden states.

Operators that follow one another when a speculative window is decoded:

  transform  hidden states through a prediction head's layer, activation(hidden W^T + bias) + residual, for one row up
             to all rows of a batch of windows; what comes out goes to the output layer
  sample     the laws softmax(logits / T) cut to their top-k, top-p and min-p sets, and one token of each, drawn with
             given random numbers (or the cut laws alone, as the target side needs them)
  verify     the verification of drafts when both laws are cut

`own` false: elementary torch operations.  `own` true: the package's calls.
"""
import math

import numpy as np
import torch

own = False

NEG_INF = float("-inf")
LOG2E = 1.4426950408889634


# ------------------------------------------------------------------ cases ----
def _sample(name, B, K, V, dtype, rules, law="peaked", temperature=1.0, pad=0, ragged=False, draw=True):
    return dict(name=name, op="sample", B=B, K=K, V=V, dtype=dtype, rules=rules, law=law, temperature=temperature, pad=pad,
                ragged=ragged, draw=draw)


def _verify(name, B, K, V, dtype, rules, law="peaked", temperature=1.0, pad=0, ragged=False):
    return dict(name=name, op="verify", B=B, K=K, V=V, dtype=dtype, rules=rules, law=law, temperature=temperature, pad=pad,
                ragged=ragged)


def _transform(name, rows, n, d, activation, bias, residual, out="bfloat16"):
    return dict(name=name, op="transform", rows=rows, n=n, d=d, activation=activation, bias=bias, residual=residual, out=out)


def listed():
    return [
        # one position of one request, all three rules: the smallest call, its latency
        _sample("sample_one_position", 1, 1, 126464, "float32", "kpm", temperature=0.8),
        # one speculative window, nucleus sampling
        _sample("sample_one_window", 1, 32, 126464, "bfloat16", "p"),
        # a few windows whose requests carry different rules (or none), odd vocabulary, padded rows, short windows among them
        _sample("sample_ragged_mixed", 5, 7, 50257, "bfloat16", "mixed", temperature=0.7, pad=7, ragged=True),
        # a batch of draft laws in 32 bits, top-k and top-p together
        _sample("sample_batch_float32", 16, 32, 152064, "float32", "kp", temperature=0.7),
        # the batch the verification is quoted on, nucleus sampling
        _sample("sample_full_batch", 64, 32, 126464, "bfloat16", "p"),
        # target laws of a batch: the cut laws alone; flat laws, so that tens of thousands of entries stay
        _sample("law_batch_flat", 32, 32, 126464, "bfloat16", "p", law="flat", draw=False),
        # one window against cut laws
        _verify("verify_one_window", 1, 32, 126464, "bfloat16", "kp"),
        # all windows of the batch
        _verify("verify_full_batch", 64, 32, 126464, "bfloat16", "p"),
        # one hidden state through a residual block
        _transform("transform_one_row", 1, 4096, 4096, "silu", False, True),
        # the rows of one short window, odd sizes on all sides, logits-like output in 32 bits
        _transform("transform_odd", 9, 5003, 1056, "gelu", True, False, "float32"),
        # draft and target rows of one full window
        _transform("transform_window_pair", 64, 3584, 3584, "gelu_tanh", True, False),
        # all rows of a batch
        _transform("transform_batch", 2048, 4096, 4096, "silu", True, True),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("sample", "sample", "verify", "transform", "transform"))
    if op == "transform":
        n, d = _log_uniform(rng, 128, 8192), 8 * _log_uniform(rng, 16, 1024)
        rows = min(_log_uniform(rng, 1, 2048), 2048 * 4096 * 4096 // (n * d))
        c = _transform("", rows, n, d, rng.choice(("none", "relu", "silu", "gelu", "gelu_tanh")), rng.random() < 0.5,
                       rng.random() < 0.5, rng.choice(("bfloat16", "bfloat16", "float32")))
    else:
        V = _log_uniform(rng, 500, 152064)
        K = _log_uniform(rng, 1, 64)
        B = _log_uniform(rng, 1, max(1, min(64, 64 * 32 * 126464 // (K * V) // 2)))
        dtype, rules = rng.choice(("float32", "bfloat16")), rng.choice(("k", "p", "m", "kp", "kpm", "mixed", "none"))
        law, temperature = rng.choice(("peaked", "peaked", "flat")), rng.choice((0.6, 0.7, 1.0, 1.3))
        pad, ragged = rng.choice((0, 0, 5, 24)), rng.random() < 0.5
        if op == "sample":
            c = _sample("", B, K, V, dtype, rules, law, temperature, pad, ragged, rng.random() < 0.7)
        else:
            c = _verify("", B, K, V, dtype, rules, law, temperature, pad, ragged)
    del c["name"]
    return c


# ----------------------------------------------------------------- inputs ----
def _ld(case):
    per_vec = 8 if case["dtype"] == "bfloat16" else 4
    return -(-(case["V"] + case["pad"]) // per_vec) * per_vec


def _logits(case, g, near=None):
    """[B, K, ld]: Gaussian logits, of which in a peaked law the likely hundredth stands out by 8; or close to others."""
    B, K, ld = case["B"], case["K"], _ld(case)
    out = torch.empty((B, K, ld), dtype=getattr(torch, case["dtype"]), device="cuda")
    for b in range(B):
        if near is not None:
            out[b] = near[b].float() + 0.7 * torch.randn((K, ld), generator=g, device="cuda")
            continue
        x = torch.randn((K, ld), generator=g, device="cuda") * 2
        if case["law"] == "peaked":
            x += 8 * (torch.rand((K, ld), generator=g, device="cuda") < 0.01)
        out[b] = x
    return out


def _rules(case, g):
    """top_k [B] int32, top_p [B], min_p [B] float32, or None: each request's own, as its sampling parameters say."""
    B, kind = case["B"], case["rules"]
    rnd = lambda: torch.rand((B,), generator=g, device="cuda")  # noqa: E731
    top_k = torch.exp(rnd() * math.log(1000.0)).round().to(torch.int32)
    top_p = 0.8 + 0.18 * rnd()
    min_p = 0.1 * 10.0 ** (-rnd())
    on = rnd(), rnd(), rnd()   # with mixed rules a request has each of them or not: 0, 1 and 0 turn them off
    if kind == "mixed":
        return (torch.where(on[0] < 0.5, top_k, torch.zeros_like(top_k)), torch.where(on[1] < 0.5, top_p, torch.ones_like(top_p)),
                torch.where(on[2] < 0.5, min_p, torch.zeros_like(min_p)))
    return tuple(t if letter in kind and kind != "none" else None for t, letter in zip((top_k, top_p, min_p), "kpm"))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "transform":
        rows, n, d = case["rows"], case["n"], case["d"]
        normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
        s.update(hidden=normal(rows, d), weight=normal(n, d).mul_(1.0 / math.sqrt(d)),
                 bias=normal(n).mul_(0.5) if case["bias"] else None, residual=normal(rows, n) if case["residual"] else None)
        return s
    B, K = case["B"], case["K"]
    s["row_len"] = torch.randint(0, K + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if case["ragged"] else None
    s["top_k"], s["top_p"], s["min_p"] = _rules(case, g)
    s["uniforms"] = torch.rand((B, K), generator=g, device="cuda")
    if case["op"] == "sample":
        s["logits"] = _logits(case, g)
        return s
    # a verification: the drafts and both cut laws are there already, from the calls before it
    s["draft"] = _logits(case, g)
    s["target"] = _logits(case, g, near=s["draft"])
    s["seed"], s["step"] = seed * 7919 + 11, seed % 1000
    s["q_law"] = _plain_sample(s, s["draft"])
    s["p_law"] = _plain_sample(s, s["target"])
    return s


# -------------------------------------------------------------- plain form ----
def _plain_sample(s, logits):
    """Cut laws, and the token that each row's random number picks.  In 64 bits: whether an entry belongs to a set, or which
    one a number falls on, is decided by sums next to a border."""
    case = s["case"]
    B, K, V, T = case["B"], case["K"], case["V"], float(torch.tensor(case["temperature"], dtype=torch.float32))
    dev = logits.device
    at = torch.arange(V, device=dev)
    out = {n: [] for n in ("tokens", "conf", "log2_norm", "cut_logit", "cut_id", "kept")}
    no = torch.zeros((), dtype=torch.bool, device=dev)
    for b in range(B):
        v, ids = torch.sort(logits[b, :, :V].float(), dim=-1, descending=True, stable=True)   # ties: lowest id first
        w = torch.exp((v.double() - v[:, :1].double()) / T)
        keep = v > NEG_INF
        cut = no
        if s["top_k"] is not None:
            k = s["top_k"][b]
            on = (k > 0) & (k < V)
            keep, cut = keep & (~on | (at < k)), cut | on
        if s["top_p"] is not None:   # the shortest prefix whose mass is at least top_p of what top_k left
            p = s["top_p"][b].double()
            upto = torch.cumsum(w * keep, -1)
            before = torch.cat((torch.zeros_like(upto[:, :1]), upto[:, :-1]), -1)
            keep, cut = keep & ((p >= 1) | (before < p * upto[:, -1:]) | (at == 0)), cut | (p < 1)
        if s["min_p"] is not None:
            m = s["min_p"][b].double()
            keep, cut = keep & ((m <= 0) | (w >= m)), cut | (m > 0)
        w = w * keep
        n = keep.sum(-1, dtype=torch.int32)
        last = (n - 1).long()[:, None]
        of_id = torch.zeros_like(w).scatter_(1, ids, w)
        upto = torch.cumsum(of_id, -1)
        total = upto[:, -1:]
        token = (upto <= s["uniforms"][b].double()[:, None] * total).sum(-1, dtype=torch.int64)
        out["tokens"].append(token.to(torch.int32))
        out["conf"].append((of_id.gather(1, token[:, None]) / total)[:, 0].float())
        out["log2_norm"].append(v[:, 0].double() * (LOG2E / T) + torch.log2(total[:, 0]))
        out["cut_logit"].append(torch.where(cut, v.gather(1, last)[:, 0], torch.full_like(v[:, 0], NEG_INF)))
        out["cut_id"].append(torch.where(cut, ids.gather(1, last)[:, 0], torch.full_like(last[:, 0], -1)).to(torch.int32))
        out["kept"].append(n)
    out = {n: torch.stack(t) for n, t in out.items()}
    if s["row_len"] is not None:   # positions behind a window's end
        unused = torch.arange(K, device=dev) >= s["row_len"][:, None]
        for n, value in (("tokens", -1), ("conf", -1.0), ("log2_norm", 0.0), ("cut_logit", 0.0), ("cut_id", -1), ("kept", 0)):
            out[n] = torch.where(unused, torch.full_like(out[n], value), out[n])
    return out


def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 of tensors of counter words (int64 tensors that hold 32 bits)."""
    low = 0xFFFFFFFF
    k0, k1 = seed & low, (seed >> 32) & low

    def wide(a, m):   # a * m in halves: 32 x 16 bits fit
        lo, hi = a * (m & 0xFFFF), a * (m >> 16)
        mid = hi + (lo >> 16)
        return mid >> 16, ((mid & 0xFFFF) << 16) | (lo & 0xFFFF)

    for _ in range(10):
        h0, l0 = wide(c0, 0xD2511F53)
        h1, l1 = wide(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _uniform(word):
    return ((word >> 9).double() + 0.5) / 8388608.0


def _plain_probability(x, ids, law, at, T):
    """Probabilities of entries x (with their ids) under a cut law."""
    cut, last = law["cut_logit"][at], law["cut_id"][at]
    while cut.dim() < x.dim():
        cut, last = cut[..., None], last[..., None]
    norm = law["log2_norm"][at].view(cut.shape)
    inside = (x > cut) | ((x == cut) & (ids <= last))
    return torch.where(inside, torch.exp2(x.double() * (LOG2E / T) - norm), torch.zeros_like(norm))


def _plain_verify(s):
    case = s["case"]
    B, K, V, T = case["B"], case["K"], case["V"], float(torch.tensor(case["temperature"], dtype=torch.float32))
    p, q = s["target"], s["draft"]
    dev, seed, step = p.device, s["seed"], s["step"]
    tokens = s["q_law"]["tokens"]
    x = tokens.clamp(min=0).long()[..., None]
    n = torch.full((B,), K, device=dev) if s["row_len"] is None else s["row_len"].long()
    everywhere = slice(None), slice(None)
    pi = _plain_probability(p.gather(2, x)[..., 0].float(), x[..., 0], s["p_law"], everywhere, T)
    rho = _plain_probability(q.gather(2, x)[..., 0].float(), x[..., 0], s["q_law"], everywhere, T)
    window, i = torch.arange(B, device=dev), torch.arange(K, device=dev)
    zero = torch.zeros((B, K), dtype=torch.int64, device=dev)
    u = _uniform(_philox(zero, zero + window[:, None], zero + i, zero + step, seed)[0])
    accept = torch.where(rho > 0, u <= pi / rho, pi > 0) | (i >= n[:, None])
    a = accept.long().cumprod(-1).sum(-1).clamp(max=n)
    # the corrected token of the first rejected position
    at = a.clamp(max=K - 1)
    ids = torch.arange(V, device=dev).expand(B, V)
    lp, lq = p[window, at, :V].float(), q[window, at, :V].float()
    pi_row = _plain_probability(lp, ids, s["p_law"], (window, at), T)
    r = pi_row - _plain_probability(lq, ids, s["q_law"], (window, at), T)
    quads = torch.arange((V + 3) // 4, device=dev).expand(B, -1) | (1 << 30)
    w = _philox(quads, window[:, None].expand_as(quads), at[:, None].expand_as(quads), torch.full_like(quads, step), seed)
    u = _uniform(torch.stack(w, -1).view(B, -1)[:, :V])
    score = torch.where(r > 0, torch.log(r) - torch.log(-torch.log(u)), NEG_INF)
    z = torch.where((r > 0).any(-1), torch.argmax(score, -1), torch.argmax(lp, -1))
    fix = (i == a[:, None]) & (a < n)[:, None]
    kept = i < a[:, None]
    out = torch.where(kept, tokens, torch.where(fix, z[:, None].to(torch.int32), torch.full_like(tokens, -1)))
    conf = torch.where(kept, pi.float(), torch.where(fix, pi_row.gather(1, z[:, None]).float(), torch.full_like(pi, -1.0).float()))
    return dict(accept_len=a.to(torch.int32), tokens=out, conf=conf)


def _plain_transform(s):
    case = s["case"]
    y = s["hidden"].float() @ s["weight"].float().T
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if case["activation"] == "relu":
        y = torch.where(y > 0, y, torch.zeros_like(y))
    elif case["activation"] == "silu":
        y = y / (1.0 + torch.exp(-y))
    elif case["activation"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    elif case["activation"] == "gelu_tanh":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return dict(out=y.to(getattr(torch, case["out"])))


# --------------------------------------------------------------------- run ----
def _laws(got):
    return dict(log2_norm=got.log2_norm, cut_logit=got.cut_logit, cut_id=got.cut_id, kept=got.kept)


def run(s):
    case = s["case"]
    if own:
        import paper_2605_14305_b200 as fef

        if case["op"] == "transform":
            out, _ = fef.fef_hidden_transform(s["hidden"], s["weight"], bias=s["bias"], residual=s["residual"],
                                              activation=case["activation"], dtype=getattr(torch, case["out"]))
            return dict(out=out)
        if case["op"] == "verify":
            laws = [fef.TruncatedLaw(s[n]["log2_norm"], s[n]["cut_logit"], s[n]["cut_id"], s[n]["kept"], None)
                    for n in ("q_law", "p_law")]
            r = fef.fef_spec_verify_truncated(s["draft"], s["target"], s["q_law"]["tokens"], case["temperature"], s["seed"],
                                              s["step"], *laws, row_len=s["row_len"], V=case["V"])
            return dict(accept_len=r.accept_len, tokens=r.tokens, conf=r.conf)
        rules = dict(top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], row_len=s["row_len"], V=case["V"])
        if not case["draw"]:
            return _laws(fef.fef_law_truncate(s["logits"], case["temperature"], **rules))
        r = fef.fef_draft_sample_truncated(s["logits"], case["temperature"], uniforms=s["uniforms"], **rules)
        return dict(tokens=r.tokens, conf=r.conf, **_laws(r.law))
    if case["op"] == "transform":
        return _plain_transform(s)
    if case["op"] == "verify":
        return _plain_verify(s)
    got = _plain_sample(s, s["logits"])
    laws = {n: got[n] for n in ("log2_norm", "cut_logit", "cut_id", "kept")}
    return laws if not case["draw"] else dict(tokens=got["tokens"], conf=got["conf"], **laws)


def work(case):
    if case["op"] == "transform":
        rows, n, d = case["rows"], case["n"], case["d"]
        out = rows * n * (2 if case["out"] == "bfloat16" else 4)
        extra = (rows * n * 2 if case["residual"] else 0) + (n * 2 if case["bias"] else 0)
        return dict(bytes=(rows + n) * d * 2 + out + extra, flops=2 * rows * n * d)
    B, K, V, size = case["B"], case["K"], case["V"], 2 if case["dtype"] == "bfloat16" else 4
    used = 0.5 if case["ragged"] else 1.0
    if case["op"] == "verify":   # both rows of the rejected position; a window without one is rare
        return dict(bytes=used * B * (2 * V * size + K * 60), flops=used * B * V * 12)
    return dict(bytes=used * B * K * (V * size + 28), flops=used * B * K * V * 4)


# ------------------------------------------------------------------- exact ----
def _exact_rows(s, logits):
    case = s["case"]
    B, K, V, T = case["B"], case["K"], case["V"], float(np.float32(case["temperature"]))
    names = dict(tokens=-1, conf=-1.0, log2_norm=0.0, cut_logit=0.0, cut_id=-1, kept=0)
    whole = ("tokens", "cut_id", "kept")
    out = {n: torch.full((B, K), v, dtype=torch.int32 if n in whole else torch.float64, device="cuda") for n, v in names.items()}
    lens = [K] * B if s["row_len"] is None else s["row_len"].tolist()
    rule = lambda n, b, off: off if s[n] is None else s[n][b].item()  # noqa: E731
    for b in range(B):
        k, p, m = rule("top_k", b, 0), rule("top_p", b, 1.0), rule("min_p", b, 0.0)
        for i in range(lens[b]):
            y = logits[b, i, :V].double()
            order = torch.argsort(-y, stable=True)
            law = torch.exp(y / T - torch.logsumexp(y / T, 0))
            n = torch.count_nonzero(torch.isfinite(y))
            if 0 < k < V:
                n = n.clamp(max=k)
            if p < 1:
                mass = law[order].cumsum(0)
                n = torch.minimum(n, torch.searchsorted(mass, p * mass[n - 1]) + 1)
            if m > 0:
                n = torch.minimum(n, torch.count_nonzero(law / law.max() >= m))
            first = order[:n]
            mask = torch.zeros_like(law)
            mask[first] = law[first]
            mass = mask.cumsum(0)
            token = torch.searchsorted(mass, s["uniforms"][b, i].double() * mass[-1], right=True)
            out["tokens"][b, i], out["conf"][b, i] = token, law[token] / mass[-1]
            out["log2_norm"][b, i] = (torch.logsumexp(y[first] / T, 0)) / math.log(2.0)
            active = 0 < k < V or p < 1 or m > 0
            out["cut_logit"][b, i], out["cut_id"][b, i] = (y[first[-1]], first[-1]) if active else (NEG_INF, -1)
            out["kept"][b, i] = n
    return out


def _exact_words(first, b, i, step, seed):
    """Output words of Philox4x32-10 for counters (first, b, i, step), on the host."""
    m0, m1 = np.uint64(0xD2511F53), np.uint64(0xCD9E8D57)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.asarray(first, dtype=np.uint64)] + [np.full(len(first), v, dtype=np.uint64) for v in (b, i, step)]
    for r in range(10):
        key0 = np.uint64(((seed & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF)
        key1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        a, d = c[0] * m0, c[2] * m1
        c = [(d >> half) ^ c[1] ^ key0, d & low, (a >> half) ^ c[3] ^ key1, a & low]
    return np.stack(c, -1)


def _exact_verify(s):
    case = s["case"]
    B, K, V, T = case["B"], case["K"], case["V"], float(np.float32(case["temperature"]))
    accept_len = torch.zeros((B,), dtype=torch.int32)
    tokens = torch.full((B, K), -1, dtype=torch.int32)
    conf = torch.full((B, K), -1.0, dtype=torch.float64)
    lens = [K] * B if s["row_len"] is None else s["row_len"].tolist()
    drafts, ids = s["q_law"]["tokens"].cpu(), torch.arange(V, device="cuda")

    def law_of(logits, law, b, i):
        y = logits[b, i, :V].double()
        cut, last = law["cut_logit"][b, i].double(), law["cut_id"][b, i]
        outside = (y < cut) | ((y == cut) & (ids > last))
        return torch.exp((y / T - law["log2_norm"][b, i] * math.log(2.0))).masked_fill(outside, 0.0)

    uniform = lambda w: ((w >> np.uint64(9)).astype(np.float64) + 0.5) * 2.0 ** -23  # noqa: E731
    for b in range(B):
        for i in range(lens[b]):
            pi, rho = law_of(s["target"], s["p_law"], b, i), law_of(s["draft"], s["q_law"], b, i)
            x = int(drafts[b, i])
            u = float(uniform(_exact_words([0], b, i, s["step"], s["seed"])[0, 0]))
            here, there = float(pi[x]), float(rho[x])
            if (u * there <= here) if there > 0 else here > 0:
                accept_len[b], tokens[b, i], conf[b, i] = i + 1, x, here
                continue
            words = _exact_words(np.arange((V + 3) // 4) | (1 << 30), b, i, s["step"], s["seed"]).reshape(-1)[:V]
            rest = (pi - rho).clamp(min=0.0)
            weight = rest / -torch.log(torch.from_numpy(uniform(words)).cuda())
            z = int(weight.argmax()) if float(rest.max()) > 0 else int(pi.argmax())
            tokens[b, i], conf[b, i] = z, float(pi[z])
            break
    return dict(accept_len=accept_len.cuda(), tokens=tokens.cuda(), conf=conf.cuda())


def _exact_transform(s):
    y = torch.einsum("rd,nd->rn", s["hidden"].double(), s["weight"].double())
    if s["bias"] is not None:
        y += s["bias"].double()[None, :]
    act = s["case"]["activation"]
    if act == "relu":
        y = y.clamp(min=0.0)
    elif act == "silu":
        y = y * torch.sigmoid(y)
    elif act == "gelu":
        y = y * torch.special.ndtr(y)
    elif act == "gelu_tanh":   # (1 + tanh z) / 2 = sigmoid(2 z)
        y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
    return dict(out=y if s["residual"] is None else y + s["residual"].double())


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "transform":
        return _exact_transform(s)
    if case["op"] == "verify":
        return _exact_verify(s)
    got = _exact_rows(s, s["logits"])
    return got if case["draw"] else {n: got[n] for n in ("log2_norm", "cut_logit", "cut_id", "kept")}
