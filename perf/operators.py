"""Cases and plain forms of the operators on logits and on the 4-bit output layer.

Three operators that follow one another when a speculative window is decoded:

  quantize  an output layer [V, d] in bfloat16 brought to 4 bits with one scale (and, asked for, one zero
            point) per group of 32, 64 or 128 weights of a row
  product   logits = hidden x that layer, for one row up to all rows of a batch of windows
  adjust    penalties for repeated tokens, biases and grammar masks on the logits of a window, with the
            normaliser of each adjusted row

`own` false: elementary torch operations in 32 bits.  `own` true: the package's calls.
"""
import math

import torch

own = False

NEG_INF = float("-inf")
LOG2E = 1.4426950408889634


# ------------------------------------------------------------------ cases ----
def _adjust(name, B, K, V, L, dtype, pad=0, temperature=1.0, ragged=False, drafts=True, bias="none", masks="none", norm=True):
    return dict(name=name, op="adjust", B=B, K=K, V=V, L=L, dtype=dtype, pad=pad, temperature=temperature, ragged=ragged,
                drafts=drafts, bias=bias, masks=masks, norm=norm)


def _product(name, rows, V, d, group, zero, out):
    return dict(name=name, op="product", rows=rows, V=V, d=d, group=group, zero=zero, out=out)


def _quantize(name, V, d, group, zero):
    return dict(name=name, op="quantize", V=V, d=d, group=group, zero=zero)


def listed():
    return [
        # one position of one sequence with repetition penalties only: the smallest call, its latency
        _adjust("adjust_one_position", 1, 1, 126464, 64, "float32", drafts=False, norm=False),
        # one speculative window under a grammar: every position has its own mask
        _adjust("adjust_one_window", 1, 32, 126464, 1024, "bfloat16", masks="position"),
        # a few windows, a vocabulary that no vector width divides, padded rows, a long history, short windows among them
        _adjust("adjust_ragged_long_history", 5, 7, 50257, 32781, "bfloat16", pad=7, temperature=0.7, ragged=True, bias="window",
                masks="position"),
        # a batch of draft laws in 32 bits: one bias for all, one mask per sequence, no drafts yet
        _adjust("adjust_batch_float32", 16, 32, 152064, 2048, "float32", drafts=False, bias="shared", masks="window"),
        # the batch the verification is quoted on, everything at once
        _adjust("adjust_full_batch", 64, 32, 126464, 1024, "bfloat16", bias="window", masks="position"),
        # one hidden state
        _product("product_one_row", 1, 126464, 4096, 128, False, "float32"),
        # the rows of one short window, the other family's sizes, zero points
        _product("product_short_window", 8, 152064, 3584, 64, True, "float32"),
        # odd sizes, smallest group
        _product("product_odd", 5, 5003, 1056, 32, True, "bfloat16"),
        # draft and target rows of one full window
        _product("product_window_pair", 64, 126464, 4096, 128, False, "float32"),
        # all rows of sixteen windows
        _product("product_batch", 512, 126464, 4096, 128, False, "bfloat16"),
        # a small layer of odd sizes
        _quantize("quantize_odd", 5003, 1056, 32, True),
        # a whole output layer
        _quantize("quantize_layer", 126464, 4096, 128, False),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("adjust", "adjust", "product", "product", "quantize"))
    if op == "adjust":
        V = _log_uniform(rng, 500, 152064)
        K = _log_uniform(rng, 1, 64)
        B = _log_uniform(rng, 1, max(1, min(64, 64 * 32 * 126464 // (K * V) // 2)))
        c = _adjust("", B, K, V, _log_uniform(rng, 1, 40000), rng.choice(("float32", "bfloat16")), pad=rng.choice((0, 0, 5, 24)),
                    temperature=rng.choice((0.0, 0.7, 1.0, 1.3)), ragged=rng.random() < 0.5, drafts=rng.random() < 0.7,
                    bias=rng.choice(("none", "shared", "window")), masks=rng.choice(("none", "window", "position")),
                    norm=rng.random() < 0.7)
    elif op == "product":
        group = rng.choice((32, 64, 128))
        V = _log_uniform(rng, 500, 152064)
        d = group * max(1, _log_uniform(rng, 128, 6144 if V < 80000 else 4096) // group)
        c = _product("", _log_uniform(rng, 1, 512), V, d, group, rng.random() < 0.5, rng.choice(("float32", "bfloat16")))
        if c["rows"] * V * d > 512 * 126464 * 4096:
            c["rows"] = 512 * 126464 * 4096 // (V * d)
    else:
        group = rng.choice((32, 64, 128))
        V = _log_uniform(rng, 500, 126464)
        c = _quantize("", V, group * max(1, _log_uniform(rng, 128, 4096) // group), group, rng.random() < 0.5)
    del c["name"]
    return c


# ----------------------------------------------------------------- inputs ----
def _ld(case):
    per_vec = 8 if case["dtype"] == "bfloat16" else 4
    return -(-(case["V"] + case["pad"]) // per_vec) * per_vec


def _pack_rows(q):
    """[V, d] values 0..15, d a multiple of 128 -> [V, d / 2] bytes: 64 bytes for every 128 columns, in which the 32-bit
    word 4 t + w holds columns 32 w + 8 t .. 32 w + 8 t + 7, lowest nibble first."""
    V, d = q.shape
    x = q.view(V, d // 128, 4, 4, 4, 2).transpose(2, 3)
    return (x[..., 0] | (x[..., 1] << 4)).reshape(V, d // 2).contiguous()


def _layer(case, g):
    """Four-bit layer as a program keeps it, from a Gaussian layer of logits with standard deviation 2."""
    V, d, group = case["V"], case["d"], case["group"]
    dp = -(-d // 128) * 128
    packed = torch.empty((V, dp // 2), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((dp // 128, (V + 31) // 32 * 32, 128 // group), dtype=torch.bfloat16, device="cuda")
    zero = torch.full(scale.shape, 8, dtype=torch.uint8, device="cuda") if case["zero"] else None
    step = max(1, (1 << 26) // d)
    for r in range(0, V, step):
        w = torch.randn((min(step, V - r), d), generator=g, device="cuda") * (2.0 / math.sqrt(d))
        w = w.view(w.shape[0], d // group, group)
        if case["zero"]:
            w += 0.3 / math.sqrt(d)  # groups that are not centred, which zero points are for
            lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
            s = ((hi - lo) / 15).to(torch.bfloat16)
            z = torch.round(-lo / s.float()).clamp(0, 15)
        else:
            s = (w.abs().amax(-1) / 7).to(torch.bfloat16)
            z = torch.full_like(s, 8.0, dtype=torch.float32)
        q = (torch.round(w / s.float()[..., None]) + z[..., None]).clamp(0, 15).to(torch.uint8)
        n = q.shape[0]
        full = torch.full((n, dp), 8, dtype=torch.uint8, device="cuda")
        full[:, :d] = q.view(n, d)
        packed[r:r + n] = _pack_rows(full)
        for src, dst in ((s, scale), (z.to(torch.uint8), zero)):
            if dst is not None:
                flat = torch.zeros((n, dp // group), dtype=dst.dtype, device="cuda")
                flat[:, :d // group] = src
                dst[:, r:r + n] = flat.view(n, dp // 128, 128 // group).transpose(0, 1)
    return packed, scale, zero


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "quantize":
        w = torch.empty((case["V"], case["d"]), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        s["weight"] = w.mul_(2.0 / math.sqrt(case["d"]))
        return s
    if case["op"] == "product":
        s["hidden"] = torch.randn((case["rows"], case["d"]), generator=g, device="cuda").to(torch.bfloat16)
        s["packed"], s["scale"], s["zero"] = _layer(case, g)
        return s
    B, K, V, L = case["B"], case["K"], case["V"], case["L"]
    dtype, ld = getattr(torch, case["dtype"]), _ld(case)
    logits = torch.empty((B, K, ld), dtype=dtype, device="cuda")
    for b in range(B):  # the likely hundredth of a vocabulary stands out by 8
        x = torch.randn((K, ld), generator=g, device="cuda") * 2
        logits[b] = x + 8 * (torch.rand((K, ld), generator=g, device="cuda") < 0.01)

    def ids(shape):  # low ids are the common ones
        return (V * torch.rand(shape, generator=g, device="cuda") ** 3).to(torch.int32).clamp_(0, V - 1)

    tokens = ids((B, L))
    tokens[torch.rand((B, L), generator=g, device="cuda") < 0.1] = -1  # positions that are still masked
    s.update(
        logits=logits, out=torch.zeros_like(logits), tokens=tokens,
        prompt_len=torch.randint(0, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32),
        drafts=ids((B, K)) if case["drafts"] else None,
        row_len=torch.randint(0, K + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if case["ragged"] else None,
        penalties=torch.rand((B, 3), generator=g, device="cuda") * 0.5 + torch.tensor([1.0, 0.0, 0.0], device="cuda"),
        bias=None, allowed=None)
    if case["bias"] != "none":
        bias = torch.randn((1 if case["bias"] == "shared" else B, V), generator=g, device="cuda")
        bias *= torch.rand(bias.shape, generator=g, device="cuda") < 0.02
        s["bias"] = bias[0] if case["bias"] == "shared" else bias
    if case["masks"] != "none":
        shape = (B, (V + 31) // 32) if case["masks"] == "window" else (B, K, (V + 31) // 32)
        words = torch.randint(-(1 << 31), 1 << 31, shape, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
        free = torch.rand(shape[:-1], generator=g, device="cuda") < 0.3  # states of the grammar that allow anything
        s["allowed"] = torch.where(free[..., None], torch.full_like(words, -1), words)
    return s


# -------------------------------------------------------------- plain form ----
def _plain_scale(case, weight):
    w = weight.float().view(case["V"], case["d"] // case["group"], case["group"])
    if case["zero"]:
        lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
        s = ((hi - lo) / 15).to(torch.bfloat16).float()
        some = torch.where(s == 0, torch.ones_like(s), s)
        z = torch.round(-lo / some).clamp(0, 15)
    else:
        s = (w.abs().amax(-1) / 7).to(torch.bfloat16).float()
        some = torch.where(s == 0, torch.ones_like(s), s)
        z = torch.full_like(s, 8.0)
    q = (torch.round(w / some[..., None]) + z[..., None]).clamp(0, 15)
    return ((q - z[..., None]) * s[..., None]).view(case["V"], case["d"])


def _plain_product(s):
    case = s["case"]
    V, d, group = case["V"], case["d"], case["group"]
    blocks = s["packed"].shape[1] // 64
    x = s["packed"].view(V, blocks, 4, 4, 4)
    q = torch.stack((x & 15, x >> 4), -1).transpose(2, 3).reshape(V, blocks * 128 // group, group).float()
    per_row = lambda t: t[:, :V].transpose(0, 1).reshape(V, blocks * 128 // group, 1).float()  # noqa: E731
    q -= per_row(s["zero"]) if s["zero"] is not None else 8.0
    q *= per_row(s["scale"])
    w = q.view(V, blocks * 128)[:, :d]
    return (s["hidden"].float() @ w.T).to(getattr(torch, case["out"]))


def _plain_adjust(s):
    case = s["case"]
    B, K, V = case["B"], case["K"], case["V"]
    dev = s["logits"].device
    tokens, rep, freq, pres = s["tokens"], *(s["penalties"].view(B, 3, 1, 1).unbind(1))
    # how often a token stands in the answer so far (freq, pres) and whether it stands anywhere (rep)
    in_prompt = torch.arange(tokens.shape[1], device=dev) < s["prompt_len"][:, None]
    known = tokens >= 0
    at = tokens.clamp(min=0).long()
    seen = torch.zeros((B, V), dtype=torch.int32, device=dev).scatter_add_(1, at, known.int())[:, None]
    count = torch.zeros((B, V), dtype=torch.int32, device=dev).scatter_add_(1, at, (known & ~in_prompt).int())[:, None]
    if s["drafts"] is not None:  # position i also counts the drafts of the window's earlier positions
        one = torch.zeros((B, K + 1, V), dtype=torch.int32, device=dev)
        one[:, 1:].scatter_(2, s["drafts"].long()[..., None], 1)
        earlier = one.cumsum(1, dtype=torch.int32)[:, :K]
        seen, count = seen + earlier, count + earlier
    x = s["logits"][..., :V].float()
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * count - pres * (count > 0)
    if s["bias"] is not None:
        x = x + (s["bias"] if s["bias"].dim() == 1 else s["bias"][:, None])
    if s["allowed"] is not None:
        words = s["allowed"] if s["allowed"].dim() == 3 else s["allowed"][:, None]
        bits = (words[..., None] >> torch.arange(32, device=dev, dtype=torch.int32)) & 1
        x = torch.where(bits.flatten(-2)[..., :V] != 0, x, NEG_INF)
    x = x.to(s["logits"].dtype)
    used = torch.ones((B, K), dtype=torch.bool, device=dev)
    if s["row_len"] is not None:
        used = torch.arange(K, device=dev) < s["row_len"][:, None]
    out = s["out"][..., :V]
    out.copy_(torch.where(used[..., None], x, out))
    if not case["norm"]:
        return dict(logits=out)
    y = x.float() * (LOG2E / (case["temperature"] or 1.0))
    top = y.amax(-1, keepdim=True)
    norm = top[..., 0] + torch.log2(torch.exp2(y - top).sum(-1))
    return dict(logits=out, log2_norm=torch.where(used, norm, torch.zeros_like(norm)))


# --------------------------------------------------------------------- run ----
def run(s):
    case = s["case"]
    if own:
        import paper_2605_14305_b200 as fef

        if case["op"] == "quantize":
            return dict(values=fef.fef_lmhead_dequantize(fef.fef_lmhead_quantize(s["weight"], case["group"], case["zero"])))
        if case["op"] == "product":
            layer = fef.QuantizedLayer(s["packed"], s["scale"], s["zero"], case["d"], case["group"])
            out, _ = fef.fef_lmhead_logits_quantized(s["hidden"], layer, dtype=getattr(torch, case["out"]))
            return dict(logits=out[:, :case["V"]])
        r = fef.fef_logits_adjust(s["logits"], tokens=s["tokens"], prompt_len=s["prompt_len"], draft_tokens=s["drafts"],
                                  penalties=s["penalties"], bias=s["bias"], allowed=s["allowed"], row_len=s["row_len"],
                                  temperature=case["temperature"], V=case["V"], out=s["out"], with_norm=case["norm"])
        got = dict(logits=r.logits[..., :case["V"]])
        if case["norm"]:
            got["log2_norm"] = r.log2_norm.float()
        return got
    if case["op"] == "quantize":
        return dict(values=_plain_scale(case, s["weight"]))
    if case["op"] == "product":
        return dict(logits=_plain_product(s))
    return _plain_adjust(s)


def work(case):
    V = case["V"]
    if case["op"] == "adjust":
        B, K, size = case["B"], case["K"], 2 if case["dtype"] == "bfloat16" else 4
        rows = B * K * (0.5 if case["ragged"] else 1.0)
        n = rows * V * size * 2 + B * case["L"] * 4
        n += {"none": 0, "shared": 1, "window": B}[case["bias"]] * V * 4
        n += {"none": 0, "window": B, "position": rows}[case["masks"]] * V / 8
        return dict(bytes=n + B * 16 + (B * K * 4 if case["norm"] else 0), flops=rows * V * (5 if case["norm"] else 2))
    d, group = case["d"], case["group"]
    if case["op"] == "quantize":
        return dict(bytes=V * d * 6, flops=V * d * 4)
    layer = V * d / 2 + V * d / group * (3 if case["zero"] else 2)
    out = case["rows"] * V * (2 if case["out"] == "bfloat16" else 4)
    return dict(bytes=layer + case["rows"] * d * 2 + out, flops=2 * case["rows"] * V * d)


# ------------------------------------------------------------------- exact ----
def _exact_layer(case, weight):
    """Values of the quantised layer in 64 bits, some rows at a time."""
    V, d, group = case["V"], case["d"], case["group"]
    out = torch.empty((V, d), dtype=torch.float64, device=weight.device)
    for r in range(0, V, 8192):
        w = weight[r:r + 8192].double().unflatten(1, (d // group, group))
        if case["zero"]:
            low, high = torch.minimum(w.min(2)[0], w.new_zeros(())), torch.maximum(w.max(2)[0], w.new_zeros(()))
            scale = ((high - low) / 15.0).to(torch.bfloat16).double().unsqueeze(2)
            centre = torch.where(scale > 0, -low.unsqueeze(2) / scale, 0.0).round().clamp(0, 15)
        else:
            scale = (torch.maximum(-w.min(2)[0], w.max(2)[0]) / 7.0).to(torch.bfloat16).double().unsqueeze(2)
            centre = torch.full_like(scale, 8.0)
        level = torch.where(scale > 0, w / scale, 0.0).round() + centre
        out[r:r + 8192] = ((level.clamp(0, 15) - centre) * scale).flatten(1)
    return out


def _exact_product(s):
    case = s["case"]
    V, d, group = case["V"], case["d"], case["group"]
    k = torch.arange(d, device="cuda")
    block, inside = k // 128, k % 128
    word, lane, nibble = inside // 32, inside % 32 // 8, inside % 8
    byte = block * 64 + lane * 16 + word * 4 + nibble // 2
    h = s["hidden"].double()
    out = torch.empty((case["rows"], V), dtype=torch.float64, device="cuda")
    for r in range(0, V, 8192):
        n = min(8192, V - r)
        level = (s["packed"][r:r + n][:, byte].int() >> (4 * (nibble % 2)).int()) & 15
        scale = s["scale"][:, r:r + n][block, :, inside // group].double().T
        centre = 8 if s["zero"] is None else s["zero"][:, r:r + n][block, :, inside // group].int().T
        out[:, r:r + n] = h @ ((level - centre).double() * scale).T
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return dict(values=_exact_layer(case, s["weight"]))
    if case["op"] == "product":
        return dict(logits=_exact_product(s))
    B, K, V = case["B"], case["K"], case["V"]
    out = torch.zeros((B, K, V), dtype=torch.float64, device="cuda")
    norms = torch.zeros((B, K), dtype=torch.float64, device="cuda")
    column = torch.arange(V, device="cuda")
    for b in range(B):
        rep, freq, pres = s["penalties"][b].double()
        all_tokens, answer = s["tokens"][b].long(), s["tokens"][b, s["prompt_len"][b]:].long()
        seen = torch.bincount(all_tokens[all_tokens >= 0], minlength=V)
        count = torch.bincount(answer[answer >= 0], minlength=V)
        for i in range(K if s["row_len"] is None else int(s["row_len"][b])):
            y = s["logits"][b, i, :V].double()
            y = torch.where(seen > 0, torch.where(y > 0, y / rep, y * rep), y) - freq * count - pres * (count > 0).double()
            if s["bias"] is not None:
                y = y + (s["bias"] if s["bias"].dim() == 1 else s["bias"][b]).double()
            if s["allowed"] is not None:
                words = (s["allowed"][b] if s["allowed"].dim() == 2 else s["allowed"][b, i]).long()
                y = y.masked_fill((words[column // 32] >> (column % 32)) & 1 == 0, NEG_INF)
            out[b, i] = y
            if case["norm"]:  # of the row as it is stored
                z = y.to(s["logits"].dtype).double() / (case["temperature"] or 1.0)
                norms[b, i] = torch.logsumexp(z, 0) / math.log(2.0)
            if s["drafts"] is not None:
                seen[s["drafts"][b, i]] += 1
                count[s["drafts"][b, i]] += 1
    return dict(logits=out, log2_norm=norms) if case["norm"] else dict(logits=out)
