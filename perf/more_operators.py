"""Cases of further operators of a generation step: attention of sequences that share cached
prefixes, the rotary embedding of a projection's rows on their way into a cache, and penalties,
biases and grammar masks on logits.

Shared prefixes.  A batch of sequences forms a tree: all begin with the same `prefix` tokens,
groups of them go on with the same `mid` tokens, each ends in tokens of its own.  Per sequence, with
the query at its last position i and s = q . k / sqrt(head_dim):
    a = cap * tanh(s / cap) if cap > 0 else s          b = a - slope_h * (i - j)
    out = sum_j softmax_j(b) v_j        over all of its keys j <= i

Rotary embedding.  Channel pairs (x, y) of a head at position t turn by the angle t * f_p, f_p the
pair's frequency: x' = x cos - y sin, y' = x sin + y cos.  Pairs are (2p, 2p + 1), or (p, p + n/2)
of the n rotated channels; channels from n on stay as they are.  Queries and keys are rotated,
values are not; keys and values are stored, or handed back as plain tensors.

Logits.  Per row, with c the times a token was generated and seen whether it occurs at all:
    a = seen ? (x > 0 ? x / repetition : x * repetition) : x
    b = a - frequency * c - (c > 0 ? presence : 0)
    y = (b + bias) / temperature        tokens that the row's mask forbids: -inf
"""
import math
import random

import torch

own = False

NEG = float("-inf")
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.bfloat16}   # fp8: the cache's storage


# ---------------------------------------------------------------- cases
def _shared(name, groups, each, prefix, mid, own_lo, own_hi, heads, dtype, cap, bias):
    return {"name": name, "kind": "shared", "groups": groups, "each": each, "prefix": prefix, "mid": mid,
            "own_lo": own_lo, "own_hi": own_hi, "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2],
            "dtype": dtype, "cap": cap, "bias": bias}


def _rope(name, mode, seqs, len_lo, len_hi, start, window, heads, dtype, rotary, halves, stretched):
    return {"name": name, "kind": "rope", "mode": mode, "seqs": seqs, "len_lo": len_lo, "len_hi": len_hi,
            "start": start, "window": window, "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2],
            "dtype": dtype, "rotary": rotary, "halves": halves, "stretched": stretched}


def _logits(name, rows, vocab, dtype, hist_lo, hist_hi, n_bias, masked):
    return {"name": name, "kind": "logits", "rows": rows, "vocab": vocab, "dtype": dtype, "hist_lo": hist_lo,
            "hist_hi": hist_hi, "n_bias": n_bias, "masked": masked}


MID = (32, 8, 128)    # query heads, KV heads, head_dim of the 24-layer configurations
TINY = (4, 2, 64)     # of the small parity configuration
PAPER = (12, 3, 128)  # of the paper's model


def listed():
    return [
        # four hypotheses of a short prompt on the fp32 parity configuration: latency only
        _shared("shared_tiny_f32", 1, 4, 200, 0, 1, 57, TINY, "f32", 30.0, True),
        # one prompt of 8k tokens answered eight times
        _shared("shared_answers", 1, 8, 8191, 0, 1, 300, MID, "bf16", 0.0, False),
        # 64 requests behind one long instruction, questions and answers of their own
        _shared("shared_instruction", 1, 64, 32768, 0, 16, 2048, MID, "bf16", 0.0, False),
        # eight requests behind one instruction, four hypotheses each, quantised cache, distance bias
        _shared("shared_tree_fp8", 8, 4, 6000, 1500, 1, 200, MID, "fp8", 0.0, True),
        # narrow heads with capped scores
        _shared("shared_narrow_capped", 1, 40, 20011, 0, 1, 1000, (16, 4, 64), "bf16", 50.0, False),
        # one step of 64 sequences on a layer that reuses another one's cache: queries only
        _rope("rope_queries", "queries", 64, 1, 1, 31000, 0, MID, "bf16", 128, True, False),
        # short prompts of the fp32 configuration, half of the channels rotated, stored
        _rope("rope_ragged_f32", "store", 3, 1, 200, 0, 0, TINY, "f32", 32, False, False),
        # a chunk of two prompts into sliding-window caches, frequencies stretched for long contexts
        _rope("rope_window", "store", 2, 2048, 2048, 0, 1024, MID, "bf16", 128, True, True),
        # a long chunk's rows rotated into plain tensors, as attention over a chunk takes them
        _rope("rope_chunk", "plain", 1, 8192, 8192, 120000, 0, MID, "bf16", 128, False, False),
        # one request's answer so far: latency
        _logits("logits_one", 1, 32000, "bf16", 700, 700, 0, False),
        # a batch with an odd vocabulary in fp32, biases
        _logits("logits_odd_f32", 128, 50021, "f32", 1, 4000, 40, False),
        # a large batch over a large vocabulary, half of the rows under a grammar: 268 MB
        _logits("logits_large", 512, 131072, "bf16", 100, 9000, 8, True),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["shared", "shared", "shared", "rope", "rope", "logits", "logits"])
    heads = rng.choice([MID, MID, PAPER, TINY, (16, 4, 64), (16, 16, 128), (8, 1, 128), (20, 2, 64)])
    if kind == "shared":
        dtype = rng.choice(["bf16", "bf16", "fp8", "f32"]) if heads[2] == 128 else rng.choice(["bf16", "bf16", "f32"])
        cap, bias = rng.choice([(0.0, False), (0.0, False), (50.0, False), (30.0, True), (0.0, True)])
        groups = rng.choice([1, 1, 2, 5, 8])
        each = _log_between(rng, 1 if groups > 1 else 2, 64 // groups)
        top = 1024 if dtype == "f32" else min(65536, (1 << 25) // (heads[1] * heads[2]))
        prefix = _log_between(rng, 16, top)
        mid = rng.choice([0, _log_between(rng, 1, max(2, top // 16))]) if groups > 1 else 0
        hi = _log_between(rng, 1, 200 if dtype == "f32" else 2048)
        return _shared("", groups, each, prefix, mid, rng.choice([1, hi]), hi, heads, dtype, cap, bias)
    if kind == "rope":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        mode = rng.choice(["queries", "store", "store", "plain"])
        seqs = _log_between(rng, 1, 64 if mode != "store" else 8)
        hi = _log_between(rng, 1, (8192 if dtype == "bf16" else 1000) // seqs)
        start = 0 if mode == "store" else _log_between(rng, 1, 200000)
        rotary = rng.choice([heads[2], heads[2], heads[2] // 2, 48])
        return _rope("", mode, seqs, rng.choice([1, hi]), hi, start, rng.choice([0, 0, 1000, 1024]), heads, dtype, rotary,
                     rng.random() < 0.5, rng.random() < 0.5)
    dtype = rng.choice(["bf16", "f32"])
    rows = _log_between(rng, 1, 512)
    vocab = _log_between(rng, 100, min(200000, (1 << 27) // (rows * (2 if dtype == "bf16" else 4))))
    hi = _log_between(rng, 1, 16000 if rows < 64 else 4000)
    return _logits("", rows, vocab, dtype, rng.choice([1, hi]), hi, rng.choice([0, 0, 3, 300]), rng.random() < 0.5)


def _spread(lo, hi, n):
    """n lengths spread evenly over the logarithm of lo .. hi, in a fixed mixed order."""
    lens = [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) if n > 1 else hi for i in range(n)]
    random.Random(n).shuffle(lens)
    return lens


def _slopes(case):
    """The usual geometric slopes: 2^-8/H, 2^-16/H, ..., 2^-8 over the H query heads."""
    n = case["q_heads"]
    return [2.0 ** (-8.0 * (h + 1) / n) for h in range(n)] if case["bias"] else None


def _frequencies(case):
    """The usual powers of a base; `stretched`: those that turn less than once in 8192 positions eight times slower,
    those that turn more than four times as they are, in between by interpolation."""
    n = case["rotary"]
    freq = [500000.0 ** (-2.0 * p / n) for p in range(n // 2)]
    if not case["stretched"]:
        return freq
    turns = [8192 * f / (2 * math.pi) for f in freq]
    keep = [min(1.0, max(0.0, (t - 1.0) / 3.0)) for t in turns]
    return [f * (k + (1 - k) / 8) for f, k in zip(freq, keep)]


# ---------------------------------------------------------------- inputs
def _on_e4m3(x):
    """The nearest values that 8-bit storage with a shared power-of-two exponent per head vector holds."""
    top = x.abs().amax(-1, keepdim=True).float()
    scale = torch.exp2(torch.floor(torch.log2(torch.clamp(top, min=1e-30))) - 8)
    return (torch.clamp(x.float() / scale, -448, 448).to(torch.float8_e4m3fn).float() * scale).to(x.dtype)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(int(seed) * 1000003 + 29)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    s = {"case": dict(case)}
    if case["kind"] == "logits":
        return _prepare_logits(s, case, normal, uniform)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "rope":
        s["host_lens"] = lens = _spread(case["len_lo"], case["len_hi"], case["seqs"])
        s["host_starts"] = [case["start"] + 17 * i if case["start"] else 0 for i in range(case["seqs"])]
        s["pos"] = torch.cat([torch.arange(b, b + n, device="cuda") for b, n in zip(s["host_starts"], lens)])
        s["freq"] = _frequencies(case)
        s["qkv"] = normal(sum(lens), (hq + 2 * hkv) * d)      # rows of one projection
        if own:
            from paper_2409_15012_b200 import binding as mx
            s["ctx"] = _context(case, case["seqs"], max(lens), case["window"])
            s["rope"] = mx.Rope(case["rotary"], inv_freq=s["freq"], halves=case["halves"])
            s["ids"] = list(range(case["seqs"]))
        return s
    # shared: sequence i belongs to group i % groups
    groups, n = case["groups"], case["groups"] * case["each"]
    s["host_own"] = lens = _spread(case["own_lo"], case["own_hi"], n)
    s["own_len"] = torch.tensor(lens, device="cuda")
    sharp = torch.linspace(1, 3, hq, device="cuda")[:, None]         # some heads look sharply, some broadly
    s["q"] = (normal(n, hq, d, dtype=torch.float32) * sharp).to(dt)
    put = _on_e4m3 if case["dtype"] == "fp8" else (lambda x: x)
    s["prefix"] = [put(normal(case["prefix"], hkv, d)) for _ in range(2)]
    s["mid"] = [put(normal(groups, case["mid"], hkv, d)) for _ in range(2)] if case["mid"] else None
    s["tail"] = [put(normal(n, max(lens), hkv, d)) for _ in range(2)]
    s["out"] = torch.empty_like(s["q"])
    if own:
        ctx = s["ctx"] = _context(case, n + groups, case["prefix"] + case["mid"] + max(lens), 0)
        roots = list(range(n, n + groups))
        ctx.append_kv(0, roots[:1], [case["prefix"]], *s["prefix"])
        ctx.fork_seqs([roots[0]] * groups, roots)
        if case["mid"]:
            ctx.append_kv(0, roots, [case["mid"]] * groups, *s["mid"])
        ctx.fork_seqs([roots[i % groups] for i in range(n)], list(range(n)))
        for i, m in enumerate(lens):
            ctx.append_kv(0, [i], [m], s["tail"][0][i, :m], s["tail"][1][i, :m])
        s["ids"] = list(range(n))
    return s


def _prepare_logits(s, case, normal, uniform):
    rows, vocab = case["rows"], case["vocab"]
    s["logits"] = normal(rows, vocab) * 3
    lens = _spread(case["hist_lo"], case["hist_hi"], rows)
    # what has been read and written so far; small ids are common words
    s["tokens"] = (uniform(rows, max(lens)) ** 3 * vocab).int().clamp_(max=vocab - 1)
    s["n_tokens"] = torch.tensor(lens, device="cuda", dtype=torch.int32)
    s["n_prompt"] = torch.tensor([n // 2 for n in lens], device="cuda", dtype=torch.int32)
    s["repetition"] = 1 + 0.3 * uniform(rows)
    s["frequency"] = 0.5 * uniform(rows)
    s["presence"] = uniform(rows)
    s["temperature"] = 0.5 + uniform(rows)
    s["bias_tokens"] = s["bias_values"] = s["allowed"] = s["allowed_rows"] = None
    if case["n_bias"]:
        n = min(case["n_bias"], vocab)
        first = (uniform(rows, 1) * vocab).int()
        s["bias_tokens"] = ((first + torch.arange(n, device="cuda") * max(1, vocab // n)) % vocab).int()   # distinct
        s["bias_values"] = normal(rows, n, dtype=torch.float32) * 4
    if case["masked"]:
        # every other row follows a grammar, which allows from a handful of tokens to most of them
        n = (rows + 1) // 2
        share = uniform(n, 1) ** 4
        bits = (uniform(n, (vocab + 31) // 32 * 32) < share).view(n, -1, 32)
        words = (bits.long() << torch.arange(32, device="cuda")).sum(-1)
        s["allowed"] = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
        which = torch.full((rows,), -1, device="cuda", dtype=torch.int32)
        which[::2] = torch.arange(n, device="cuda", dtype=torch.int32).flip(0)
        s["allowed_rows"] = which
    if own:
        from paper_2409_15012_b200 import binding as mx
        s["ctx"] = mx.Context([(mx.FULL, 0, 0)], 4, 2, 64, mx.BF16, 1, 1, device=0)
        s["out"] = torch.empty_like(s["logits"])
    return s


def _context(case, seqs, longest, window):
    """The cache handle a program keeps: layer 0 owns a cache, layer 1 reads it."""
    from paper_2409_15012_b200 import binding as mx
    layer = (mx.SLIDING, window) if window else (mx.FULL, 0)
    pages = seqs * (-(-longest // 16) + 1)
    ctx = mx.Context([(*layer, 0), (*layer, 0)], case["q_heads"], case["kv_heads"], case["dim"],
                     mx.F32 if case["dtype"] == "f32" else mx.BF16, seqs, pages, max_seq_len=longest + 16, device=0,
                     kv_format=mx.KV_FP8_E4M3 if case["dtype"] == "fp8" else mx.KV_NATIVE)
    if case["kind"] == "shared" and (case["cap"] or case["bias"]):
        for l in (0, 1):
            ctx.set_layer_scores(l, case["cap"], _slopes(case))
    return ctx


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"shared": _plain_shared, "rope": _plain_rope, "logits": _plain_logits}[case["kind"]](s, case)


def _heads(s, case):
    """The projection's rows as queries, keys and values: views, tokens (q_heads + 2 kv_heads) * dim apart."""
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    rows = s["qkv"].view(-1, hq + 2 * hkv, d)
    return rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]


def _run_own(s, case):
    ctx, stream = s["ctx"], torch.cuda.current_stream()
    if case["kind"] == "shared":
        ctx.decode_shared(1, s["ids"], s["q"], s["out"], stream=stream)
        return s["out"]
    if case["kind"] == "logits":
        ctx.adjust_logits(s["logits"], s["out"], tokens=s["tokens"], n_tokens=s["n_tokens"], n_prompt=s["n_prompt"],
                          repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                          temperature=s["temperature"], bias_tokens=s["bias_tokens"], bias_values=s["bias_values"],
                          allowed=s["allowed"], allowed_rows=s["allowed_rows"], stream=stream)
        return s["out"]
    q, k, v = _heads(s, case)
    if case["mode"] == "queries":
        return ctx.rope_qkv(1, s["ids"], s["host_lens"], s["rope"], q=q, first_pos=s["host_starts"], stream=stream)[0]
    if case["mode"] == "plain":
        return ctx.rope_qkv(0, s["ids"], s["host_lens"], s["rope"], q=q, k=k, v=v, first_pos=s["host_starts"], stream=stream)
    for i in s["ids"]:          # the slots' earlier sequences have ended
        ctx.seq_reset(i)
    q_out = ctx.rope_qkv(0, s["ids"], s["host_lens"], s["rope"], q=q, k=k, v=v, store=True, stream=stream)[0]
    return q_out, *ctx.read_kv(0, s["ids"], stream=stream)


def _plain_shared(s, case):
    groups, each, hkv, d = case["groups"], case["each"], case["kv_heads"], case["dim"]
    n, p, m = groups * each, case["prefix"], case["mid"]
    q = s["q"].float().view(n, hkv, -1, d).permute(1, 2, 0, 3)                     # [hkv, group, n, d]
    g = q.shape[1]
    flat = q.reshape(hkv, g * n, d)

    def by_group(x):            # [hkv, g, n, ...] -> [hkv, groups, g * each, ...]
        return x.view(hkv, g, each, groups, -1).permute(0, 3, 1, 2, 4).reshape(hkv, groups, g * each, -1)

    def from_group(x):
        return x.view(hkv, groups, g, each, -1).permute(0, 2, 3, 1, 4).reshape(hkv, g, n, -1)

    parts = [(flat @ s["prefix"][0].float().permute(1, 2, 0)).view(hkv, g, n, p)]
    if m:
        parts.append(from_group(by_group(q) @ s["mid"][0].float().permute(2, 0, 3, 1)))
    tail_k, tail_v = (x.float().permute(2, 0, 1, 3) for x in s["tail"])            # [hkv, n, t, d]
    parts.append((q.permute(0, 2, 1, 3) @ tail_k.transpose(-1, -2)).permute(0, 2, 1, 3))
    scores = torch.cat(parts, -1).mul_(1 / math.sqrt(d))
    distance = (p + m + s["own_len"] - 1)[:, None] - torch.arange(scores.shape[-1], device="cuda")
    if case["cap"]:
        scores.div_(case["cap"]).tanh_().mul_(case["cap"])
    if case["bias"]:
        slopes = torch.tensor(_slopes(case), device="cuda").view(hkv, g, 1, 1)
        scores.addcmul_(slopes, distance.float(), value=-1)
    scores.masked_fill_(distance < 0, NEG)
    w = scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    out = (w[..., :p].reshape(hkv, g * n, p) @ s["prefix"][1].float().transpose(0, 1)).view(hkv, g, n, d)
    if m:
        out += from_group(by_group(w[..., p:p + m]) @ s["mid"][1].float().permute(2, 0, 1, 3))
    out += (w[..., p + m:].permute(0, 2, 1, 3) @ tail_v).permute(0, 2, 1, 3)
    out /= w.sum(-1, keepdim=True)
    return out.permute(2, 0, 1, 3).reshape(n, case["q_heads"], d).to(s["q"].dtype)


def _turn(x, cos, sin, case):
    """x [tokens, heads, dim] in fp32, its rotated channels turned."""
    n = case["rotary"]
    out = x.clone()
    a, b = (slice(0, n // 2), slice(n // 2, n)) if case["halves"] else (slice(0, n, 2), slice(1, n, 2))
    out[..., a] = x[..., a] * cos - x[..., b] * sin
    out[..., b] = x[..., a] * sin + x[..., b] * cos
    return out


def _plain_rope(s, case):
    q, k, v = _heads(s, case)
    angle = s["pos"].double()[:, None, None] * torch.tensor(s["freq"], device="cuda", dtype=torch.float64)
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _turn(q.float(), cos, sin, case).to(q.dtype)
    if case["mode"] == "queries":
        return q
    k = _turn(k.float(), cos, sin, case).to(q.dtype)
    if case["mode"] == "plain":
        return q, k, v.contiguous()
    return q, _kept(k, s, case), _kept(v, s, case)


def _kept(x, s, case):
    """The rows a cache holds in the end: all of them, or the last `window` of each sequence."""
    if not case["window"]:
        return x.contiguous()
    return torch.cat([part[-case["window"]:] for part in x.split(s["host_lens"])])


def _plain_logits(s, case):
    rows, vocab = case["rows"], case["vocab"]
    x = s["logits"].float()
    at = torch.arange(s["tokens"].shape[1], device="cuda")[None]
    valid = at < s["n_tokens"][:, None]
    made = valid & (at >= s["n_prompt"][:, None])
    index = s["tokens"].long()
    seen = torch.zeros(rows, vocab, device="cuda").scatter_add_(1, index, valid.float()) > 0
    count = torch.zeros(rows, vocab, device="cuda").scatter_add_(1, index, made.float())
    r = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if s["bias_tokens"] is not None:
        x.scatter_add_(1, s["bias_tokens"].long(), s["bias_values"])
    x /= s["temperature"][:, None]
    if s["allowed"] is not None:
        bits = (s["allowed"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        bits = bits.view(bits.shape[0], -1)[:, :vocab].bool()
        which = s["allowed_rows"]
        x.masked_fill_(~bits[which.clamp(min=0).long()] & (which >= 0)[:, None], NEG)
    return x.to(s["logits"].dtype)


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"shared": _exact_shared, "rope": _exact_rope, "logits": _exact_logits}[case["kind"]](s, case)


def _exact_shared(s, case):
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    slopes = _slopes(case)
    for i, m in enumerate(s["host_own"]):
        k, v = (torch.cat([s["prefix"][j]] + ([s["mid"][j][i % case["groups"]]] if case["mid"] else []) +
                          [s["tail"][j][i, :m]]).double() for j in (0, 1))
        back = torch.arange(len(k) - 1, -1, -1, device="cuda", dtype=torch.float64)
        for g in range(hkv):
            mine = slice(g * (hq // hkv), (g + 1) * (hq // hkv))
            z = torch.einsum("hd,nd->hn", s["q"][i, mine].double(), k[:, g]) * d ** -0.5
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if slopes:
                z = z - torch.tensor(slopes[mine], device="cuda", dtype=torch.float64)[:, None] * back
            out[i, mine] = torch.softmax(z, dim=1) @ v[:, g]
    return out


def _exact_rope(s, case):
    n, d = case["rotary"], case["dim"]
    cis = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                      torch.outer(s["pos"].double(), torch.tensor(s["freq"], device="cuda", dtype=torch.float64)))
    outs = []
    for x in _heads(s, case)[:2]:
        x = x.double()
        turned, rest = x[..., :n], x[..., n:]
        pairs = turned.unflatten(-1, (2, n // 2)).transpose(-1, -2) if case["halves"] else turned.unflatten(-1, (n // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * cis[:, None])
        z = z.transpose(-1, -2) if case["halves"] else z
        outs.append(torch.cat([z.flatten(-2), rest], -1))
    if case["mode"] == "queries":
        return outs[0]
    outs.append(_heads(s, case)[2].double())
    if case["mode"] == "plain" or not case["window"]:
        return tuple(outs)
    first = [0]
    for length in s["host_lens"]:
        first.append(first[-1] + length)
    keep = [t for a, b in zip(first, first[1:]) for t in range(max(a, b - case["window"]), b)]
    keep = torch.tensor(keep, device="cuda")
    return outs[0], outs[1][keep], outs[2][keep]


def _exact_logits(s, case):
    out = s["logits"].double()
    lens, prompts = s["n_tokens"].tolist(), s["n_prompt"].tolist()
    par = {k: s[k].double() for k in ("repetition", "frequency", "presence", "temperature")}
    for i in range(case["rows"]):
        x, ids = out[i], s["tokens"][i, :lens[i]].long()
        seen = ids.unique()
        x[seen] = torch.where(x[seen] > 0, x[seen] / par["repetition"][i], x[seen] * par["repetition"][i])
        made, times = ids[prompts[i]:].unique(return_counts=True)
        x[made] -= par["frequency"][i] * times.double() + par["presence"][i]
        if s["bias_tokens"] is not None:
            x[s["bias_tokens"][i].long()] += s["bias_values"][i].double()
        x /= par["temperature"][i]
        if s["allowed"] is not None and int(s["allowed_rows"][i]) >= 0:
            words = s["allowed"][int(s["allowed_rows"][i])].long() & 0xffffffff
            token = torch.arange(case["vocab"], device="cuda")
            x[(words[token // 32] >> (token % 32)) % 2 == 0] = NEG
    return out


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "logits":
        rows, vocab = case["rows"], case["vocab"]
        lens = _spread(case["hist_lo"], case["hist_hi"], rows)
        mask = (rows + 1) // 2 * ((vocab + 31) // 32) * 4 + 4 * rows if case["masked"] else 0
        return {"bytes": 2 * rows * vocab * size + 4 * sum(lens) + 8 * rows * case["n_bias"] + mask + 24 * rows,
                "flops": 4 * rows * vocab}
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "rope":
        lens = _spread(case["len_lo"], case["len_hi"], case["seqs"])
        tokens, vector = sum(lens), d * size
        turned = hq + (0 if case["mode"] == "queries" else hkv)
        moved = 2 * tokens * hq
        if case["mode"] == "plain":
            moved += 4 * tokens * hkv
        elif case["mode"] == "store":       # read where kept, stored, read back and handed over
            moved += 8 * hkv * sum(min(n, case["window"] or n) for n in lens)
        return {"bytes": moved * vector, "flops": 3 * tokens * turned * case["rotary"]}
    n = case["groups"] * case["each"]
    lens = _spread(case["own_lo"], case["own_hi"], n)
    held = case["prefix"] + case["groups"] * case["mid"] + sum(lens)
    seen = n * (case["prefix"] + case["mid"]) + sum(lens)
    token = 2 * hkv * (d + 1) if case["dtype"] == "fp8" else 2 * hkv * d * size
    return {"bytes": held * token + 2 * n * hq * d * size, "flops": 4 * seen * hq * d}
