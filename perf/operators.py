"""Cases of the operators of one generation step with several hypotheses: attention whose scores
are capped or biased by distance (one query per sequence, prompts, chunks behind a cache), the
selection over beams and vocabulary, and the forking of cached sequences.

Attention, per query at position i and key at position j (j <= i, and i - j < window on a
sliding-window layer), with s = q . k / sqrt(head_dim):
    a = cap * tanh(s / cap) if cap > 0 else s          b = a - slope_h * (i - j)
    out = sum_j softmax_j(b) v_j

Selection, per group of beams with a score each and a row of logits each:
    candidate (beam, token) = score_beam + logit - log(sum exp(logits of the beam))
and the best `n_out` of the group in descending order, ties to the lowest beam * vocab + token.
Only finite logits and scores count.  A finished beam has one candidate: its end token, at the
beam's own score.  Places without a candidate hold score -inf, beam -1 and token -1.

Forking: every listed copy of a sequence ends up with the sequence's cached keys and values,
read back as plain tensors (a sliding-window cache holds the last `window` tokens).
"""
import math
import random

import torch

own = False

NEG = float("-inf")
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.bfloat16}   # fp8: the cache's storage


# ---------------------------------------------------------------- cases
def _decode(name, batch, ctx_lo, ctx_hi, window, heads, dtype, cap, bias):
    return {"name": name, "kind": "decode", "batch": batch, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "window": window,
            "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "dtype": dtype, "cap": cap, "bias": bias}


def _prompt(name, batch, prefix, len_lo, len_hi, window, heads, dtype, cap, bias):
    return {"name": name, "kind": "prompt", "batch": batch, "prefix": prefix, "len_lo": len_lo, "len_hi": len_hi,
            "window": window, "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "dtype": dtype, "cap": cap,
            "bias": bias}


def _select(name, groups, beams, vocab, n_out, dtype, finished, banned):
    return {"name": name, "kind": "select", "groups": groups, "beams": beams, "vocab": vocab, "n_out": n_out,
            "dtype": dtype, "finished": finished, "banned": banned}


def _fork(name, seqs, copies, tokens, window, heads, dtype):
    return {"name": name, "kind": "fork", "seqs": seqs, "copies": copies, "tokens": tokens, "window": window,
            "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "dtype": dtype}


MID = (32, 8, 128)    # query heads, KV heads, head_dim of the 24-layer configurations
TINY = (4, 2, 64)     # of the small parity configuration
PAPER = (12, 3, 128)  # of the paper's model


def listed():
    return [
        # one step of two short sequences on the fp32 parity configuration: latency only
        _decode("decode_tiny_f32", 2, 200, 257, 64, TINY, "f32", 30.0, True),
        # a standard layer of the mid configuration: 32 sequences of 32k tokens, capped scores
        _decode("decode_full_32k", 32, 32768, 32768, 0, MID, "bf16", 50.0, False),
        # a sliding-window layer of the same step, rings at arbitrary offsets, cap and bias
        _decode("decode_window", 32, 1100, 5000, 1024, MID, "bf16", 50.0, True),
        # a mixed serving batch on a quantised cache, distance bias, lengths from 1 to 64k
        _decode("decode_ragged_fp8", 17, 1, 65536, 0, MID, "fp8", 0.0, True),
        # a whole prompt on a standard layer, capped scores
        _prompt("prompt_causal_8k", 1, 0, 8192, 8192, 0, MID, "bf16", 50.0, False),
        # short prompts of odd lengths packed into one call, sliding window, cap and bias
        _prompt("prompt_ragged_window", 5, 0, 1, 2500, 512, (16, 4, 64), "bf16", 30.0, True),
        # a chunk of two prompts behind what is cached, sliding-window layer, distance bias
        _prompt("chunk_window", 2, 6144, 2048, 2048, 1024, MID, "bf16", 0.0, True),
        # one request with four beams: latency
        _select("select_one", 1, 4, 32000, 8, "bf16", False, False),
        # a batch of requests with an odd vocabulary in fp32, some beams finished, tokens banned
        _select("select_odd_f32", 32, 4, 50021, 8, "f32", True, True),
        # a large batch over a large vocabulary: 134 MB of logits
        _select("select_large", 64, 8, 131072, 16, "bf16", False, False),
        # one short prompt continued four ways
        _fork("fork_one", 1, 4, 201, 64, TINY, "f32"),
        # eight prompts of 4k tokens continued four ways each
        _fork("fork_batch", 8, 4, 4103, 1024, MID, "bf16"),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "prompt", "prompt", "select", "select", "fork"])
    heads = rng.choice([MID, PAPER, TINY, (16, 4, 64), (16, 16, 128), (8, 1, 128), (20, 2, 64)])
    cap, bias = rng.choice([(50.0, False), (30.0, True), (0.0, True), (20.0, False)])
    if kind == "decode":
        dtype = rng.choice(["bf16", "bf16", "fp8", "f32"]) if heads[2] == 128 else rng.choice(["bf16", "bf16", "f32"])
        batch = _log_between(rng, 1, 64)
        top = 1024 if dtype == "f32" else max(2, min(131072, (1 << 30) // (batch * heads[1] * heads[2])))
        hi = _log_between(rng, 1, top)
        lo = rng.choice([1, hi, max(1, hi // 3)])
        window = rng.choice([0, 0, _log_between(rng, 1, 4096)])
        return _decode("", batch, lo, hi, window, heads, dtype, cap, bias)
    if kind == "prompt":
        window = rng.choice([0, 128 * rng.randint(1, 16), _log_between(rng, 1, 2048)])
        batch = rng.choice([1, 1, 2, 3, 5])
        if rng.random() < 0.25:      # the exact fp32 mode: short prompts
            hi = _log_between(rng, 1, 200)
            return _prompt("", batch, rng.choice([0, 100]), rng.choice([1, hi]), hi, window, TINY, "f32", cap, bias)
        hi = _log_between(rng, 1, 8192 // batch)
        prefix = rng.choice([0, _log_between(rng, 1, 4096)]) if hi * batch <= 4096 else 0
        return _prompt("", batch, prefix, rng.choice([1, hi, hi]), hi, window, heads, "bf16", cap, bias)
    if kind == "select":
        dtype = rng.choice(["bf16", "f32"])
        groups, beams = _log_between(rng, 1, 64), rng.choice([1, 2, 3, 4, 5, 8, 16])
        room = (1 << 27) // (groups * beams * (2 if dtype == "bf16" else 4))
        vocab = _log_between(rng, 100, min(131072, room))
        n_out = rng.choice([beams, 2 * beams, beams + 1])
        return _select("", groups, beams, vocab, n_out, dtype, rng.random() < 0.5, rng.random() < 0.5)
    seqs, copies = _log_between(rng, 1, 16), rng.choice([1, 2, 3, 4, 8])
    tokens = _log_between(rng, 1, min(8192, 131072 // (seqs * copies)))
    return _fork("", seqs, copies, tokens, rng.choice([64, 1000, 1024]), heads, rng.choice(["bf16", "f32"]))


def _lengths(case):
    """The lengths of a case's sequences: spread evenly over the logarithm of its range, in a fixed mixed order."""
    lo, hi = (case["ctx_lo"], case["ctx_hi"]) if case["kind"] == "decode" else (case["len_lo"], case["len_hi"])
    b = case["batch"]
    lens = [int(round(lo * (hi / lo) ** (i / max(1, b - 1)))) if b > 1 else hi for i in range(b)]
    random.Random(b).shuffle(lens)
    return lens


def _slopes(case):
    """The usual geometric slopes: 2^-8/H, 2^-16/H, ..., 2^-8 over the H query heads."""
    n = case["q_heads"]
    return [2.0 ** (-8.0 * (h + 1) / n) for h in range(n)] if case["bias"] else None


# ---------------------------------------------------------------- inputs
def _on_e4m3(x):
    """The nearest values that 8-bit storage with a shared power-of-two exponent per head vector holds."""
    top = x.abs().amax(-1, keepdim=True).float()
    exp = torch.floor(torch.log2(torch.clamp(top, min=1e-30))) - 8
    scale = torch.exp2(exp)
    q = torch.clamp(x.float() / scale, -448, 448).to(torch.float8_e4m3fn)
    return (q.float() * scale).to(x.dtype)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(int(seed) * 1000003 + 17)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    s = {"case": dict(case)}
    kind = case["kind"]
    if kind == "select":
        g, b, v = case["groups"], case["beams"], case["vocab"]
        dt = DTYPES[case["dtype"]]
        logits = normal(g, b, v, dtype=dt) * 3
        if case["banned"]:      # tokens that may not follow
            logits[torch.rand(g, b, v, generator=gen, device="cuda") < 0.01] = NEG
        s["logits"] = logits
        s["scores"] = -20 * torch.rand(g, b, generator=gen, device="cuda")
        s["finished"] = None
        if case["finished"]:
            s["finished"] = (torch.rand(g, b, generator=gen, device="cuda") < 0.2).to(torch.uint8)
        if own:
            from paper_2409_15012_b200 import binding as mx
            s["ctx"] = mx.Context([(mx.FULL, 0, 0)], 4, 2, 64, mx.BF16, 1, 1, device=0)
        return s

    dt = DTYPES[case["dtype"]]
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    # some heads look sharply, some broadly
    sharp = torch.linspace(1, 3, hq, device="cuda")[:, None]
    if kind == "decode":
        lens = _lengths(case)
        s["lens"] = torch.tensor(lens, device="cuda")
        s["q"] = (normal(case["batch"], hq, d, dtype=torch.float32) * sharp).to(dt)
        kv = [normal(case["batch"], max(lens), hkv, d, dtype=dt) for _ in range(2)]
        s["k"], s["v"] = (_on_e4m3(x) for x in kv) if case["dtype"] == "fp8" else kv
        s["out"] = torch.empty_like(s["q"])
        if own:
            s["ctx"] = _context(case, case["batch"], max(lens))
            for i, n in enumerate(lens):
                s["ctx"].append_kv(0, [i], [n], s["k"][i, :n], s["v"][i, :n])
            s["ids"] = list(range(case["batch"]))
        return s
    if kind == "prompt":
        lens, b, p = _lengths(case), case["batch"], case["prefix"]
        s["lens"] = torch.tensor(lens, device="cuda")
        s["q"] = (normal(sum(lens), hq, d, dtype=torch.float32) * sharp).to(dt)
        s["k"], s["v"] = normal(sum(lens), hkv, d, dtype=dt), normal(sum(lens), hkv, d, dtype=dt)
        s["k_cached"], s["v_cached"] = normal(b, p, hkv, d, dtype=dt), normal(b, p, hkv, d, dtype=dt)
        s["out"] = torch.empty_like(s["q"])
        if own:
            s["ctx"] = _context(case, b, p + max(lens), chunk=sum(lens) + b * p)
            s["ids"], s["host_lens"] = list(range(b)), lens
            if p:
                s["ctx"].append_kv(0, s["ids"], [p] * b, s["k_cached"], s["v_cached"])
        return s
    # fork
    n, copies = case["seqs"], case["copies"]
    s["full"] = [normal(n, case["tokens"], hkv, d, dtype=dt) for _ in range(2)]
    s["ring"] = [normal(n, case["tokens"], hkv, d, dtype=dt) for _ in range(2)]
    s["parents"] = torch.arange(n, device="cuda").repeat_interleave(copies)
    if own:
        s["ctx"] = _context(case, n * (1 + copies), case["tokens"])
        for layer, kv in ((0, s["full"]), (1, s["ring"])):
            s["ctx"].append_kv(layer, list(range(n)), [case["tokens"]] * n, kv[0], kv[1])
        s["src"] = [i // copies for i in range(n * copies)]
        s["dst"] = list(range(n, n * (1 + copies)))
    return s


def _context(case, seqs, longest, chunk=0):
    """The cache handle a program keeps: layer 0 owns a cache, layer 1 reads it (forking: layer 1 owns a ring)."""
    from paper_2409_15012_b200 import binding as mx
    window = case["window"]
    layer = (mx.SLIDING, window) if window else (mx.FULL, 0)
    layout = [(*layer, 0), (*layer, 0)]
    if case["kind"] == "fork":
        layout = [(mx.FULL, 0, 0), (mx.SLIDING, window, 1)]
    pages = seqs * (-(-longest // 16) + 1)
    ctx = mx.Context(layout, case["q_heads"], case["kv_heads"], case["dim"], mx.F32 if case["dtype"] == "f32" else mx.BF16,
                     seqs, pages, max_seq_len=longest + 16, device=0, chunk_scratch_tokens=chunk,
                     kv_format=mx.KV_FP8_E4M3 if case["dtype"] == "fp8" else mx.KV_NATIVE)
    if case["kind"] != "fork":
        for l in (0, 1):
            ctx.set_layer_scores(l, case["cap"], _slopes(case))
    return ctx


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["kind"] == "decode":
        return _plain_decode(s, case)
    if case["kind"] == "prompt":
        return _plain_prompt(s, case)
    if case["kind"] == "select":
        return _plain_select(s, case)
    return _plain_fork(s, case)


def _run_own(s, case):
    ctx, stream = s["ctx"], torch.cuda.current_stream()
    if case["kind"] == "decode":
        ctx.decode(1, s["ids"], s["q"], s["out"], stream=stream)
        return s["out"]
    if case["kind"] == "prompt":
        call = ctx.attend_chunk if case["prefix"] else ctx.prefill
        call(1, s["ids"], s["host_lens"], s["q"], s["k"], s["v"], s["out"], stream=stream)
        return s["out"]
    if case["kind"] == "select":
        return ctx.beam_select(s["logits"], s["scores"], case["n_out"], finished=s["finished"], eos_token=2, stream=stream)
    ctx.fork_seqs(s["src"], s["dst"], stream=stream)
    return [ctx.read_kv(l, s["dst"], stream=stream) for l in (0, 1)]


def _shape_scores(scores, distance, case):
    """Cap and distance bias, in place; scores [kv_heads, group, ...], distance broadcastable to the rest."""
    if case["cap"]:
        scores.div_(case["cap"]).tanh_().mul_(case["cap"])
    if case["bias"]:
        slopes = torch.tensor(_slopes(case), device=scores.device, dtype=scores.dtype)
        shape = (case["kv_heads"], -1) + (1,) * (scores.dim() - 2)
        scores.addcmul_(slopes.view(shape), distance.to(scores.dtype), value=-1)


def _plain_decode(s, case):
    b, hkv, d, n = case["batch"], case["kv_heads"], case["dim"], s["k"].shape[1]
    q = s["q"].float().view(b, hkv, -1, d).permute(1, 0, 2, 3)                  # [hkv, b, group, d]
    scores = q @ s["k"].float().permute(2, 0, 3, 1)                             # [hkv, b, group, n]
    scores = scores.permute(0, 2, 1, 3).mul_(1 / math.sqrt(d))                  # [hkv, group, b, n]
    distance = s["lens"][:, None] - 1 - torch.arange(n, device="cuda")[None]    # [b, n]
    _shape_scores(scores, distance, case)
    seen = distance >= 0
    if case["window"]:
        seen &= distance < case["window"]
    scores.masked_fill_(~seen, NEG)
    p = scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1)[..., None]
    out = p.permute(0, 2, 1, 3) @ s["v"].float().permute(2, 0, 1, 3)            # [hkv, b, group, d]
    out = out / total.permute(0, 2, 1, 3)
    return out.permute(1, 0, 2, 3).reshape(b, case["q_heads"], d).to(s["q"].dtype)


def _plain_prompt(s, case):
    b, hkv, d, p = case["batch"], case["kv_heads"], case["dim"], case["prefix"]
    t = s["q"].shape[0]
    lens = s["lens"]
    seq = torch.repeat_interleave(torch.arange(b, device="cuda"), lens, output_size=t)
    pos = p + torch.arange(t, device="cuda") - (lens.cumsum(0) - lens)[seq]
    k_seq = torch.cat([torch.arange(b, device="cuda").repeat_interleave(p), seq])
    k_pos = torch.cat([torch.arange(p, device="cuda").repeat(b), pos])
    k = torch.cat([s["k_cached"].reshape(-1, hkv, d), s["k"]]).float().permute(1, 2, 0)   # [hkv, d, keys]
    v = torch.cat([s["v_cached"].reshape(-1, hkv, d), s["v"]]).float().permute(1, 0, 2)   # [hkv, keys, d]
    q = s["q"].float().view(t, hkv, -1, d).permute(1, 2, 0, 3)                             # [hkv, group, t, d]
    group = q.shape[1]
    scores = (q.reshape(hkv, group * t, d) @ k).view(hkv, group, t, -1).mul_(1 / math.sqrt(d))
    distance = pos[:, None] - k_pos[None]
    _shape_scores(scores, distance, case)
    seen = (seq[:, None] == k_seq[None]) & (distance >= 0)
    if case["window"]:
        seen &= distance < case["window"]
    scores.masked_fill_(~seen, NEG)
    w = scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    out = (w.view(hkv, group * t, -1) @ v).view(hkv, group, t, d) / w.sum(-1, keepdim=True)
    return out.permute(2, 0, 1, 3).reshape(t, case["q_heads"], d).to(s["q"].dtype)


def _plain_select(s, case):
    g, b, v, n = case["groups"], case["beams"], case["vocab"], case["n_out"]
    # candidates of different beams may lie next to each other: 64 bits
    x = s["logits"].double()
    x = torch.where(torch.isfinite(x), x, NEG)
    top = x.amax(-1, keepdim=True)
    lse = (x - top).exp_().sum(-1, keepdim=True).log() + top
    beam = torch.where(torch.isfinite(s["scores"]), s["scores"], NEG).double()[..., None]
    score = x.sub_(lse).add_(beam)
    if s["finished"] is not None:
        done = s["finished"].bool()[..., None]
        end = torch.arange(v, device="cuda") == 2
        score = torch.where(done, torch.where(end, beam, NEG), score)
    score = torch.where(torch.isnan(score), NEG, score).view(g, b * v)
    # the n best: all above the n-th value, then those equal to it with the lowest index
    last = score.topk(n, dim=-1).values[:, -1:]
    where = torch.arange(b * v, device="cuda")[None]
    order = where + torch.where(score > last, 0, torch.where(score == last, b * v, 2 * b * v))
    index = order.topk(n, dim=-1, largest=False).values % (b * v)
    index = index.sort(dim=-1).values
    best, at = score.gather(-1, index).sort(dim=-1, descending=True, stable=True)
    index = index.gather(-1, at)
    none = best == NEG
    return best.float(), torch.where(none, -1, index // v).int(), torch.where(none, -1, index % v).int()


def _plain_fork(s, case):
    w = min(case["window"], case["tokens"])
    rows = (-1,) + tuple(s["full"][0].shape[2:])
    return [[x.index_select(0, s["parents"]).view(rows) for x in s["full"]],
            [x[:, case["tokens"] - w:].index_select(0, s["parents"]).view(rows) for x in s["ring"]]]


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    if case["kind"] == "fork":
        w = min(case["window"], case["tokens"])
        pick = [i for i in range(case["seqs"]) for _ in range(case["copies"])]
        return [[torch.cat([x[i] for i in pick]).double() for x in s["full"]],
                [torch.cat([x[i, -w:] for i in pick]).double() for x in s["ring"]]]
    if case["kind"] == "select":
        return _exact_select(s, case)
    slopes = _slopes(case)
    group, d = case["q_heads"] // case["kv_heads"], case["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lens = _lengths(case)
    row = 0
    for i, n in enumerate(lens):
        if case["kind"] == "decode":
            q, keys, values = s["q"][i:i + 1], s["k"][i, :n], s["v"][i, :n]
            at = torch.tensor([n - 1], device="cuda")
        else:
            q = s["q"][row:row + n]
            keys = torch.cat((s["k_cached"][i], s["k"][row:row + n]))
            values = torch.cat((s["v_cached"][i], s["v"][row:row + n]))
            at = torch.arange(n, device="cuda") + case["prefix"]
        back = at.unsqueeze(1) - torch.arange(len(keys), device="cuda")
        hidden = back < 0
        if case["window"]:
            hidden |= back >= case["window"]
        for h in range(case["q_heads"]):
            z = torch.einsum("td,nd->tn", q[:, h].double(), keys[:, h // group].double()) * d ** -0.5
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if slopes:
                z = z - slopes[h] * back.double()
            z[hidden] = NEG
            weights = torch.exp(z - torch.logsumexp(z, dim=1, keepdim=True))
            got = torch.einsum("tn,nd->td", weights, values[:, h // group].double())
            if case["kind"] == "decode":
                out[i, h] = got[0]
            else:
                out[row:row + n, h] = got
        row += n
    return out


def _exact_select(s, case):
    g, b, v, n = case["groups"], case["beams"], case["vocab"], case["n_out"]
    scores = torch.full((g, n), NEG, dtype=torch.float64, device="cuda")
    parents = torch.full((g, n), -1, dtype=torch.int32, device="cuda")
    tokens = torch.full((g, n), -1, dtype=torch.int32, device="cuda")
    for i in range(g):
        found = []
        for j in range(b):
            start = float(s["scores"][i, j])
            if s["finished"] is not None and int(s["finished"][i, j]):
                found.append((start, j * v + 2))
                continue
            ll = torch.log_softmax(s["logits"][i, j].double(), -1) + start
            value, index = ll.sort(dim=-1, descending=True, stable=True)
            found += [(a, j * v + c) for a, c in zip(value[:n].tolist(), index[:n].tolist()) if a > NEG]
        found.sort(key=lambda c: (-c[0], c[1]))
        for r, (a, c) in enumerate(found[:n]):
            scores[i, r], parents[i, r], tokens[i, r] = a, c // v, c % v
    return scores, parents, tokens


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "select":
        size = 4 if case["dtype"] == "f32" else 2
        rows = case["groups"] * case["beams"]
        return {"bytes": rows * (case["vocab"] * size + 4) + case["groups"] * case["n_out"] * 12, "flops": 3 * rows * case["vocab"]}
    size = 4 if case["dtype"] == "f32" else 2
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    if kind == "fork":
        kept = case["tokens"] + min(case["tokens"], case["window"])
        return {"bytes": 2 * kept * hkv * d * size * case["seqs"] * (1 + case["copies"]), "flops": 0}
    lens = _lengths(case)
    w = case["window"] or 1 << 40
    if kind == "decode":
        seen = sum(min(n, w) for n in lens)
        token = 2 * hkv * (d + 1) if case["dtype"] == "fp8" else 2 * hkv * d * size
        return {"bytes": seen * token + 2 * case["batch"] * hq * d * size, "flops": 4 * seen * hq * d}
    p = case["prefix"]
    pairs = sum(_band(p, n, w) for n in lens)
    cached = min(p, w - 1) * len(lens)
    return {"bytes": size * d * (2 * sum(lens) * (hq + hkv) + 2 * cached * hkv), "flops": 4 * pairs * hq * d}


def _band(p, n, w):
    """(query, key) pairs of n queries at positions p .. p + n - 1 that see the last w keys each."""
    grow = max(0, min(n, w - p))            # queries that still see every key
    return grow * p + grow * (grow + 1) // 2 + (n - grow) * min(w, p + n)
