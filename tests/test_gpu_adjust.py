"""Penalties, biases, temperature and masks on logits on a B200 against the formula in 64 bits.

Bound: the fp32 steps are x / r or x * r, f * c, + p, the difference, + bias and the division (or, for bf16
outputs, the reciprocal and its product): seven roundings of at most half a step of the largest value on
the way, 7 * 2^-24 (|a| + f c + p + |bias|) / T, then half a step of the output's type."""
import random

import pytest
import torch

from gpu_common import load_lib

pytestmark = pytest.mark.gpu

NEG = float("-inf")


def context():
    mx, _ = load_lib()
    return mx, mx.Context([(mx.FULL, 0, 0)], 4, 2, 64, mx.BF16, 1, 1, device=0)


def expect(logits, tokens=None, n_tokens=None, n_prompt=None, repetition=None, frequency=None, presence=None, temperature=None,
           bias_tokens=None, bias_values=None, allowed=None, allowed_rows=None):
    """(y, sum of the magnitudes on the way) in 64 bits, row by row."""
    x = logits.double().cpu()
    rows, vocab = x.shape
    size = x.abs().clone()

    def par(t, i, default):
        return default if t is None else float(t[i])

    for i in range(rows):
        n = 0
        if tokens is not None:
            n = tokens.shape[1] if n_tokens is None else min(max(int(n_tokens[i]), 0), tokens.shape[1])
        prompt = 0 if n_prompt is None else min(max(int(n_prompt[i]), 0), n)
        r, f, p, T = par(repetition, i, 1.0), par(frequency, i, 0.0), par(presence, i, 0.0), par(temperature, i, 1.0)
        ids = tokens[i, :n].cpu().long() if n else torch.zeros(0, dtype=torch.long)
        ok = (ids >= 0) & (ids < vocab)
        seen = ids[ok].unique()
        made, times = ids[prompt:][ok[prompt:]].unique(return_counts=True)
        x[i, seen] = torch.where(x[i, seen] > 0, x[i, seen] / r, x[i, seen] * r)
        size[i, seen] = x[i, seen].abs()
        x[i, made] -= f * times.double() + p
        size[i, made] += abs(f) * times.double() + abs(p)
        if bias_tokens is not None:
            last = {}
            for t, b in zip(bias_tokens[i].tolist(), bias_values[i].tolist()):
                if 0 <= t < vocab:
                    last[t] = b
            for t, b in last.items():
                x[i, t] += b
                size[i, t] += abs(b)
        x[i] /= T
        size[i] /= T
        if allowed is not None:
            which = i if allowed_rows is None else int(allowed_rows[i])
            if 0 <= which < allowed.shape[0]:
                words = allowed[which].cpu().long() & 0xffffffff
                t = torch.arange(vocab)
                x[i, (words[t // 32] >> (t % 32)) & 1 == 0] = NEG
    return x.cuda(), size.cuda()


def compare(got, logits, **rules):
    want, size = expect(logits, **rules)
    torch.cuda.synchronize()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    odd = torch.isinf(want) | torch.isnan(want)
    assert torch.equal(got.double()[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)])
    bound = torch.finfo(got.dtype).eps / 2 * want.abs() * 1.001 + 7 * 2.0 ** -24 * size + 1e-38
    err = (got.double() - want).abs()
    err[odd] = 0
    assert (err[~odd] <= bound[~odd]).all(), float((err - bound)[~odd].max())


def rules_of(rows, vocab, n, seed, masks=None, n_bias=0, part=range(8)):
    gen = torch.Generator("cuda").manual_seed(seed)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    r = {}
    if 0 in part:
        r["tokens"] = (uniform(rows, n) ** 3 * vocab * 1.01).int() - 1      # a few outside the vocabulary
        r["n_tokens"] = (uniform(rows) * (n + 1)).int()
        r["n_prompt"] = (uniform(rows) * (n + 1)).int()
    if 1 in part:
        r["repetition"] = 0.8 + uniform(rows)
    if 2 in part:
        r["frequency"] = uniform(rows) - 0.2
    if 3 in part:
        r["presence"] = uniform(rows) - 0.2
    if 4 in part:
        r["temperature"] = 0.3 + uniform(rows)
    if 5 in part and n_bias:
        r["bias_tokens"] = (uniform(rows, n_bias) * vocab * 1.02).int() - 1   # some twice, some outside
        r["bias_values"] = (uniform(rows, n_bias) - 0.5) * 20
    if 6 in part and masks:
        words = torch.randint(-2**31, 2**31, (masks, (vocab + 31) // 32 + seed % 3), generator=gen, device="cuda").int()
        words[0] = 0                                                            # a row that allows nothing
        if masks > 1:
            words[1] = -1
        r["allowed"] = words
        if masks != rows:
            r["allowed_rows"] = (uniform(rows) * (masks + 2)).int() - 1
    return r


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32)]


@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (2, 31), (2, 33), (5, 1000), (3, 2049), (33, 4099), (2, 50021), (7, 32000), (1, 131072), (2, 200003),
                                        (300, 513)])
def test_all_rules(rows, vocab, ti, to):
    mx, ctx = context()
    gen = torch.Generator("cuda").manual_seed(vocab)
    logits = (torch.randn(rows, vocab, generator=gen, device="cuda") * 4).to(ti)
    r = rules_of(rows, vocab, 777, vocab, masks=max(1, rows - 1), n_bias=17)
    out = torch.full((rows, vocab), 123.0, device="cuda", dtype=to)
    ctx.adjust_logits(logits, out, **r)
    compare(out, logits, **r)
    if ti == to:
        here = logits.clone()
        ctx.adjust_logits(here, **r)
        assert torch.equal(here.view(torch.uint8), out.view(torch.uint8))


@pytest.mark.parametrize("part", [(), (0, 1), (0, 2), (0, 3), (4,), (5,), (6,), (0, 1, 2, 3), (5, 6), (0, 1, 4), (0,)])
@pytest.mark.parametrize("in_place", [False, True])
def test_some_rules(part, in_place):
    mx, ctx = context()
    rows, vocab = 4, 5003
    gen = torch.Generator("cuda").manual_seed(8)
    logits = (torch.randn(rows, vocab, generator=gen, device="cuda") * 4).bfloat16()
    r = rules_of(rows, vocab, 300, 9, masks=4, n_bias=33, part=part)
    was = logits.clone()
    out = logits if in_place else torch.full_like(logits, 123.0)
    ctx.adjust_logits(logits, None if in_place else out, **r)
    compare(out, was, **r)


@pytest.mark.parametrize("shift_in,shift_out", [(0, 0), (1, 1), (3, 3), (1, 0), (0, 5), (7, 2)])
@pytest.mark.parametrize("ti,to", TYPES)
def test_any_alignment_and_neighbours_untouched(ti, to, shift_in, shift_out):
    mx, ctx = context()
    rows, vocab = 3, 3001
    gen = torch.Generator("cuda").manual_seed(8)
    big_in = (torch.randn(rows, vocab + 21, generator=gen, device="cuda") * 4).to(ti)
    big_out = torch.full((rows, vocab + 10), 55.0, device="cuda", dtype=to)
    logits, out = big_in[:, shift_in:shift_in + vocab], big_out[:, shift_out:shift_out + vocab]
    r = rules_of(rows, vocab, 300, 4, masks=3, n_bias=5)
    ctx.adjust_logits(logits, out, **r)
    compare(out, logits, **r)
    assert bool((big_out[:, :shift_out] == 55).all()) and bool((big_out[:, shift_out + vocab:] == 55).all())


def test_lists_of_any_length():
    mx, ctx = context()
    rows, vocab = 6, 900
    gen = torch.Generator("cuda").manual_seed(3)
    logits = torch.randn(rows, vocab, generator=gen, device="cuda")
    for n in (0, 1, 255, 256, 257, 70001):
        tokens = torch.randint(-5, vocab + 5, (rows, n), generator=gen, device="cuda").int()
        r = {"tokens": tokens, "n_tokens": torch.tensor([n, 0, -3, n + 10, n // 2, 1], device="cuda", dtype=torch.int32),
             "n_prompt": torch.tensor([0, 4, 5, n, 2 * n, -1], device="cuda", dtype=torch.int32),
             "repetition": torch.full((rows,), 1.3, device="cuda"), "frequency": torch.full((rows,), 0.01, device="cuda"),
             "presence": torch.full((rows,), 0.5, device="cuda")}
        out = torch.empty_like(logits)
        ctx.adjust_logits(logits, out, **r)
        compare(out, logits, **r)
        del r["n_tokens"], r["n_prompt"]
        ctx.adjust_logits(logits, out, **r)
        compare(out, logits, **r)
    # one token over and over: the largest count a row can have
    tokens = torch.full((1, mx.MAX_RULE_TOKENS), 5, device="cuda", dtype=torch.int32)
    r = {"tokens": tokens, "frequency": torch.ones(1, device="cuda")}
    out = torch.empty(1, vocab, device="cuda")
    ctx.adjust_logits(logits[:1], out, **r)
    compare(out, logits[:1], **r)


@pytest.mark.parametrize("ti", [torch.bfloat16, torch.float32])
def test_infinite_and_nan_logits(ti):
    mx, ctx = context()
    vocab = 3000
    gen = torch.Generator("cuda").manual_seed(3)
    logits = torch.randn(2, vocab, generator=gen, device="cuda").to(ti)
    lowest = torch.finfo(ti).min
    for i, x in enumerate((NEG, float("inf"), float("nan"), lowest, -lowest, 0.0, -0.0)):
        logits[:, i::17] = x
    r = {"tokens": torch.arange(0, vocab, 2, device="cuda").int().repeat(2, 1), "repetition": torch.tensor([1.5, 1.0], device="cuda"),
         "frequency": torch.tensor([0.5, 0.0], device="cuda"), "presence": torch.tensor([0.5, 0.0], device="cuda")}
    mask = torch.randint(-2**31, 2**31, (1, 94), generator=gen, device="cuda").int()
    out = torch.empty_like(logits)
    ctx.adjust_logits(logits, out, **r, allowed=mask, allowed_rows=torch.tensor([0, -1], device="cuda", dtype=torch.int32))
    want, _ = expect(logits, **r, allowed=mask, allowed_rows=[0, -1])
    limit = torch.finfo(ti).max
    want = torch.where(want.abs() > limit * (1 + torch.finfo(ti).eps / 2), torch.sign(want) * float("inf"), want)   # (overflows)
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(torch.isinf(out), torch.isinf(want))
    assert torch.equal(out[torch.isinf(want)] > 0, want[torch.isinf(want)] > 0)


def test_the_last_bias_counts():
    mx, ctx = context()
    logits = torch.zeros(2, 100, device="cuda")
    out = torch.empty_like(logits)
    n = mx.MAX_RULE_BIASES
    ctx.adjust_logits(logits, out, bias_tokens=torch.full((2, n), 7, device="cuda", dtype=torch.int32),
                      bias_values=torch.arange(2 * n, device="cuda").float().view(2, n))
    assert out[:, 7].tolist() == [n - 1.0, 2 * n - 1.0] and int((out != 0).sum()) == 2


def test_then_selected():
    """Adjusted logits go to beam_select as they are."""
    mx, ctx = context()
    g, b, v = 3, 4, 5000
    gen = torch.Generator("cuda").manual_seed(3)
    logits = torch.randn(g * b, v, generator=gen, device="cuda").bfloat16()
    r = rules_of(g * b, v, 300, 6, masks=5, n_bias=5)
    out = torch.empty(g * b, v, device="cuda")
    ctx.adjust_logits(logits, out, **r)
    scores, beams, tokens = ctx.beam_select(out.view(g, b, v), torch.zeros(g, b, device="cuda"), 8)
    x = out.double().view(g, b, v)
    ll = (x - torch.logsumexp(x, -1, keepdim=True)).nan_to_num(nan=NEG, neginf=NEG)   # (a beam that may say nothing)
    best = ll.view(g, -1).sort(dim=-1, descending=True, stable=True)
    gap = best.values[:, :8].diff().abs().min()
    assert float(gap) > 1e-6      # the order is decided beyond the scores' error of 2^-20
    assert torch.equal(beams.long() * v + tokens.long(), best.indices[:, :8])


def test_captured_and_replayed_with_other_data():
    mx, ctx = context()
    rows, vocab = 5, 9001
    logits = torch.randn(rows, vocab, device="cuda").bfloat16()
    r = rules_of(rows, vocab, 300, 6, masks=5, n_bias=5)
    out = torch.empty_like(logits)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.adjust_logits(logits, out, **r, stream=side)
    for seed in (7, 8):
        logits.copy_(torch.randn(rows, vocab, device="cuda"))
        for name, t in rules_of(rows, vocab, 300, seed, masks=5, n_bias=5).items():
            if t.shape == r[name].shape:
                r[name].copy_(t)
        graph.replay()
        compare(out, logits, **r)


def test_refusals():
    mx, ctx = context()
    x = torch.zeros(4, 100, device="cuda")
    f = torch.ones(4, device="cuda")
    i = torch.zeros(4, device="cuda", dtype=torch.int32)
    t = torch.zeros(4, 10, device="cuda", dtype=torch.int32)
    m = torch.zeros(4, 4, device="cuda", dtype=torch.int32)
    bad = [dict(tokens=t.long()), dict(tokens=t[:3]), dict(tokens=t.cpu()), dict(tokens=t.t().contiguous().t()), dict(n_tokens=i), dict(n_prompt=i),
           dict(tokens=t, n_tokens=i[:3]), dict(tokens=t, n_prompt=i.long()), dict(repetition=f.double()), dict(frequency=f[:3]),
           dict(presence=f.cpu()), dict(temperature=torch.ones(8, device="cuda")[::2]), dict(bias_tokens=t), dict(bias_values=f.view(4, 1)),
           dict(bias_tokens=t, bias_values=torch.ones(4, 9, device="cuda")), dict(allowed=m[:, :3]), dict(allowed=m[:3]), dict(allowed_rows=i),
           dict(allowed=m, allowed_rows=i[:2]), dict(allowed=m.long()),
           dict(bias_tokens=torch.zeros(4, 2048, device="cuda", dtype=torch.int32), bias_values=torch.zeros(4, 2048, device="cuda")),
           dict(tokens=torch.zeros(4, 1 << 20, device="cuda", dtype=torch.int32))]
    out = torch.full_like(x, 3.0)
    for rules in bad:
        assert ctx.rc_adjust_logits(x, out, **rules) == mx.ERR_INVALID_ARG, list(rules)
    for a, o in ((x.half(), out), (x, out.half()), (x.view(-1), out.view(-1)), (x, out[:3]), (x.cpu(), out), (x, out.cpu()), (x.t(), out.t())):
        assert ctx.rc_adjust_logits(a, o) == mx.ERR_INVALID_ARG
    assert ctx.rc_adjust_logits(x, out.bfloat16()) == mx.ERR_UNSUPPORTED
    assert bool((out == 3).all())
    assert ctx.rc_adjust_logits(x[:0], out[:0]) == 0


def test_random_calls():
    """Sizes, types and rules at random."""
    mx, ctx = context()
    for seed in range(40):
        rng = random.Random(seed)
        rows, vocab = rng.choice([1, 2, 9, 40, 170]), rng.choice([3, 100, 1023, 4096, 8191, 30011])
        ti, to = rng.choice(TYPES)
        gen = torch.Generator("cuda").manual_seed(seed)
        logits = (torch.randn(rows, vocab, generator=gen, device="cuda") * 4).to(ti)
        r = rules_of(rows, vocab, rng.choice([1, 10, 3000]), seed, masks=rng.choice([0, 1, rows]), n_bias=rng.choice([0, 1, 300]),
                     part=[i for i in range(7) if rng.random() < 0.7])
        out = torch.full((rows, vocab), 123.0, device="cuda", dtype=to)
        ctx.adjust_logits(logits, out, **r)
        compare(out, logits, **r)
