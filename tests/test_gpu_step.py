"""Generation steps with the operators run together as a program runs them: projections rotated into the
caches, attention over the tree of hypotheses, logits adjusted, hypotheses selected and forked.  Every
output is checked against 64-bit definitions on the data that the step before left."""
import math

import numpy as np
import pytest
import torch

from gpu_common import load_lib

pytestmark = pytest.mark.gpu

HALF_STEP = torch.finfo(torch.bfloat16).eps / 2    # 2^-8: bf16 has 8 significant bits


def turned(x, pos, freq):
    """Halves, in 64 bits."""
    n = len(freq)
    a = torch.outer(torch.as_tensor(pos, dtype=torch.float64, device="cuda"), torch.tensor(freq, dtype=torch.float64, device="cuda"))
    c, s = a.cos()[:, None], a.sin()[:, None]
    x = x.double()
    return torch.cat([x[..., :n] * c - x[..., n:2 * n] * s, x[..., :n] * s + x[..., n:2 * n] * c, x[..., 2 * n:]], -1)


@pytest.mark.parametrize("fp8", [False, True])
def test_generation_with_several_hypotheses(fp8):
    mx, _ = load_lib()
    groups, beams, vocab, prompt_len, steps, window = 2, 3, 3001, 450, 6, 128
    hq, hkv, d = 8, 2, 128
    # a standard layer, one that reuses its cache, a sliding-window layer, one that reuses that
    layout = [(mx.FULL, 0, 0), (mx.FULL, 0, 0), (mx.SLIDING, window, 2), (mx.SLIDING, window, 2)]
    n = groups * beams
    ctx = mx.Context(layout, hq, hkv, d, mx.BF16, n, 400, max_seq_len=600, device=0, kv_format=mx.KV_FP8_E4M3 if fp8 else mx.KV_NATIVE)
    ctx.set_prefix_sharing(True)
    ctx.set_share_min_bytes(0)
    gen = torch.Generator("cuda").manual_seed(11)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").bfloat16()

    freq = [10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
    rope = mx.Rope(d, 10000.0, halves=True)
    firsts = [g * beams for g in range(groups)]
    lens = [prompt_len, prompt_len - 37]
    tokens = torch.full((n, 700), -1, device="cuda", dtype=torch.int32)
    for g, f in enumerate(firsts):
        tokens[f, :lens[g]] = torch.randint(0, vocab, (lens[g],), generator=gen, device="cuda").int()
    counts = [lens[i // beams] for i in range(n)]
    prompts = list(counts)
    for owner in (0, 2):
        rows = normal(sum(lens), (hq + 2 * hkv) * d).view(-1, hq + 2 * hkv, d)
        ctx.rope_qkv(owner, firsts, lens, rope, k=rows[:, hq:hq + hkv], v=rows[:, hq + hkv:], store=True)
    scores = torch.full((groups, beams), float("-inf"), device="cuda")
    scores[:, 0] = 0.0
    for g, f in enumerate(firsts):
        ctx.fork_seqs([f] * (beams - 1), list(range(f + 1, f + beams)))
        tokens[f + 1:f + beams] = tokens[f]
    ids = list(range(n))
    assert ctx.get_distinct_tokens(1, ids) < 2 * prompt_len + 40
    bias_tokens = torch.tensor([[5, 9, -1]] * n, device="cuda", dtype=torch.int32)
    bias_values = torch.tensor([[2.5, -3.0, 7.0]] * n, device="cuda")
    allowed = torch.full((1, (vocab + 31) // 32), -1, device="cuda", dtype=torch.int32)
    allowed[0, :40] = 0x0f0f0f0f
    allowed_rows = torch.tensor([0] * beams + [-1] * beams, device="cuda", dtype=torch.int32)
    penalty = dict(repetition=torch.full((n,), 1.2, device="cuda"), frequency=torch.full((n,), 0.3, device="cuda"),
                   presence=torch.full((n,), 0.1, device="cuda"), temperature=torch.full((n,), 0.8, device="cuda"))
    for step in range(steps):
        at = [ctx.get_len(0, s) for s in ids]
        for layer in range(4):
            rows = normal(n, (hq + 2 * hkv) * d).view(n, hq + 2 * hkv, d)
            if layer in (0, 2):
                q = ctx.rope_qkv(layer, ids, None, rope, q=rows[:, :hq], k=rows[:, hq:hq + hkv], v=rows[:, hq + hkv:], store=True)[0]
            else:      # the owner has stored the token already
                q = ctx.rope_qkv(layer, ids, None, rope, q=rows[:, :hq], first_pos=at)[0]
            want_q = turned(rows[:, :hq], at, freq)
            assert ((q.double() - want_q).abs() <= HALF_STEP * want_q.abs() * 1.01 + 2.0 ** -20 * 10).all()
            out = torch.full((n, hq, d), float("nan"), device="cuda", dtype=torch.bfloat16)
            ctx.decode(layer, ids, q, out)
            stored = ctx.get_stored(layer, ids)
            K, V = ctx.read_kv(layer, ids)
            row = 0
            for i, m in enumerate(stored):
                assert m == (at[i] + 1 if layer < 2 else min(at[i] + 1, window))
                k, v = K[row:row + m].double(), V[row:row + m].double()
                row += m
                z = torch.einsum("gcd,ngd->gcn", q[i].double().view(hkv, -1, d), k) / math.sqrt(d)
                p = torch.softmax(z, -1)
                want = torch.einsum("gcn,ngd->gcd", p, v).reshape(hq, d)
                A = torch.einsum("gcn,ngd->gcd", p, v.abs()).reshape(hq, d)
                # half a step of the output, weights to 11 bits or more, scores of magnitude 40 at most (test_gpu_shared.py)
                bound = HALF_STEP * want.abs() * 1.01 + (2.0 ** -11 + 2.0 ** -24 * 40 * 48 * 1.4 + 2.0 ** -16) * A + m * 2.0 ** -25 * 448 * fp8 + 1e-30
                assert ((out[i].double() - want).abs() <= bound).all(), (step, layer, i)
        logits = normal(n, vocab).float() * 3
        adjusted = torch.empty_like(logits)
        n_tokens = torch.tensor(counts, device="cuda", dtype=torch.int32)
        ctx.adjust_logits(logits, adjusted, tokens=tokens, n_tokens=n_tokens, n_prompt=torch.tensor(prompts, device="cuda", dtype=torch.int32),
                          bias_tokens=bias_tokens, bias_values=bias_values, allowed=allowed, allowed_rows=allowed_rows, **penalty)
        x = logits.double()
        for i in range(n):
            mine = tokens[i, :counts[i]].long()
            made, times = mine[prompts[i]:].unique(return_counts=True)
            seen = mine.unique()
            x[i, seen] = torch.where(x[i, seen] > 0, x[i, seen] / 1.2, x[i, seen] * 1.2)
            x[i, made] -= 0.3 * times.double() + 0.1
            x[i, 5] += 2.5
            x[i, 9] -= 3.0
        x /= 0.8
        t = torch.arange(vocab, device="cuda")
        x[:beams, (t < 40 * 32) & (t % 8 >= 4)] = float("-inf")
        same = torch.isinf(x)
        assert torch.equal(torch.isinf(adjusted), same)
        # (parameters given as 0.3, 1.2, ... are fp32 numbers: 2^-24 more of each step)
        assert ((adjusted.double() - x)[~same].abs() <= 2.0 ** -24 * 16 * (x[~same].abs() + 40)).all()
        was = scores
        scores, parents, picked = ctx.beam_select(adjusted.view(groups, beams, vocab), scores, beams)
        ll = torch.log_softmax(adjusted.double().view(groups, beams, vocab), -1) + was.double()[..., None]
        best = ll.view(groups, -1).sort(dim=-1, descending=True, stable=True)
        gap = best.values[:, :beams + 1].diff(dim=-1).abs()
        assert ((gap == 0) | (gap > 1e-5)).all()    # (the choice is not a matter of rounding; equal logits go by their index)
        assert torch.equal(parents.long() * vocab + picked.long(), best.indices[:, :beams])
        src = [g * beams + b for g, row in enumerate(parents.tolist()) for b in row]
        ctx.fork_seqs(src, ids)
        tokens = tokens[src].contiguous()
        tokens[torch.arange(n, device="cuda"), n_tokens.long()[src]] = picked.view(-1)
        counts = [counts[s] + 1 for s in src]
        assert bool((allowed_rows[src] == allowed_rows).all())
    assert ctx.get_device_status() == 0
    ctx.close()


def test_two_contexts_on_two_streams():
    """Calls that overlap on the GPU, each context on its own stream and workspace."""
    mx, _ = load_lib()
    jobs = []
    for seed in (1, 2):
        gen = torch.Generator("cuda").manual_seed(seed)
        ctx = mx.Context([(mx.FULL, 0, 0)], 16, 4, 128, mx.BF16, 17, 900, max_seq_len=6000, device=0)
        kv = [torch.randn(5000, 4, 128, generator=gen, device="cuda").bfloat16() for _ in range(2)]
        ctx.set_share_min_bytes(0)
        ctx.append_kv(0, [16], [5000], *kv)
        ctx.fork_seqs([16] * 16, list(range(16)))
        for s in range(16):
            ctx.append_kv(0, [s], [1 + s], kv[0][:1 + s], kv[1][:1 + s])
        q = torch.randn(16, 16, 128, generator=gen, device="cuda").bfloat16()
        want = torch.empty_like(q)
        ctx.decode_shared(0, list(range(16)), q, want)
        jobs.append((ctx, q, want, [torch.empty_like(q) for _ in range(30)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(30):
        for ctx, q, want, outs, stream in jobs:
            ctx.decode_shared(0, list(range(16)), q, outs[i], stream=stream)
    torch.cuda.synchronize()
    for ctx, q, want, outs, stream in jobs:
        assert all(torch.equal(o, want) for o in outs) and ctx.get_device_status() == 0


def test_captured_step():
    """Rotation of queries, attention and adjustment replayed from one graph."""
    mx, _ = load_lib()
    gen = torch.Generator("cuda").manual_seed(3)
    ctx = mx.Context([(mx.FULL, 0, 0), (mx.FULL, 0, 0)], 8, 2, 64, mx.BF16, 5, 200, max_seq_len=1000, device=0)
    kv = [torch.randn(600, 2, 64, generator=gen, device="cuda").bfloat16() for _ in range(2)]
    ctx.set_share_min_bytes(0)
    ctx.append_kv(0, [4], [600], *kv)
    ctx.fork_seqs([4] * 4, [0, 1, 2, 3])
    for s in range(4):
        ctx.append_kv(0, [s], [s + 1], kv[0][:s + 1], kv[1][:s + 1])
    rows = torch.randn(4, 8, 64, generator=gen, device="cuda").bfloat16()
    q, out = torch.empty_like(rows), torch.empty_like(rows)
    logits = torch.randn(4, 999, generator=gen, device="cuda")
    y = torch.empty_like(logits)
    temperature = torch.full((4,), 0.5, device="cuda")
    rope = mx.Rope(64)
    pos = [ctx.get_len(0, s) - 1 for s in range(4)]

    def step(stream):
        ctx.rope_qkv(1, [0, 1, 2, 3], None, rope, q=rows, first_pos=pos, out=(q, None, None), stream=stream)
        ctx.decode_shared(1, [0, 1, 2, 3], q, out, stream=stream)
        ctx.adjust_logits(logits, y, temperature=temperature, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for _ in range(3):
        rows.copy_(torch.randn(4, 8, 64, generator=gen, device="cuda"))
        logits.copy_(torch.randn(4, 999, generator=gen, device="cuda"))
        step(torch.cuda.current_stream())
        torch.cuda.synchronize()
        eager = (q.clone(), out.clone(), y.clone())
        for t in (q, out, y):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (q, out, y)))
    assert ctx.get_device_status() == 0


def test_profile_classes():
    """The new kernels are counted under their classes."""
    mx, _ = load_lib()
    ctx = mx.Context([(mx.FULL, 0, 0)], 8, 2, 128, mx.BF16, 3, 100, max_seq_len=500, device=0)
    ctx.profile_enable(True)
    ctx.set_share_min_bytes(0)
    rows = torch.randn(300, 12, 128, device="cuda").bfloat16()
    ctx.rope_qkv(0, [0], [300], mx.Rope(128), k=rows[:, 8:10], v=rows[:, 10:], store=True)
    ctx.fork_seqs([0, 0], [1, 2])
    q = rows[:3, :8].contiguous()
    ctx.decode_shared(0, [0, 1, 2], q, torch.empty_like(q))
    ctx.adjust_logits(torch.zeros(2, 100, device="cuda"), temperature=torch.ones(2, device="cuda"))
    for cls in (mx.K_SHARED, mx.K_MERGE, mx.K_ROPE, mx.K_ADJUST):
        assert ctx.profile_read(cls)[0] == 1
