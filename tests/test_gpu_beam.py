"""Beam selection on a B200 against the definition in 64 bits.  Choices have to be equal; scores
are off by the rounding to fp32 (2^-24 of the value) and by the sum's error: its fp32 terms carry
about 2^-22 each of the exponential and of the exponent's rounding, 2^-21 in all, in a sum of
positive terms, so the logarithm is off by at most 2^-20."""
import numpy as np
import pytest
import torch

from gpu_common import load_lib

pytestmark = pytest.mark.gpu


def context(mx):
    return mx.Context([(mx.FULL, 0, 0)], 2, 1, 64, mx.BF16, 1, 1, device=0)   # the smallest workspace


def reference(logits, scores, n_out, finished=None, eos=0):
    g, b, v = logits.shape
    x = logits.double().cpu().numpy()
    start = scores.double().cpu().numpy()
    done = None if finished is None else finished.cpu().numpy()
    S, B, T = np.full((g, n_out), -np.inf), np.full((g, n_out), -1), np.full((g, n_out), -1)
    for i in range(g):
        found = []
        for j in range(b):
            if not np.isfinite(start[i, j]):
                continue
            if done is not None and done[i, j]:
                found.append((-start[i, j], j * v + eos))
                continue
            ok = np.flatnonzero(np.isfinite(x[i, j]))
            if not len(ok):
                continue
            r = x[i, j, ok]
            s = r - (r.max() + np.log(np.exp(r - r.max()).sum())) + start[i, j]
            first = np.lexsort((ok, -r))[:n_out]
            found += [(-s[t], j * v + ok[t]) for t in first]
        found.sort()
        for r, (s, f) in enumerate(found[:n_out]):
            S[i, r], B[i, r], T[i, r] = -s, f // v, f % v
    return S, B, T


def check(ctx, logits, scores, n_out, finished=None, eos=0):
    s, b, t = ctx.beam_select(logits, scores, n_out, finished=finished, eos_token=eos)
    torch.cuda.synchronize()
    S, B, T = reference(logits, scores, n_out, finished, eos)
    s, b, t = s.double().cpu().numpy(), b.cpu().numpy(), t.cpu().numpy()
    assert (b == B).all() and (t == T).all(), np.argwhere((b != B) | (t != T))[:4]
    none = B < 0
    assert (s[none] == -np.inf).all()
    err = np.abs(s[~none] - S[~none])
    assert (err <= 2.0 ** -24 * np.abs(S[~none]) + 2.0 ** -20).all(), err.max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups,beams,vocab,n_out", [
    (1, 1, 1, 1), (1, 1, 3, 5), (2, 3, 7, 8), (1, 4, 255, 8), (3, 2, 256, 64), (2, 5, 1000, 10), (1, 4, 32000, 8),
    (5, 8, 8191, 16), (3, 4, 50021, 8), (2, 64, 3001, 64), (40, 4, 2049, 8), (1, 1, 200003, 64), (600, 3, 130, 4)])
def test_selection(dtype, groups, beams, vocab, n_out):
    mx, _ = load_lib()
    ctx = context(mx)
    gen = torch.Generator("cuda").manual_seed(vocab)
    logits = (3 * torch.randn(groups, beams, vocab, generator=gen, device="cuda")).to(dtype)
    scores = -20 * torch.rand(groups, beams, generator=gen, device="cuda")
    check(ctx, logits, scores, n_out)
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_orders_and_empty_rows(dtype):
    mx, _ = load_lib()
    ctx = context(mx)
    v = 9001
    up = torch.arange(v, device="cuda", dtype=torch.float32) / 512
    rows = [torch.zeros(v, device="cuda"), up, up.flip(0), torch.full((v,), -1e4, device="cuda"),
            torch.where(torch.arange(v, device="cuda") % 2 == 0, 0.0, -0.0)]
    logits = torch.stack(rows).to(dtype)[None]
    for n_out in (1, 7, 64):
        check(ctx, logits, torch.tensor([[-1.0, -1.0, -2.0, -0.5, -1.0]], device="cuda"), n_out)
    # two equal beams: the lower one first
    check(ctx, logits[:, :1].expand(1, 3, v).contiguous(), torch.zeros(1, 3, device="cuda"), 9)
    # banned tokens, NaN, infinities, a row without any continuation, beams that are out
    x = logits[:, :3].clone()
    x[0, 0, 5:] = float("-inf")
    x[0, 1, ::3] = float("nan")
    x[0, 1, 1::3] = float("inf")
    x[0, 2] = float("-inf")
    for scores in ([-1.0, -9.0, 0.0], [float("-inf"), -9.0, 0.0], [float("nan"), float("inf"), -1.0]):
        check(ctx, x, torch.tensor([scores], device="cuda"), 12)
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_finished_beams(dtype):
    mx, _ = load_lib()
    ctx = context(mx)
    gen = torch.Generator("cuda").manual_seed(9)
    logits = torch.randn(6, 4, 5003, generator=gen, device="cuda").to(dtype)
    finished = (torch.rand(6, 4, generator=gen, device="cuda") < 0.5).to(torch.uint8)
    finished[0] = 1
    logits[finished.bool()] = float("nan")      # not read
    scores = -3 * torch.rand(6, 4, generator=gen, device="cuda")
    scores[1, 2] = float("-inf")
    check(ctx, logits, scores, 8, finished, eos=5002)
    check(ctx, logits, scores, 3, finished, eos=0)
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,stride", [(1, 1003), (3, 1010), (7, 2001), (0, 1000)])
def test_strided_unaligned_rows(dtype, offset, stride):
    mx, _ = load_lib()
    ctx = context(mx)
    gen = torch.Generator("cuda").manual_seed(11)
    flat = torch.randn(6 * stride + offset, generator=gen, device="cuda").to(dtype)
    flat[:offset] = 1e4                          # what lies between the rows does not count
    logits = flat[offset:].as_strided((2, 3, 1000), (3 * stride, stride, 1))
    for r in range(6):
        flat[offset + r * stride + 1000: offset + (r + 1) * stride] = 1e4
    check(ctx, logits, -torch.rand(2, 3, generator=gen, device="cuda"), 6)
    ctx.close()


def test_wide_values():
    mx, _ = load_lib()
    ctx = context(mx)
    gen = torch.Generator("cuda").manual_seed(12)
    logits = torch.randn(2, 3, 4000, generator=gen, device="cuda") * 1e30
    logits[1] = torch.randn(3, 4000, generator=gen, device="cuda") * 1e-3 - 500
    s, b, t = ctx.beam_select(logits, torch.zeros(2, 3, device="cuda"), 5)
    S, B, T = reference(logits, torch.zeros(2, 3), 5)
    assert (b.cpu().numpy() == B).all() and (t.cpu().numpy() == T).all()
    assert np.abs(s[1].double().cpu().numpy() - S[1]).max() <= 2.0 ** -24 * 600 + 2.0 ** -20
    ctx.close()


def test_refusals_of_the_binding():
    mx, _ = load_lib()
    ctx = context(mx)
    x, s = torch.zeros(2, 3, 100, device="cuda"), torch.zeros(2, 3, device="cuda")
    for bad in (dict(logits=x.half()), dict(logits=x.transpose(1, 2)), dict(scores=s.double()), dict(scores=s[:1]),
                dict(finished=s), dict(logits=x.transpose(0, 1)), dict(logits=x.cpu()), dict(scores=s.cpu()),
                dict(finished=torch.zeros(2, 3, dtype=torch.uint8)), dict(n_out=65), dict(n_out=0)):
        with pytest.raises(mx.MixAttnError):
            ctx.beam_select(**{"logits": x, "scores": s, "n_out": 4, **bad})
    ctx.close()


def test_captured_and_on_another_stream():
    mx, _ = load_lib()
    ctx = context(mx)
    gen = torch.Generator("cuda").manual_seed(13)
    logits = torch.randn(3, 4, 20011, generator=gen, device="cuda").bfloat16()
    scores = -torch.rand(3, 4, generator=gen, device="cuda")
    outs = (torch.empty(3, 8, device="cuda"), torch.empty(3, 8, dtype=torch.int32, device="cuda"),
            torch.empty(3, 8, dtype=torch.int32, device="cuda"))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        assert ctx.rc_beam_select(logits, scores, 8, *outs, stream=torch.cuda.current_stream()) == 0
    logits.copy_(torch.randn(3, 4, 20011, generator=gen, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    S, B, T = reference(logits, scores, 8)
    assert (outs[1].cpu().numpy() == B).all() and (outs[2].cpu().numpy() == T).all()
    first = [o.clone() for o in outs]
    for _ in range(20):                       # the same bits every time
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
    ctx.close()
