"""Beam selection on a B200 where the launch takes other ways: several launches for one call, chunks
made longer to fit the workspace, more lists than a block has threads, logits masked with the
type's lowest value."""
import numpy as np
import pytest
import torch

from gpu_common import load_lib
from test_gpu_beam_sums import check as check_values

pytestmark = pytest.mark.gpu


def reference(logits, scores, n_out, finished, eos):
    g, b, v = logits.shape
    x, start = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    done = np.zeros((g, b)) if finished is None else finished.cpu().numpy()
    S, B, T = np.full((g, n_out), -np.inf), np.full((g, n_out), -1), np.full((g, n_out), -1)
    for i in range(g):
        found = []
        for j in range(b):
            ok = np.flatnonzero(np.isfinite(x[i, j]))
            if done[i, j]:
                found.append((-start[i, j], j * v + eos))
            elif len(ok):
                r = x[i, j, ok]
                r = r - r.max()          # (first, or 1e38 would swallow the logarithm)
                s = r - np.log(np.exp(r).sum()) + start[i, j]
                first = np.lexsort((ok, -x[i, j, ok]))[:n_out]
                found += [(-s[t], j * v + ok[t]) for t in first]
        found.sort()
        for k, (s, f) in enumerate(found[:n_out]):
            S[i, k], B[i, k], T[i, k] = -s, f // v, f % v
    return S, B, T


def check(ctx, logits, scores, n_out, finished=None, eos=0):
    s, b, t = (x.cpu().numpy() for x in ctx.beam_select(logits, scores, n_out, finished=finished, eos_token=eos))
    S, B, T = reference(logits, scores, n_out, finished, eos)
    assert (b == B).all() and (t == T).all(), np.argwhere((b != B) | (t != T))[:4]
    none = B < 0
    assert (s[none] == -np.inf).all()
    err = np.abs(s[~none] - S[~none])
    assert (err <= 2.0 ** -24 * np.abs(S[~none]) + 2.0 ** -20).all(), err.max()


def context(mx):
    return mx.Context([(mx.FULL, 0, 0)], 1, 1, 64, mx.BF16, 1, 1, device=0)   # the smallest workspace: one query head


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups,beams,vocab,n_out", [
    (1100, 1, 300, 3), (2100, 2, 130, 64),     # more groups than one launch has counters for
    (40, 64, 2500, 64),                        # batches by the workspace
    (1, 64, 40000, 64), (2, 64, 70003, 63), (1, 8, 128256, 8), (1, 4, 151936, 16), (1, 8, 50257, 64), (1, 16, 18000, 32), (1, 1, 400003, 64)])   # many lists
def test_other_ways_through_the_launch(dtype, groups, beams, vocab, n_out):
    mx, _ = load_lib()
    ctx = context(mx)
    gen = torch.Generator("cuda").manual_seed(vocab + groups)
    logits = (3 * torch.randn(groups, beams, vocab, generator=gen, device="cuda")).to(dtype)
    scores = -20 * torch.rand(groups, beams, generator=gen, device="cuda")
    finished = (torch.rand(groups, beams, generator=gen, device="cuda") < 0.2).to(torch.uint8)
    for _ in range(2):       # (the second call finds counters and workspace as the first one left them)
        check(ctx, logits, scores, n_out, finished, eos=5)
    check(ctx, logits, scores, n_out)
    assert ctx.get_device_status() == 0
    ctx.close()


@pytest.mark.parametrize("dtype,groups,beams,vocab", [(torch.float32, 2, 54, 1326344), (torch.bfloat16, 2, 60, 1861771)])
def test_chunks_made_longer_to_fit_the_workspace(dtype, groups, beams, vocab):
    # (14 and 16 chunks per row would be best, of which the lists of one group do not fit)
    mx, _ = load_lib()
    ctx = context(mx)
    gen = torch.Generator("cuda").manual_seed(84)
    logits = torch.randn(groups, beams, vocab, generator=gen, device="cuda", dtype=dtype) * 3
    scores = -torch.rand(groups, beams, generator=gen, device="cuda")
    check_values(ctx, logits, scores, 64)
    check_values(ctx, logits, scores, 64)
    assert ctx.get_device_status() == 0
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_lists_with_ties_and_orders(dtype):
    mx, _ = load_lib()
    ctx = context(mx)
    v = 130000
    up = torch.arange(v, device="cuda", dtype=torch.float32) / 8192
    rows = [up, up.flip(0), torch.zeros(v, device="cuda"), up * 0 - 1e4, up, up.flip(0), -up, up % 1]
    logits = torch.stack(rows).to(dtype)[None]
    for n_out in (1, 16, 64):
        check(ctx, logits, torch.tensor([[-1.0, -1.0, 9.0, 9.0, -1.0, -1.0, -2.0, 3.0]], device="cuda"), n_out)
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,allowed", [(1000, 3), (50021, 3), (50021, 0), (50021, 40000)])
def test_tokens_masked_with_the_lowest_value(dtype, vocab, allowed):
    # finite, so they are continuations, behind all others; a row of nothing else is uniform
    mx, _ = load_lib()
    ctx = context(mx)
    gen = torch.Generator("cuda").manual_seed(82)
    logits = torch.randn(2, 3, vocab, generator=gen, device="cuda").to(dtype)
    low = torch.finfo(dtype).min
    for row in logits.view(6, vocab)[:5]:
        row[torch.randperm(vocab, generator=gen, device="cuda")[allowed:]] = low
    logits[1, 1, 17] = float("-inf")
    check(ctx, logits, -torch.rand(2, 3, generator=gen, device="cuda"), 8)
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_whole_finite_range(dtype):
    mx, _ = load_lib()
    ctx = context(mx)
    f = torch.finfo(dtype)
    gen = torch.Generator("cuda").manual_seed(83)
    logits = torch.randn(1, 4, 30001, generator=gen, device="cuda").to(dtype)
    logits[0, 0, 20000] = f.max
    logits[0, 1, ::2] = f.min
    logits[0, 2] = f.min
    logits[0, 2, 3:6] = f.max
    logits[0, 3, 9] = float("inf")
    logits[0, 3, 10] = f.max
    logits[0, 3, 11] = float("nan")
    check(ctx, logits, torch.tensor([[-1.0, -2.0, -3.0, -4.0]], device="cuda"), 16)
    ctx.close()
