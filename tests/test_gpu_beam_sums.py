"""Beam selection on a B200: the sums of exponentials where a late tile of the vocabulary holds
nearly all of them.  A score is off by the rounding to fp32 (2^-24 of the value) and by the sum:
next to a term's largest neighbour the exponent is small, so a term carries 2^-22 of the
exponential and, at the distances where terms still matter together (up to ln of a thread's share
of the vocabulary, 9), at most 2^-21 of the subtraction and the product; the terms of a thread's
tile add up to 2^-22 more, everything after that is compensated or in double precision.  In all
2^-20, of positive terms, so the logarithm is off by at most 2^-20."""
import pytest
import torch

from gpu_common import load_lib

pytestmark = pytest.mark.gpu


def check(ctx, logits, scores, n_out):
    """Scores of what came back against the definition in 64 bits, and against the best there are."""
    s, b, t = (x.double() if x.dtype == torch.float32 else x.long() for x in ctx.beam_select(logits, scores, n_out))
    g, beams, vocab = logits.shape
    x = logits.double()
    total = torch.log_softmax(x, -1) + scores.double()[..., None]
    best = total.view(g, -1).topk(n_out, dim=-1).values
    got = total.view(g, -1).gather(1, b * vocab + t)
    bound = 2.0 ** -24 * best.abs() + 2.0 ** -20
    assert (got - best).abs().max() == 0
    worst = ((s - best).abs() / bound).max().item()
    assert worst <= 1, worst
    assert (s <= scores.double().amax(1, keepdim=True) + bound).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups,beams,vocab", [(1, 4, 40009), (16, 8, 70001), (64, 8, 33000)])   # few and many tiles per CTA
@pytest.mark.parametrize("lead", [5.0, 20.0, 40.0, 59.0, 200.0])
def test_one_logit_far_above_the_rest_in_a_late_tile(dtype, groups, beams, vocab, lead):
    mx, _ = load_lib()
    ctx = mx.Context([(mx.FULL, 0, 0)], 2, 1, 64, mx.BF16, 1, 1, device=0)
    gen = torch.Generator("cuda").manual_seed(31)
    logits = torch.randn(groups, beams, vocab, generator=gen, device="cuda")
    at = torch.randint(vocab * 3 // 4, vocab, (groups, beams, 1), generator=gen, device="cuda")
    peak = logits.amax(-1, keepdim=True) + lead + torch.rand(groups, beams, 1, generator=gen, device="cuda")
    logits = logits.scatter(-1, at, peak).to(dtype)
    check(ctx, logits, -3 * torch.rand(groups, beams, generator=gen, device="cuda"), 1)
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rising_logits(dtype):
    # every tile leads the one before it: by a little, by a lot, and with the rows' ends out of line
    mx, _ = load_lib()
    ctx = mx.Context([(mx.FULL, 0, 0)], 2, 1, 64, mx.BF16, 1, 1, device=0)
    gen = torch.Generator("cuda").manual_seed(32)
    vocab = 100003
    ramp = torch.arange(vocab, device="cuda") / vocab
    rows = [c * ramp + torch.randn(vocab, generator=gen, device="cuda") for c in (3.0, 30.0, 300.0, 3000.0)]
    logits = torch.stack(rows).to(dtype).view(4, 1, vocab).repeat(100, 1, 1)     # (many rows: long chunks)
    check(ctx, logits, torch.zeros(400, 1, device="cuda"), 1)
    ctx.close()
