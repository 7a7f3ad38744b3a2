"""Quotients of adjusted logits: fp32 results carry the formula's own quotient, not a product with a reciprocal; what is
divided by may be anywhere in the range of fp32.

A rule alone is one operation on numbers that fp32 holds.  fp32 results: half a step of the exact quotient, (1 + 2^-21) times:
the reciprocal may come in two terms, hi cut off to 24 bits and lo < 2^-23 hi, off by 2^-24 of itself, whose product with x is
rounded (2^-24 of it): together 2^-46 of the quotient, whose half step is at least 2^-25 of it; what is lost below fp32's
smallest step on the way, 2^-149 / |x| of the result; results below fp32's normals may be off by
one smallest step, 2^-149.  bf16 results may be products with a reciprocal: two roundings of 2^-24, then half a
step of bf16, at least half of its smallest, 2^-134, and what fp32 loses on the way, 2^-149."""
import pytest
import torch

from gpu_common import load_lib

pytestmark = pytest.mark.gpu

ENDS = [2.0 ** -149, 1e-42, 1e-39, 2.0 ** -126, 1.5e-38, 1e-30, 3e-20, 0.7, 1.3, 3e20, 1e30, 8e37, 2.0 ** 127, 3.4028235e38]


def context():
    mx, _ = load_lib()
    return mx, mx.Context([(mx.FULL, 0, 0)], 4, 2, 64, mx.BF16, 1, 1, device=0)


def close(out, want, x):
    """Whether fp32 results are within their bound of quotients `want` (in 64 bits) of x."""
    _, e = torch.frexp(want)                                   # want in [2^(e-1), 2^e)
    half = torch.exp2(torch.clamp(e - 25, min=-150).double())
    lost = torch.where(x == 0, 0.0, want.abs() * 2.0 ** -149 / x.abs())
    low = torch.where(want.abs() < 2.0 ** -125, 2.0 ** -149, 0.0)
    return (out.double() - want).abs() <= half * (1 + 2.0 ** -21) + lost + low


@pytest.mark.parametrize("ti", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [5000, 4097])
def test_fp32_results_are_rounded_once(ti, vocab):
    mx, ctx = context()
    gen = torch.Generator("cuda").manual_seed(5)
    rows = 40
    logits = (torch.randn(rows, vocab, generator=gen, device="cuda") * 4).to(ti)
    divisor = 0.3 + 2 * torch.rand(rows, generator=gen, device="cuda")
    x, by = logits.double(), divisor.double()[:, None]
    for place in (False, True):
        here = logits.clone()
        out = here if place and ti == torch.float32 else torch.empty(rows, vocab, device="cuda")
        ctx.adjust_logits(here, out, temperature=divisor)
        assert close(out, x / by, x).all()
    out = torch.empty(rows, vocab, device="cuda")
    everything = torch.arange(vocab, device="cuda", dtype=torch.int32).repeat(rows, 1)
    ctx.adjust_logits(logits, out, tokens=everything, repetition=divisor)
    assert close(out, torch.where(x > 0, x / by, x * by), x).all()


def test_zeros_keep_their_sign():
    mx, ctx = context()
    x = torch.zeros(2, 999, device="cuda")
    x[:, ::2] = -0.0
    out = torch.empty_like(x)
    ctx.adjust_logits(x, out, temperature=torch.tensor([0.7, 1.0], device="cuda"))
    assert torch.equal(out.view(torch.int32), x.view(torch.int32))


@pytest.mark.parametrize("rule", ["temperature", "repetition"])
@pytest.mark.parametrize("ti,to", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_divisors_from_end_to_end(ti, to, rule):
    mx, ctx = context()
    rows, vocab = len(ENDS), 4100
    gen = torch.Generator("cuda").manual_seed(6)
    size = torch.exp2(torch.rand(rows, vocab, generator=gen, device="cuda") * 250 - 125)
    logits = (torch.randn(rows, vocab, generator=gen, device="cuda") * size).clamp(-3e38, 3e38).to(ti)
    logits[:, ::41] = 0.0
    divisor = torch.tensor(ENDS, device="cuda")
    rules = {"temperature": divisor} if rule == "temperature" else \
        {"repetition": divisor, "tokens": torch.arange(vocab, device="cuda", dtype=torch.int32).repeat(rows, 1)}
    out = torch.empty(rows, vocab, device="cuda", dtype=to)
    ctx.adjust_logits(logits, out, **rules)
    x, by = logits.double(), divisor.double()[:, None]
    want = x / by if rule == "temperature" else torch.where(x > 0, x / by, x * by)
    limit = torch.finfo(to).max * (1 + torch.finfo(to).eps / 4)       # where rounding gives infinity
    sure, near = want.abs() >= limit * (1 + 2.0 ** -20), want.abs() >= limit * (1 - 2.0 ** -20)
    assert torch.isfinite(want).all() and not torch.isnan(out).any()
    assert torch.equal(out.double()[sure], torch.sign(want[sure]) * float("inf"))
    if to == torch.float32:
        assert close(out, want, x)[~near].all()
    else:
        bound = torch.finfo(to).eps / 2 * want.abs() * 1.001 + 4 * 2.0 ** -24 * want.abs() + 2.0 ** -134 + 2.0 ** -149
        assert ((out.double() - want).abs()[~near] <= bound[~near]).all()


@pytest.mark.parametrize("ti,to", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_a_divisor_of_zero_leaves_no_nan(ti, to):
    """It is none, but loops that set it for their greedy rows keep the order of what fp32 can tell apart."""
    mx, ctx = context()
    gen = torch.Generator("cuda").manual_seed(7)
    logits = (torch.randn(3, 4097, generator=gen, device="cuda") * 2).to(ti)
    logits[:, ::9] = 0.0
    zero = torch.tensor([0.0, 1.0, 0.0], device="cuda")
    out = torch.empty(3, 4097, device="cuda", dtype=to)
    ctx.adjust_logits(logits, out, temperature=zero)
    want = logits.float() * torch.where(zero == 0, torch.finfo(torch.float32).max, 1.0)[:, None]
    assert torch.equal(out, want.to(to))
    everything = torch.arange(4097, device="cuda", dtype=torch.int32).repeat(3, 1)
    ctx.adjust_logits(logits, out, tokens=everything, repetition=zero)
    assert not torch.isnan(out).any() and torch.equal(out[1], logits[1].to(to))
