"""Quantised caches whose values are tiny: what a shared decode makes of exponents down to the format's lowest, beside
ordinary ones and alone, against the definition in 64 bits on the values that the cache gives back.

Bound, p the softmax weights: the output's rounding, half a step of bf16; 2^-11 of A = sum p |v|, and 2^-24 of the
largest contribution for each key (test_gpu_shared.py); 2^-16 A and the scores' share as there; values below 2^-51 are
held in steps of 2^-84 (codes times the rest of their exponent, in fp16), so half a step of that for every key's
weight, together 2^-85; a vector below 2^-118 reads as zero.  Own keys (the last twelve, in pages of their own) go
through the split pass: half the fp16 subnormal step times 448 each where their values are ordinary, and no more than what
they contribute, 12 * 2^-100, where they are tiny too."""
import math

import pytest
import torch

from test_gpu_shared import Tree

pytestmark = pytest.mark.gpu


def run(n, size_of, own_size, sharp):
    """n tokens, of which n % 16 == 12 are behind the pages that the four forks share; size_of gives the tokens' scale."""
    assert n % 16 == 12
    tree = Tree((8, 2, 128), "fp8", 5, 4 * (n // 16 + 4), n + 16)
    gen = torch.Generator("cuda").manual_seed(n)
    size = size_of(n, gen)
    size[n - 12:] = own_size
    k = torch.randn(n, 2, 128, generator=gen, device="cuda").bfloat16()
    v = (torch.randn(n, 2, 128, generator=gen, device="cuda") * size.float()).bfloat16()
    tree.ctx.append_kv(0, [4], [n], k, v)
    tree.ctx.fork_seqs([4] * 4, [0, 1, 2, 3])
    back = [x.clone() for x in tree.ctx.read_kv(0, [4])]
    for s in range(5):
        tree.kv[s] = back
    q = tree.queries(4, sharp=sharp)
    out = torch.full_like(q, float("nan"))
    before = tree.ctx.get_launch_count()
    tree.ctx.decode_shared(1, [0, 1, 2, 3], q, out)
    assert tree.ctx.get_launch_count() - before == 3
    torch.cuda.synchronize()
    assert tree.ctx.get_device_status() == 0
    want, A, top = tree.expect([0, 1, 2, 3], q)
    largest = torch.zeros_like(want)
    for i in range(4):
        p = torch.softmax(torch.einsum("gcd,ngd->gcn", q[i].double().view(2, -1, 128), back[0].double()) / math.sqrt(128), -1)
        big = back[1].double().abs().amax(-1)
        big[n - 12:] = 0
        largest[i] = (p * big.T[:, None]).amax(-1).reshape(8, 1)
    own = 12 * 2.0 ** -25 * 448 if own_size > 2.0 ** -30 else 12 * 2.0 ** -100
    bound = torch.finfo(torch.bfloat16).eps / 2 * want.abs() * 1.001 + (2.0 ** -11 + 2.0 ** -24 * top * 48 * 1.4 + 2.0 ** -16) * A \
        + n * 2.0 ** -24 * largest + 2.0 ** -85 + own
    err = (out.double() - want).abs()
    assert torch.isfinite(out).all()
    assert (err <= bound).all(), f"{float((err / bound).max()):.3g} of the bound, max error {float(err.max()):.3e}, largest output {float(want.abs().max()):.3e}"


def of(*exponents):
    """Tokens' scales: powers of two picked from the list, None for vectors of zeros."""
    values = torch.tensor([0.0 if e is None else 2.0 ** e for e in exponents], dtype=torch.float64, device="cuda")
    return lambda n, gen: values[torch.randint(len(exponents), (n, 1, 1), generator=gen, device="cuda")]


@pytest.mark.parametrize("own", [2.0 ** -100, 1.0])
@pytest.mark.parametrize("exponents", [(-115,), (-120,), (-122, -119, -116), (-60,), (-55, -52, -49), (None,), (None, -120)])
def test_all_of_them_tiny(exponents, own):
    run(3020, of(*exponents), own, 0.5)


@pytest.mark.parametrize("sharp", [0.5, 2.0])
@pytest.mark.parametrize("exponents", [(0, -115, -116, -117), (0, 0, -60, -80, -100, None), (-40, -121), (12, -45, -118), (0, None, None, None),
                                       (-70, -90, -105, -120)])
def test_beside_others(exponents, sharp):
    run(1500, of(*exponents), 1.0, sharp)


def test_a_single_tile_in_many_is_tiny():
    def size(n, gen):
        s = torch.ones(n, 1, 1, dtype=torch.float64, device="cuda")
        s[256:384] = 2.0 ** -119
        s[700] = 2.0 ** -118
        s[901:905] = 0.0
        return s
    run(1500, size, 1.0, 1.0)
