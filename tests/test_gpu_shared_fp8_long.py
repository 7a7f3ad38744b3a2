"""Long sequences on a quantised cache, with a bound that is formed key by key, so that a lost key or page shows: the test
checks on its oracle that the loss of any of the heavy keys, and of any page looked at, would exceed the bound.

p the softmax weights, v = code * 2^X, w = p 2^X what a key's codes are multiplied by, A = sum p |v|:
- the output's rounding, half a step of bf16;
- a weight's fp16 rounding: 2^-11 of it, in all 2^-11 A; or, where it lies in fp16's subnormal range, half that range's
  step, 2^-25, and no more than the weight itself, times the key's codes.  Weights are relative to a reference that is at
  most the largest w for common keys, and the largest p of a sequence's own keys for those;
- the scores, fp32 numbers of magnitude s in base-2 units, off by at most 2^-24 s (head_dim / 4 + 16), which moves the output
  by at most twice that times ln 2 times A;
- sums and merges in fp32, 2^-16 A."""
import math

import pytest
import torch

from test_gpu_shared import Tree, grow, on_e4m3, slopes_of

pytestmark = pytest.mark.gpu

HEADS = (32, 8, 128)


def weights(tree, q, K):
    hq, hkv, d = tree.heads
    n = len(K)
    z = torch.einsum("gcd,ngd->gcn", q.double().view(hkv, -1, d), K.double()) * d ** -0.5
    if tree.cap:
        z = tree.cap * torch.tanh(z / tree.cap)
    if tree.slopes is not None:
        back = torch.arange(n - 1, -1, -1, device="cuda", dtype=torch.float64)
        z = z - torch.tensor(slopes_of(hq), device="cuda", dtype=torch.float64).view(hkv, -1, 1) * back
    p = torch.softmax(z, -1)
    return p, float(z.masked_fill(p < 2.0 ** -40, 0.0).abs().max()) / math.log(2)


def expect(tree, seq, q, common):
    """(result, bound, p, V) of one sequence whose first `common` keys are shared."""
    K, V = tree.kv[seq]
    V = V.double()
    p, top = weights(tree, q, K)
    X = torch.floor(torch.log2(V.abs().amax(-1).clamp(min=1e-30))) - 8         # [n, g]
    codes = V.abs() / torch.exp2(X)[..., None]
    w = p * torch.exp2(X).T[:, None]
    lost = torch.zeros_like(p)
    for part, unit in ((slice(0, common), w[..., :common].amax(-1, keepdim=True)),
                       (slice(common, None), p[..., common:].amax(-1, keepdim=True) if len(K) > common else None)):
        if unit is not None:
            lost[..., part] = torch.where(w[..., part] < 2.0 ** -14 * unit, torch.minimum(w[..., part], 2.0 ** -25 * unit), 0.0)
    want = torch.einsum("gcn,ngd->gcd", p, V)
    A = torch.einsum("gcn,ngd->gcd", p, V.abs())
    score = 2.0 ** -24 * top * (tree.heads[2] / 4 + 16) * 2 * math.log(2)
    bound = torch.finfo(torch.bfloat16).eps / 2 * want.abs() * 1.001 + (2.0 ** -11 + score + 2.0 ** -16) * A + torch.einsum("gcn,ngd->gcd", lost, codes)
    return want, bound, p, V


def without(want, p, V, keys):
    """The result if these keys were lost."""
    gone = p[..., keys].sum(-1, keepdim=True)
    return (want - torch.einsum("gcn,ngd->gcd", p[..., keys], V[keys])) / (1 - gone)


def check(tree, seqs, common, q):
    out = torch.full_like(q, float("nan"))
    before = tree.ctx.get_launch_count()
    tree.ctx.decode_shared(1, seqs, q, out)
    assert tree.ctx.get_launch_count() - before == 3
    torch.cuda.synchronize()
    assert tree.ctx.get_device_status() == 0
    hq, hkv, d = tree.heads
    for i, s in enumerate(seqs):
        want, bound, p, V = expect(tree, s, q[i], common)
        err = (out[i].double().view(hkv, -1, d) - want).abs()
        assert (err <= bound).all(), f"sequence {s}: {float((err / bound).max()):.3f} of the bound"
        n = len(V)
        if tree.slopes is None:      # (with a distance bias far pages hardly count)
            for page in list(range(0, n // 16, 61)) + [common // 16 - 1, n // 16 - 1]:
                moved = (without(want, p, V, list(range(16 * page, 16 * page + 16))) - want).abs() / bound
                assert float(moved.max()) > 2, f"the loss of page {page} would pass"


@pytest.mark.parametrize("cap,bias", [(0.0, False), (30.0, False), (0.0, True), (30.0, True)])
@pytest.mark.parametrize("prefix", [3000, 8000])
def test_every_key_counts(prefix, cap, bias):
    tails = [1, 300, 16, 5000]
    tree = Tree(HEADS, "fp8", 5, prefix // 16 + 500, prefix + 5100, seed=prefix)
    seqs = grow(tree, 1, 4, prefix, 0, tails)
    tree.shape(cap, bias)
    check(tree, seqs, prefix // 16 * 16, tree.queries(4, sharp=1.0))


@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_heavy_keys_at_the_edges(cap):
    """Keys that every head looks at, on both sides of pages, of half tiles and tiles, of where CTAs' shares may end and
    of where the common keys do; the others count little."""
    prefix = 8000
    hq, hkv, d = HEADS
    tree = Tree(HEADS, "fp8", 5, prefix // 16 + 500, prefix + 3100, seed=7)
    edges = [0, 15, 16, 63, 64, 127, 128, 1023, 1024, 2047, 2048, 3199, 3200, 4095, 4096, 6143, 6144, 7935, 7936, 7984, 7999]
    direction = tree.normal(1, 1, d).float()
    direction /= direction.norm()
    k, v = tree.normal(prefix, hkv, d).float(), tree.normal(prefix, hkv, d)
    k[edges] = 0.5 * k[edges] + 22.0 * direction
    k, v = on_e4m3(k.bfloat16()), on_e4m3(v)
    tree.ctx.append_kv(0, [4], [prefix], k, v)
    tree.kv[4] = [k, v]
    tree.fork([4] * 4, [0, 1, 2, 3])
    own = [1, 17, 3000, 129]
    heavy_own = [8000, 8016, 8128]
    for s, n in enumerate(own):
        k, v = tree.normal(n, hkv, d).float(), tree.normal(n, hkv, d)
        at = [x - prefix for x in heavy_own if x - prefix < n]
        k[at] = 0.5 * k[at] + 22.0 * direction
        k, v = on_e4m3(k.bfloat16()), on_e4m3(v)
        tree.ctx.append_kv(0, [s], [n], k, v)
        tree.kv[s] = [torch.cat([a, b]) for a, b in zip(tree.kv[s], (k, v))]
    tree.shape(cap, False)
    q = (0.3 * tree.normal(4, hq, d).float() + 4.0 * direction).bfloat16()
    out = torch.full_like(q, float("nan"))
    seqs = [0, 1, 2, 3]
    tree.ctx.decode_shared(1, seqs, q, out)
    torch.cuda.synchronize()
    for i, s in enumerate(seqs):
        want, bound, p, V = expect(tree, s, q[i], prefix)
        err = (out[i].double().view(hkv, -1, d) - want).abs()
        assert (err <= bound).all(), f"sequence {s}: {float((err / bound).max()):.3f} of the bound"
        for key in edges + [x for x in heavy_own if x < len(V)]:
            moved = (without(want, p, V, [key]) - want).abs() / bound
            assert float(moved.amax(-1).min()) > 2, f"the loss of key {key} would pass"
