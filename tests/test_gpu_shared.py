"""Decode over a tree of shared prefixes on a B200 against the definition in 64 bits, every storage
format; and which calls give the bits of the ordinary decode.

Bounds, with A = sum_j p_j |v_j| of the output element in question (p the softmax weights): the output's own
rounding, half a step; weights held to 16 bits by bf16 caches (2^-16 A), as fp16 by quantised ones
(2^-11 A, plus half the fp16 subnormal step times the largest element, 448, per key), in fp32 by the fp32 mode
(2^-23 A); scores are fp32 numbers of magnitude s in base-2 units, off by at most 2^-24 s (head_dim / 4 + 16), which moves
weights by that times ln 2 and the output by at most twice that times A.  Merging c partial results adds a few
fp32 roundings of each, 2^-24 (c + 8) A."""
import math
import random

import pytest
import torch

from gpu_common import load_lib

pytestmark = pytest.mark.gpu

NEG = float("-inf")
WEIGHTS = {"bf16": 2.0 ** -16, "fp8": 2.0 ** -11, "f32": 2.0 ** -23}


def slopes_of(hq):
    return [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]


def on_e4m3(x):
    top = x.abs().amax(-1, keepdim=True).float()
    scale = torch.exp2(torch.floor(torch.log2(torch.clamp(top, min=1e-30))) - 8)
    return (torch.clamp(x.float() / scale, -448, 448).to(torch.float8_e4m3fn).float() * scale).to(x.dtype)


class Tree:
    """A context whose layer 0 owns a paged cache that layer 1 reads, with a copy of every sequence's keys and values."""

    def __init__(self, heads, dtype, seqs, pages, longest, seed=1, layout=None, fill=None, chunk=0):
        self.mx, _ = load_lib()
        mx = self.mx
        self.heads, self.dtype = heads, dtype
        self.ctx = mx.Context(layout or [(mx.FULL, 0, 0), (mx.FULL, 0, 0)], *heads, mx.F32 if dtype == "f32" else mx.BF16, seqs, pages,
                              max_seq_len=longest, device=0, kv_format=mx.KV_FP8_E4M3 if dtype == "fp8" else mx.KV_NATIVE,
                              chunk_scratch_tokens=chunk)
        self.ctx.set_share_min_bytes(0)      # (small trees too)
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.t = torch.float32 if dtype == "f32" else torch.bfloat16
        self.kv = {}
        self.cap, self.slopes = 0.0, None

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen, device="cuda").to(self.t)

    def shape(self, cap, bias):
        self.cap, self.slopes = cap, slopes_of(self.heads[0]) if bias else None
        for l in (0, 1):
            self.ctx.set_layer_scores(l, cap, self.slopes)

    def append(self, seq, n):
        if n == 0:
            return
        new = [self.normal(n, self.heads[1], self.heads[2]) for _ in range(2)]
        if self.dtype == "fp8":
            new = [on_e4m3(x) for x in new]
        self.ctx.append_kv(0, [seq], [n], *new)
        old = self.kv.get(seq)
        self.kv[seq] = new if old is None else [torch.cat(p) for p in zip(old, new)]

    def fork(self, src, dst):
        self.ctx.fork_seqs(src, dst)
        was = dict(self.kv)
        for s, d in zip(src, dst):
            self.kv[d] = was[s]

    def queries(self, n, sharp=2.0):
        return (self.normal(n, self.heads[0], self.heads[2]).float() * sharp).to(self.t)

    def expect(self, seqs, q, scale=None):
        hq, hkv, d = self.heads
        out, A, top = torch.empty(q.shape, dtype=torch.float64, device="cuda"), None, 0.0
        A = torch.empty_like(out)
        for i, s in enumerate(seqs):
            K, V = (x.double() for x in self.kv[s])
            back = torch.arange(len(K) - 1, -1, -1, device="cuda", dtype=torch.float64)
            z = torch.einsum("gcd,ngd->gcn", q[i].double().view(hkv, -1, d), K) * (d ** -0.5 if scale is None else scale)
            if self.cap:
                z = self.cap * torch.tanh(z / self.cap)
            if self.slopes is not None:
                z = z - torch.tensor(self.slopes, device="cuda", dtype=torch.float64).view(hkv, -1, 1) * back
            p = torch.softmax(z, -1)
            out[i] = torch.einsum("gcn,ngd->gcd", p, V).reshape(hq, d)
            A[i] = torch.einsum("gcn,ngd->gcd", p, V.abs()).reshape(hq, d)
            top = max(top, float(z.masked_fill(p < 2.0 ** -40, 0.0).abs().max()) / math.log(2))
        return out, A, top

    def check(self, seqs, q=None, layer=1, what=""):
        q = self.queries(len(seqs)) if q is None else q
        out = torch.full_like(q, float("nan"))
        self.ctx.decode_shared(layer, seqs, q, out)
        self.compare(seqs, q, out, what)
        return q, out

    def compare(self, seqs, q, out, what=""):
        torch.cuda.synchronize()
        assert self.ctx.get_device_status() == 0
        want, A, top = self.expect(seqs, q)
        n = max(len(self.kv[s][0]) for s in seqs)
        score = 2.0 ** -24 * top * (self.heads[2] / 4 + 16) * 2 * math.log(2)
        bound = torch.finfo(out.dtype).eps / 2 * want.abs() * 1.001 + (WEIGHTS[self.dtype] + score + 2.0 ** -24 * 200) * A + 1e-30
        if self.dtype == "fp8":
            bound += n * 2.0 ** -25 * 448
        err = (out.double() - want).abs()
        assert torch.isfinite(out).all(), what
        worst = float((err / bound).max())
        assert worst <= 1, f"{what}: {worst:.3f} of the bound, max error {float(err.max()):.3e}"


def grow(tree, groups, each, prefix, mid, tails):
    n = groups * each
    roots = list(range(n, n + groups))
    tree.append(roots[0], prefix)
    tree.fork([roots[0]] * groups, roots)
    for r in roots:
        tree.append(r, mid)
    tree.fork([roots[i % groups] for i in range(n)], list(range(n)))
    for i in range(n):
        tree.append(i, tails[i % len(tails)])
    return list(range(n))


FORMS = [  # heads, dtype
    ((32, 8, 128), "bf16"), ((32, 8, 128), "fp8"), ((12, 3, 128), "bf16"), ((16, 4, 64), "bf16"), ((20, 2, 64), "bf16"),
    ((16, 16, 128), "bf16"), ((16, 1, 128), "fp8"), ((4, 2, 64), "f32"), ((6, 2, 128), "f32")]
SHAPES = [(0.0, False), (50.0, False), (0.0, True), (30.0, True)]


@pytest.mark.parametrize("cap,bias", SHAPES)
@pytest.mark.parametrize("heads,dtype", FORMS)
def test_two_levels(heads, dtype, cap, bias):
    tree = Tree(heads, dtype, 15, 400, 2000)
    seqs = grow(tree, 3, 4, 517, 203, [1, 77, 16, 0, 131])
    tree.shape(cap, bias)
    assert tree.ctx.get_distinct_tokens(1, seqs) < sum(len(tree.kv[s][0]) for s in seqs) / 2
    tree.check(seqs)


# around the edges of pages, of tiles of 32 and 128 keys, and of the shortest shared piece
@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("prefix", [127, 128, 129, 143, 144, 145, 159, 160, 255, 256, 257, 1024, 1153])
def test_prefix_lengths(prefix, dtype):
    tree = Tree((8, 2, 128), dtype, 4, 400, 2000)
    seqs = grow(tree, 1, 3, prefix, 0, [0, 1, 18])
    tree.check(seqs)


@pytest.mark.parametrize("n", [2, 31, 32, 33, 64, 65, 128, 129, 150])
def test_batch_sizes(n):
    """Rows per KV head on both sides of a chunk of rows, batches on both sides of what one launch takes."""
    tree = Tree((8, 2, 64), "bf16", n + 1, 40 * n + 100, 1200)
    seqs = grow(tree, 1, n, 300, 0, list(range(1, 40)))
    tree.check(seqs)


@pytest.mark.parametrize("heads", [(71, 1, 64), (3, 3, 64), (130, 1, 128), (9, 3, 128)])
def test_odd_groups_of_heads(heads):
    tree = Tree(heads, "bf16", 6, 400, 1200)
    seqs = grow(tree, 1, 5, 400, 0, [3, 140])
    tree.check(seqs)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
def test_any_order_and_the_same_sequence_twice(dtype):
    tree = Tree((8, 2, 128), dtype, 15, 400, 2000)
    seqs = grow(tree, 3, 4, 300, 150, [1, 20, 40])
    q = tree.queries(len(seqs))
    _, straight = tree.check(seqs, q)
    order = list(range(12))
    random.Random(3).shuffle(order)
    _, mixed = tree.check([seqs[i] for i in order], q[order].contiguous())
    assert torch.equal(mixed, straight[order])          # the same tree, the same sums
    tree.check([0, 5, 0, 0, 7, 5])
    tree.check([4] * 40)
    tree.check(seqs + [12, 13, 14])                     # sequences that others begin with


def test_two_families_and_loners():
    tree = Tree((8, 2, 128), "bf16", 20, 800, 3000)
    a = grow(tree, 1, 4, 500, 0, [5])          # 0..3, root 4
    tree.append(5, 700)
    tree.fork([5] * 4, [6, 7, 8, 9])
    for s in (6, 7, 8):
        tree.append(s, 3 * s)
    tree.append(10, 1)
    tree.append(11, 900)
    tree.check([10, 6, 0, 11, 9, 1, 7, 2, 8, 3])


def test_deep_chain():
    """Every sequence goes on where the one before stopped: a tree as deep as it has sequences."""
    tree = Tree((4, 2, 64), "bf16", 60, 1200, 9000)
    tree.append(0, 140)
    for s in range(1, 60):
        tree.fork([s - 1], [s])
        tree.append(s, 140)
    tree.check(list(range(60)))
    tree.check(list(range(59, 0, -7)))


def test_after_steps_and_reorderings():
    tree = Tree((8, 2, 128), "bf16", 5, 300, 2000)
    seqs = grow(tree, 1, 4, 333, 0, [2])
    rng = random.Random(5)
    for step in range(20):
        tree.fork([rng.choice(seqs) for _ in seqs], seqs)
        for s in seqs:
            tree.append(s, 1)
        if step % 4 == 3:
            tree.check(seqs, layer=step % 2, what=f"step {step}")
    tree.ctx.seq_reset(2)
    tree.kv.pop(2)
    tree.append(2, 400)
    tree.check(seqs)


def bits(t):
    return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
def test_without_shared_prefixes_the_bits_of_decode(dtype):
    mx, _ = load_lib()
    for layout, prefix in (([(mx.FULL, 0, 0)] * 2, 100), ([(mx.SLIDING, 256, 0)] * 2, 700)):
        tree = Tree((8, 2, 128), dtype, 6, 600, 2000, layout=layout)
        tree.append(0, prefix)
        tree.fork([0] * 3, [1, 2, 3])
        for s in range(5):
            tree.append(s, 20 + s)
        seqs = [3, 0, 4, 1]
        q = tree.queries(4)
        a, b = torch.empty_like(q), torch.empty_like(q)
        tree.ctx.decode(1, seqs, q, a)
        tree.ctx.decode_shared(1, seqs, q, b)
        assert torch.equal(bits(a), bits(b))
    tree = Tree((8, 2, 128), dtype, 6, 600, 2000)
    seqs = grow(tree, 1, 4, 600, 0, [9])
    q = tree.queries(1)
    a, b = torch.empty_like(q), torch.empty_like(q)
    tree.ctx.decode(1, [2], q, a)
    tree.ctx.decode_shared(1, [2], q, b)
    assert torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_little_to_save_gives_the_bits_of_decode(dtype):
    """On both sides of the least that is worth sharing."""
    mx, _ = load_lib()
    tree = Tree((8, 2, 128), dtype, 5, 300, 2000)
    seqs = grow(tree, 1, 4, 600, 0, [9])
    token = 2 * 2 * 129 if dtype == "fp8" else 2 * 2 * 128 * 2
    saved = 3 * (600 // 16 * 16) * token
    assert saved < mx.MIN_SAVED_BYTES
    q = tree.queries(4)
    plain, out = torch.empty_like(q), torch.empty_like(q)
    tree.ctx.decode(1, seqs, q, plain)
    for least, same in ((-1, True), (saved + 1, True), (saved, False), (0, False)):
        tree.ctx.set_share_min_bytes(least)
        before = tree.ctx.get_launch_count()
        tree.ctx.decode_shared(1, seqs, q, out)
        assert (tree.ctx.get_launch_count() - before == 3) == (not same)
        assert not same or torch.equal(bits(out), bits(plain))
        tree.compare(seqs, q, out)


def test_switch_for_decode_and_decode_layers():
    tree = Tree((8, 2, 128), "bf16", 5, 300, 2000)
    seqs = grow(tree, 1, 4, 600, 0, [9, 40])
    q = tree.queries(4)
    plain, shared, switched = (torch.empty_like(q) for _ in range(3))
    tree.ctx.decode(1, seqs, q, plain)
    tree.ctx.decode_shared(1, seqs, q, shared)
    tree.ctx.set_prefix_sharing(True)
    tree.ctx.decode(1, seqs, q, switched)
    assert torch.equal(shared, switched)
    new = [tree.normal(4, 2, 128) for _ in range(2)]
    outs = [torch.empty_like(q) for _ in range(2)]
    at = tree.ctx.pointer_table
    tree.ctx.decode_layers(0, 2, seqs, at([q, q]), at([new[0], None]), at([new[1], None]), at(outs))
    for i, s in enumerate(seqs):
        tree.kv[s] = [torch.cat([old, x[i:i + 1]]) for old, x in zip(tree.kv[s], new)]
    for o in outs:
        tree.compare(seqs, q, o)
    tree.ctx.set_prefix_sharing(False)
    tree.ctx.seq_reset(4)
    again = torch.empty_like(q)
    tree.ctx.decode(1, [0, 1], q[:2].contiguous(), again[:2])
    tree.compare([0, 1], q[:2], again[:2])


@pytest.mark.parametrize("dtype,bad", [("bf16", float("inf")), ("bf16", float("nan")), ("f32", float("nan"))])
def test_what_earlier_sequences_left_behind(dtype, bad):
    """Pages that held infinities and NaN, taken over and filled in part."""
    tree = Tree((8, 2, 128), dtype, 6, 64, 1000)
    k = torch.full((1000, 2, 128), bad, device="cuda", dtype=tree.t)
    tree.ctx.append_kv(0, [0], [1000], k, k)
    tree.ctx.seq_reset(0)
    seqs = grow(tree, 1, 5, 200, 0, [1, 17, 30])
    tree.check(seqs)
    tree.check([0, 0, 0, 1])


def test_scores_that_climb_along_the_keys():
    """Later keys outweigh earlier ones by far more than a reference taken from the first keys allows for."""
    tree = Tree((8, 2, 128), "bf16", 5, 300, 2000)
    q = tree.queries(4, sharp=1.0)
    tree.append(4, 1)
    ramp = torch.linspace(0.0, 40.0, 700, device="cuda")[:, None, None]
    direction = q[0, 0].float().view(1, 1, -1) / q[0, 0].float().norm()
    k = (tree.normal(700, 2, 128).float() * 0.1 + ramp * direction).bfloat16()
    v = tree.normal(700, 2, 128)
    tree.ctx.append_kv(0, [4], [700], k, v)
    tree.kv[4] = [torch.cat([a, b]) for a, b in zip(tree.kv[4], (k, v))]
    tree.fork([4] * 4, [0, 1, 2, 3])
    for s in range(4):
        tree.append(s, 3 + s)
    q = q.clone()
    q[:, :] = (q.float() + 3 * q[0, 0].float()).bfloat16()
    tree.check([0, 1, 2, 3], q)


def test_another_owner_behind():
    """Owners share one block table; one that lags reads its own length."""
    mx, _ = load_lib()
    tree = Tree((8, 2, 128), "bf16", 5, 400, 2000, layout=[(mx.FULL, 0, 0), (mx.FULL, 0, 0), (mx.FULL, 0, 2)])
    k2 = [tree.normal(400, 2, 128) for _ in range(2)]
    tree.append(0, 400)
    tree.ctx.append_kv(2, [0], [250], k2[0][:250].contiguous(), k2[1][:250].contiguous())
    tree.fork([0] * 3, [1, 2, 3])
    tree.append(1, 20)
    tree.ctx.append_kv(2, [1], [150], k2[0][250:].contiguous(), k2[1][250:].contiguous())
    tree.check([0, 1, 2, 3])
    own = dict(tree.kv)
    tree.kv = {s: [x[:400 if s == 1 else 250] for x in k2] for s in range(4)}
    tree.check([3, 1, 2, 0], layer=2)
    tree.kv = own


def test_captured_and_replayed():
    tree = Tree((8, 2, 128), "bf16", 5, 300, 2000)
    seqs = grow(tree, 1, 4, 600, 0, [9, 40])
    q = tree.queries(4)
    eager, out = torch.empty_like(q), torch.empty_like(q)
    tree.ctx.decode_shared(1, seqs, q, eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tree.ctx.decode_shared(1, seqs, q, out, stream=side)
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    q2 = tree.queries(4)
    q.copy_(q2)
    graph.replay()
    tree.compare(seqs, q2, out)


def test_repeated_calls_give_the_same_bits():
    tree = Tree((32, 8, 128), "bf16", 41, 2000, 9000)
    seqs = grow(tree, 1, 40, 6001, 0, list(range(1, 400, 7)))
    q = tree.queries(40)
    _, first = tree.check(seqs, q)
    for _ in range(20):
        out = torch.full_like(q, float("nan"))
        tree.ctx.decode_shared(1, seqs, q, out)
        assert torch.equal(out, first)


def test_refusals():
    mx, _ = load_lib()
    tree = Tree((8, 2, 128), "bf16", 5, 300, 2000)
    seqs = grow(tree, 1, 3, 600, 0, [9])
    q = tree.queries(4)
    out = torch.full_like(q, 7.0)
    for layer, ids, code in ((2, seqs, mx.ERR_INVALID_ARG), (-1, seqs, mx.ERR_INVALID_ARG), (1, [0, 5], mx.ERR_BAD_SEQ),
                             (1, [0, -1], mx.ERR_BAD_SEQ), (1, [0, 4], mx.ERR_EMPTY_CONTEXT)):
        assert tree.ctx.rc_decode_shared(layer, ids, q, out) == code
    assert tree.ctx.rc_decode_shared(1, [0, 1], None, out) == mx.ERR_INVALID_ARG
    assert tree.ctx.rc_decode_shared(1, [0, 1], q, None) == mx.ERR_INVALID_ARG
    assert tree.ctx.rc_decode_shared(1, [], q, out) == 0
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
def test_unaligned_tensors_give_the_bits_of_decode(dtype):
    tree = Tree((8, 2, 128), dtype, 5, 300, 2000)
    seqs = grow(tree, 1, 4, 600, 0, [9, 40])
    step = 2 if dtype != "f32" else 1         # elements: 4 bytes
    n = 4 * 8 * 128
    spare = [torch.zeros(n + 8, device="cuda", dtype=tree.t) for _ in range(3)]
    q = tree.queries(4)
    odd_q, odd_out = (s[step:step + n].view(4, 8, 128) for s in spare[:2])
    odd_q.copy_(q)
    plain = torch.empty_like(q)
    tree.ctx.decode(1, seqs, q, plain)
    if dtype != "fp8":                        # (a quantised cache's decode takes queries of 8-byte alignment)
        out = torch.empty_like(q)
        tree.ctx.decode_shared(1, seqs, odd_q, out)
        assert torch.equal(bits(out), bits(plain))
    tree.ctx.decode_shared(1, seqs, q, odd_out)
    assert torch.equal(bits(odd_out), bits(plain))
    assert bool((spare[1][:step] == 0).all()) and bool((spare[1][step + n:] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (0.0, True), (30.0, True)])
def test_own_keys_of_every_length(dtype, cap, bias):
    """Lengths on both sides of pages, tiles and splits next to each other: the shares of the two kernels, the
    order of the items and the merge."""
    tree = Tree((32, 8, 128), dtype, 25, 6000, 9000, seed=3)
    tails = [0, 1, 5000, 15, 16, 17, 63, 64, 65, 127, 128, 129, 511, 512, 513, 1023, 1025, 2, 3, 2049, 30, 700, 1, 4097]
    seqs = grow(tree, 1, 24, 3000, 0, tails)
    tree.shape(cap, bias)
    tree.check(seqs)
    tree.ctx.set_split_tokens(64)
    tree.check(seqs)
    tree.ctx.set_split_tokens(0)


def test_magnitudes_that_differ_between_tokens():
    """A quantised cache's values of 2^-20 to 2^18 beside vectors of zeros: weights are rounded relative to what
    their keys contribute: 2^-11 of A, and 2^-24 of the largest contribution for each key (half the fp16 subnormal
    step, 2^-25, times an element of 448 at most where the largest one's is 256 at least).  The last twelve
    tokens, in pages of their own, are the ordinary split pass's: half that step times 448 each."""
    tree = Tree((8, 2, 128), "fp8", 5, 200, 1200)
    gen = torch.Generator("cuda").manual_seed(9)
    k = on_e4m3(torch.randn(700, 2, 128, generator=gen, device="cuda").bfloat16())
    size = torch.exp2(torch.randint(-20, 19, (700, 2, 1), generator=gen, device="cuda").float())
    size[::5] = 0.0
    v = on_e4m3((torch.randn(700, 2, 128, generator=gen, device="cuda") * size).bfloat16())
    tree.ctx.append_kv(0, [4], [700], k, v)
    tree.kv[4] = [k, v]
    tree.fork([4] * 4, [0, 1, 2, 3])
    q = tree.queries(4, sharp=1.0)
    out = torch.empty_like(q)
    tree.ctx.decode_shared(1, [0, 1, 2, 3], q, out)
    want, A, top = tree.expect([0, 1, 2, 3], q)
    largest = torch.zeros_like(want)
    for i in range(4):
        p = torch.softmax(torch.einsum("gcd,ngd->gcn", q[i].double().view(2, -1, 128), k.double()) / math.sqrt(128), -1)
        largest[i] = (p * v.double().abs().amax(-1).T[:, None]).amax(-1).reshape(8, 1)
    # the output's rounding: half a step of bf16, whose eps is 2^-7 (8 significant bits), so 2^-8 of the value
    half_step = torch.finfo(torch.bfloat16).eps / 2
    bound = half_step * want.abs() * 1.001 + (2.0 ** -11 + 2.0 ** -24 * top * 48 * 1.4 + 2.0 ** -16) * A + 700 * 2.0 ** -24 * largest + 12 * 2.0 ** -25 * 448
    assert ((out.double() - want).abs() <= bound).all()
    assert tree.ctx.get_device_status() == 0
