"""Shared decode in an arena that ends short of the room it asks for, and next to the other users of the workspace."""
import ctypes as C

import pytest
import torch

from gpu_common import load_lib
from test_gpu_shared import Tree, bits, grow

pytestmark = pytest.mark.gpu


def recreated(tree, nbytes):
    """The tree's context again, in the first nbytes of its arena; the status of the call."""
    mx, ctx = tree.mx, tree.ctx
    mx.lib.mixattn_destroy(ctx.h)
    ctx.cfg.arena_bytes = nbytes
    h = C.c_void_p()
    rc = mx.lib.mixattn_create(C.byref(ctx.cfg), C.byref(h))
    ctx.h = h if rc == 0 else None
    ctx.set_share_min_bytes(0) if rc == 0 else None
    return rc


@pytest.mark.parametrize("share", [0.0, 0.02, 0.3, 1.0])
@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 2, 64), "bf16"), ((8, 1, 128), "fp8"), ((1, 1, 128), "bf16")])
def test_arenas_that_end_short(heads, dtype, share):
    """From the workspace of the ordinary decode alone (1408 slots of a row per query head) to all that is asked for."""
    tree = Tree(heads, dtype, 41, 1200, 6000)
    split = sum((n + 255) // 256 * 256 for n in (1408 * heads[0] * heads[2] * 4, 1408 * heads[0] * 8))
    asked = 512 * heads[0] * (heads[2] * 4 + 8) + (160 * 128 + 256 * heads[0]) * (heads[2] * 4 + 8)
    least = tree.mx.arena_bytes(tree.ctx.cfg) - (asked - split)
    nbytes = int(least + share * (asked - split)) // 256 * 256
    assert recreated(tree, nbytes) == 0
    tree.ctx.arena[nbytes:] = 0x5a
    seqs = grow(tree, 1, 40, 4003, 0, [1, 300, 16, 77])
    tree.check(seqs)
    tree.check(seqs[:3])
    assert bool((tree.ctx.arena[nbytes:] == 0x5a).all())
    assert recreated(tree, least - 256) == tree.mx.ERR_INVALID_ARG


def test_workspace_between_the_calls_that_use_it():
    """Ordinary and shared decodes and selections one after the other, which write their partial results to the same memory."""
    mx, _ = load_lib()
    tree = Tree((32, 8, 128), "bf16", 25, 2000, 4000, chunk=64)
    seqs = grow(tree, 1, 24, 2003, 0, [1, 300, 16, 77, 900])
    q = tree.queries(24)
    logits = tree.normal(24, 50021).view(6, 4, 50021)
    scores = torch.zeros(6, 4, device="cuda")
    plain, shared = torch.empty_like(q), torch.empty_like(q)
    tree.ctx.decode(1, seqs, q, plain)
    tree.ctx.decode_shared(1, seqs, q, shared)
    first = [x.clone() for x in tree.ctx.beam_select(logits, scores, 4)]
    tree.compare(seqs, q, shared)
    outs = []
    for _ in range(10):
        a, b = torch.full_like(q, float("nan")), torch.full_like(q, float("nan"))
        tree.ctx.decode_shared(1, seqs, q, b)
        tree.ctx.decode(1, seqs, q, a)
        sel = tree.ctx.beam_select(logits, scores, 4)
        c = torch.full_like(q, float("nan"))
        tree.ctx.decode_shared(1, seqs, q, c)
        outs.append((a, b, c, sel))
    torch.cuda.synchronize()
    for a, b, c, sel in outs:
        assert torch.equal(bits(a), bits(plain)) and torch.equal(bits(b), bits(shared)) and torch.equal(bits(c), bits(shared))
        assert all(torch.equal(x, y) for x, y in zip(sel, first))


def test_many_own_keys_for_the_slots():
    """More own keys than slots of the usual length: longer ones."""
    tree = Tree((8, 1, 64), "bf16", 65, 16000, 5000)
    seqs = grow(tree, 1, 64, 200, 0, [3001, 4500, 2999, 16])
    tree.check(seqs)
    tree.ctx.set_split_tokens(16)
    tree.check(seqs)
