"""Which way a shared decode goes by itself (MIXATTN_MIN_SAVED_BYTES and the estimate of both ways): what runs as the ordinary
decode has its bits and launches; where sharing pays several times over it is taken."""
import pytest
import torch

from test_gpu_shared import Tree, bits, grow

pytestmark = pytest.mark.gpu

WIDE, NARROW = (32, 8, 128), (16, 4, 64)


@pytest.mark.parametrize("heads,dtype,n,prefix,shares", [
    # more than 56 MB saved, of few distinct ones or by two sequences: ordinary
    (WIDE, "bf16", 16, 1024, False), (WIDE, "bf16", 2, 16384, False), (WIDE, "bf16", 32, 512, False), (WIDE, "fp8", 16, 2048, False),
    (WIDE, "fp8", 2, 32768, False), (NARROW, "bf16", 64, 1024, False), ((16, 16, 128), "bf16", 8, 1024, False),
    # less than that
    (WIDE, "bf16", 4, 2048, False), ((12, 3, 128), "bf16", 8, 4096, False),
    # sharing pays
    (WIDE, "bf16", 8, 8192, True), (WIDE, "bf16", 16, 4096, True), (WIDE, "bf16", 64, 2048, True), (WIDE, "fp8", 16, 8192, True),
    (NARROW, "bf16", 40, 8192, True), ((12, 3, 128), "bf16", 32, 8192, True), ((8, 1, 128), "fp8", 64, 16384, True)])
def test_the_way_taken(heads, dtype, n, prefix, shares):
    tree = Tree(heads, dtype, n + 1, prefix // 16 + 8 * n + 8, prefix + 200)
    seqs = grow(tree, 1, n, prefix, 0, [64])
    token = 2 * heads[1] * (129 if dtype == "fp8" else heads[2] * 2)
    q = tree.queries(n)
    plain, shared, out = (torch.empty_like(q) for _ in range(3))

    def launches(call):
        before = tree.ctx.get_launch_count()
        call()
        return tree.ctx.get_launch_count() - before

    of_plain = launches(lambda: tree.ctx.decode(1, seqs, q, plain))
    assert launches(lambda: tree.ctx.decode_shared(1, seqs, q, shared)) == 3
    tree.ctx.set_share_min_bytes(-1)
    assert launches(lambda: tree.ctx.decode_shared(1, seqs, q, out)) == (3 if shares else of_plain)
    assert torch.equal(bits(out), bits(shared if shares else plain))
    tree.compare(seqs, q, out)
    tree.ctx.set_share_min_bytes((n - 1) * (prefix // 16 * 16) * token)      # a measure of the caller's own
    assert launches(lambda: tree.ctx.decode_shared(1, seqs, q, out)) == 3
    tree.ctx.set_share_min_bytes(-1)
    tree.ctx.set_prefix_sharing(True)
    assert launches(lambda: tree.ctx.decode(1, seqs, q, out)) == (3 if shares else of_plain)
    assert torch.equal(bits(out), bits(shared if shares else plain))
