"""Shared decode of capped scores where the common keys end inside a page: results are functions of the keys, whatever lies
behind the last one and whatever was computed on the same SMs before."""
import pytest
import torch

from test_gpu_shared import Tree

pytestmark = pytest.mark.gpu


def bits(t):
    return t.view(torch.int16)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("heads", [(32, 8, 128), (16, 4, 64)])
@pytest.mark.parametrize("n", [129, 137, 190, 200, 333])
def test_rows_behind_the_last_key_leave_no_trace(n, heads, bias):
    """The same keys in pages that held large numbers before, in pages of zeros, and after calls on other data."""
    hq, hkv, d = heads
    results = []
    for fill in (0.0, 1e30, float("nan"), -3e4):
        tree = Tree(heads, "bf16", 5, 25, 400, seed=n)
        tree.shape(6.0, bias)
        old = torch.full((400, hkv, d), fill, device="cuda", dtype=torch.bfloat16)
        tree.ctx.append_kv(0, [3], [400], old, old)
        if fill == fill:
            q = tree.normal(2, hq, d)
            tree.ctx.decode_shared(1, [3, 3], q, torch.empty_like(q))     # (leaves its tiles in shared memory)
        tree.ctx.seq_reset(3)
        tree.gen.manual_seed(n)
        k, v = (tree.normal(n, hkv, d) for _ in range(2))
        k = (k.float() * 0.3).bfloat16()         # scores well within half the cap
        tree.ctx.append_kv(0, [0], [n], k, v)
        tree.kv[0] = [k, v]
        q = tree.normal(64, hq, d)
        out = torch.empty_like(q)
        before = tree.ctx.get_launch_count()
        tree.ctx.decode_shared(1, [0] * 64, q, out)
        assert tree.ctx.get_launch_count() - before >= 2
        tree.compare([0] * 64, q, out)
        results.append(out)
    for other in results[1:]:
        assert torch.equal(bits(other), bits(results[0]))
