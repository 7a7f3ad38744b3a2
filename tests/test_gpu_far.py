"""Pages, rows and logits whose byte offsets pass 32 bits: shared-prefix decode, rotated projections and adjusted
logits.  Strided rows are compared with the bits of the same rows lying together, decodes with the definition in
64 bits (bounds: test_gpu_shared.py)."""
import pytest
import torch

from gpu_common import load_lib
from test_gpu_shared import Tree, grow

pytestmark = pytest.mark.gpu


class FarTree(Tree):
    """The pool's pages are handed out from its end."""

    def __init__(self, heads, dtype, seqs, longest, page_bytes, **kw):
        super().__init__(heads, dtype, seqs, 64, longest, **kw)
        mx = self.mx
        pages = (1 << 32) // page_bytes + 2000
        self.ctx = mx.Context([(mx.FULL, 0, 0), (mx.FULL, 0, 0)], *heads, mx.F32 if dtype == "f32" else mx.BF16, seqs, pages,
                              max_seq_len=longest, device=0, kv_format=mx.KV_FP8_E4M3 if dtype == "fp8" else mx.KV_NATIVE,
                              free_order=list(range(pages - 1, -1, -1)))
        self.ctx.set_share_min_bytes(0)
        assert pages * page_bytes > 1 << 32


@pytest.mark.parametrize("heads,dtype,page_bytes", [((32, 8, 128), "bf16", 65536), ((32, 8, 128), "fp8", 33024), ((16, 4, 64), "bf16", 16384),
                                                    ((6, 2, 128), "f32", 32768)])
def test_pages_beyond_32_bits(heads, dtype, page_bytes):
    t = FarTree(heads, dtype, 9, 4096, page_bytes)
    seqs = grow(t, 2, 3, 700, 130, [1, 40, 300])
    table = t.ctx.get_block_table(seqs[0])
    assert min(table) * page_bytes > (1 << 32) - 2000 * page_bytes and max(table) * page_bytes >= 1 << 32
    t.check(seqs)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_rows_are_stored_beyond_32_bits(dtype):
    page_bytes = 65536 if dtype == "bf16" else 33024
    t = FarTree((32, 8, 128), dtype, 2, 4096, page_bytes)
    near = Tree((32, 8, 128), dtype, 2, 64, 512)
    rope = t.mx.Rope(128, 10000.0)
    for n in ([200, 33], [1, 1]):
        q, k, v = (t.normal(sum(n), h, 128) for h in (32, 8, 8))
        got = [x.ctx.rope_qkv(0, [0, 1], n, rope, q=q, k=k, v=v, store=True)[0] for x in (t, near)]
        assert torch.equal(*got)
    far_kv, near_kv = (x.ctx.read_kv(0, [0, 1]) for x in (t, near))
    torch.cuda.synchronize()
    assert max(t.ctx.get_block_table(0)) * page_bytes >= 1 << 32
    assert all(torch.equal(a, b) for a, b in zip(far_kv, near_kv))


def test_projection_rows_far_apart():
    t = Tree((32, 8, 128), "bf16", 2, 64, 512)
    apart = (1 << 30) + 64                          # elements: the third row begins 4 GB behind the first
    memory = torch.empty(2 * apart + 48 * 128, dtype=torch.bfloat16, device="cuda")
    rows = memory.as_strided((3, 48, 128), (apart, 128, 1))
    rows.copy_(t.normal(3, 48, 128))
    dense = rows.contiguous()
    rope = t.mx.Rope(64, 500000.0, halves=True)
    got = [t.ctx.rope_qkv(0, [1, 0], [2, 1], rope, q=x[:, :32], k=x[:, 32:40], v=x[:, 40:], first_pos=[77, 3000]) for x in (rows, dense)]
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert torch.equal(got[0][2], dense[:, 40:])


@pytest.mark.parametrize("in_place", [False, True])
def test_logits_far_apart(in_place):
    t = Tree((4, 2, 64), "bf16", 1, 4, 64)
    vocab, rows, apart = 50021, 4, (1 << 30) + 5    # elements: 2 GB, so that rows pass 2^31 elements and 2^32 bytes
    memory = torch.empty((rows - 1) * apart + vocab, dtype=torch.bfloat16, device="cuda")
    x = memory.as_strided((rows, vocab), (apart, 1))
    x.copy_((t.normal(rows, vocab).float() * 4).to(torch.bfloat16))
    dense = x.contiguous()
    tokens = torch.randint(0, vocab, (rows, 700), generator=t.gen, device="cuda", dtype=torch.int32)
    allowed = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, (vocab + 31) // 32), generator=t.gen, device="cuda", dtype=torch.int64).to(torch.int32)
    rules = dict(tokens=tokens, repetition=torch.full((rows,), 1.3, device="cuda"), frequency=torch.full((rows,), 0.2, device="cuda"),
                 temperature=torch.tensor([1.0, 0.7, 1.0, 1.5], device="cuda"), allowed=allowed)
    want = torch.empty_like(dense)
    t.ctx.adjust_logits(dense, want, **rules)
    if in_place:
        t.ctx.adjust_logits(x, **rules)
        got = x
    else:
        got = torch.empty_like(dense)
        t.ctx.adjust_logits(x, got, **rules)
    torch.cuda.synchronize()
    assert torch.equal(got.contiguous(), want)
    assert not torch.equal(want, dense)
