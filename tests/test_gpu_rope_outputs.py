"""What rope_qkv takes to write to: a triple of dense tensors, one for each that is there; anything else is refused before
the cache moves."""
import pytest
import torch

from test_gpu_rope_qkv import make, projection

pytestmark = pytest.mark.gpu


def test_outputs_that_are_no_triple_of_tensors():
    heads = (8, 2, 64)
    mx, ctx = make(heads, "bf16", 0)
    q, k, v = projection(heads, 4, "bf16")
    qo, ko, vo = torch.full_like(q, 7.0).contiguous(), torch.full_like(k, 7.0).contiguous(), torch.full_like(v, 7.0).contiguous()
    rope = mx.Rope(64)
    bad = [(), (qo,), (qo, ko), (qo, ko, vo, None), qo, 5, {"q": qo}, (qo, ko, vo.float()), (ko, ko, vo), (qo.cpu(), None, None), (q, None, None),
           (qo[:3], None, None)]
    for out in bad:
        for store in (False, True):
            with pytest.raises(mx.MixAttnError) as e:
                ctx.rope_qkv(0, [0, 1], [2, 2], rope, q=q, k=k, v=v, store=store, out=out)
            assert e.value.code == mx.ERR_INVALID_ARG
            assert ctx.get_len(0, 0) == 0
    torch.cuda.synchronize()
    assert all(bool((t == 7.0).all()) for t in (qo, ko, vo))
    want = ctx.rope_qkv(0, [0, 1], [2, 2], rope, q=q, k=k, v=v)
    got = ctx.rope_qkv(0, [0, 1], [2, 2], rope, q=q, k=k, v=v, out=[qo, ko, vo])
    assert got[0] is qo and all(torch.equal(a, b) for a, b in zip(got, want))
    assert ctx.rope_qkv(0, [0, 1], [2, 2], rope, q=q, k=k, v=v, store=True, out=None) == (None, None, None)
    assert ctx.get_len(0, 0) == 2
