"""Sets of grammar masks that hold none: a row without a mask of its own to follow is refused, not left unmasked."""
import torch
import pytest

from gpu_common import load_lib

pytestmark = pytest.mark.gpu


def test_no_masks_at_all():
    mx, _ = load_lib()
    ctx = mx.Context([(mx.FULL, 0, 0)], 4, 2, 64, mx.BF16, 1, 1, device=0)
    x, out = torch.zeros(3, 100, device="cuda"), torch.full((3, 100), 5.0, device="cuda")
    none = torch.zeros(0, 4, device="cuda", dtype=torch.int32)
    assert ctx.rc_adjust_logits(x, out, allowed=none) == mx.ERR_INVALID_ARG
    assert ctx.rc_adjust_logits(x, out, allowed=none, allowed_rows=torch.full((3,), -1, device="cuda", dtype=torch.int32)) == mx.ERR_INVALID_ARG
    with pytest.raises(mx.MixAttnError):
        ctx.adjust_logits(x, out, allowed=none)
    torch.cuda.synchronize()
    assert bool((out == 5.0).all())
    assert ctx.rc_adjust_logits(x[:0], out[:0], allowed=none) == 0       # (no row asks for one)
