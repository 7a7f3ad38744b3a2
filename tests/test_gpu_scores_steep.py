"""Prompts and chunks on a B200 whose heads are biased so steeply that a row is a mix of a few keys:
like the first rows of a sequence they carry their weights to 16 bits (two bf16 terms, off by 2^-9
times 2^-9 at most), not to one bf16 number (2^-8), so the decode calls' bound holds."""
import pytest
import torch

from gpu_common import load_lib
from test_gpu_scores import check, make, reference

pytestmark = pytest.mark.gpu

SLOPES = [0.125, 0.25, 0.5, 2.0]


@pytest.mark.parametrize("cap", [0.0, 40.0])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("window", [0, 200, 256])
def test_steep_heads(cap, d, window):
    mx, _ = load_lib()
    heads = hq, hkv, d = 4, 2, d
    gen = torch.Generator("cuda").manual_seed(51)
    n, prefix = 900, 400
    q, k, v = (torch.randn(n, h, d, generator=gen, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    want, A, top = reference(q.double(), k.double(), v.double(), torch.arange(n, device="cuda"), cap, SLOPES, window)
    for direct in (True, False):
        ctx = make(mx, "prompt", window, heads, "bf16", 1, n, chunk=2000)
        ctx.set_chunk_ring_direct(direct)
        ctx.set_layer_scores(1, cap, SLOPES)
        out = torch.full_like(q, float("nan"))
        ctx.prefill(1, [0], [n], q, k, v, out)
        ctx.append_kv(0, [0], [prefix], k[:prefix].contiguous(), v[:prefix].contiguous())
        chunk = torch.full_like(q[prefix:], float("nan"))
        ctx.attend_chunk(1, [0], [n - prefix], q[prefix:].contiguous(), k[prefix:].contiguous(), v[prefix:].contiguous(), chunk)
        torch.cuda.synchronize()
        check(out, want, A, top, "bf16", d, "decode", n, "prompt")
        check(chunk, want[prefix:], A[prefix:], top, "bf16", d, "decode", n, "chunk")
        ctx.close()
