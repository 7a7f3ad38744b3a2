"""Decode of shaped scores over a quantised cache on a B200: what an earlier sequence left behind the
last token (NaN codes, which E4M3 has, and the largest values that infinities are stored as) does
not matter.  The clearing goes by groups of four keys, so every length modulo 16 is there."""
import pytest
import torch

from gpu_common import load_lib
from test_gpu_scores import check, make, on_e4m3, reference, slopes_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [0, 64])
@pytest.mark.parametrize("cap,biased", [(30.0, True), (30.0, False), (0.0, True)])
def test_rows_behind_a_quantised_sequence_do_not_matter(window, cap, biased):
    mx, _ = load_lib()
    heads = hq, hkv, d = 4, 2, 128
    lens = list(range(17, 34)) + [1, 2, 3, 48, 63]
    gen = torch.Generator("cuda").manual_seed(61)
    ctx = make(mx, "decode", window, heads, "fp8", len(lens), 64)
    ids = list(range(len(lens)))
    bad = torch.randn(len(lens) * 64, hkv, d, generator=gen, device="cuda").bfloat16()
    bad[::2] = float("nan")
    bad[1::4, :, ::3] = float("inf")
    ctx.append_kv(0, ids, [64] * len(lens), bad, bad)
    for i in ids:
        ctx.seq_reset(i)
    K, V = [], []
    for i, n in enumerate(lens):
        k, v = (on_e4m3(torch.randn(n, hkv, d, generator=gen, device="cuda").bfloat16()) for _ in range(2))
        ctx.append_kv(0, [i], [n], k, v)
        K.append(k)
        V.append(v)
    slopes = slopes_of(hq) if biased else None
    ctx.set_layer_scores(1, cap, slopes)
    q = torch.randn(len(lens), hq, d, generator=gen, device="cuda").bfloat16()
    out = torch.empty_like(q)
    ctx.decode(1, ids, q, out)
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        want, A, top = reference(q[i:i + 1].double(), K[i].double(), V[i].double(), torch.tensor([n - 1], device="cuda"), cap, slopes,
                                 window)
        check(out[i:i + 1], want, A, top, "fp8", d, "fp8", n, f"length {n}")
    ctx.close()
