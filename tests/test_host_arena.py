"""What a context asks for beside its caches: the split-KV workspace of the ordinary decode (1408 slots of a row per
query head) and a few small arrays; shared prefixes need more only where there are few query heads."""
import pytest

from paper_2409_15012_b200 import build as mbuild

mbuild.build()
from paper_2409_15012_b200 import binding as mx  # noqa: E402


def beside_the_cache(layer, hq, hkv, d, dtype, chunk=0, fp8=False):
    cfg, keep = mx.make_config([layer], hq, hkv, d, dtype, 4, 100, chunk_scratch_tokens=chunk, kv_format=mx.KV_FP8_E4M3 if fp8 else mx.KV_NATIVE)
    return mx.arena_bytes(cfg) - mx.cache_bytes(cfg)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq", [32, 40, 64, 71])
def test_contexts_of_many_heads_pay_nothing_for_sharing(hq, fp8):
    got = beside_the_cache((mx.FULL, 0, 0), hq, 1, 128, mx.BF16, fp8=fp8)
    assert got <= 1408 * hq * (128 * 4 + 8) + 64 * 1024
    assert abs(got - beside_the_cache((mx.FULL, 0, 0), hq, 1, 128, mx.F32)) < 512      # (the caches' alignment)


@pytest.mark.parametrize("hq,d", [(1, 128), (4, 64), (8, 128), (12, 128), (16, 64), (31, 128)])
def test_contexts_of_few_heads_pay_for_what_is_missing(hq, d):
    split = 1408 * hq * (d * 4 + 8)
    got = beside_the_cache((mx.FULL, 0, 0), hq, 1, d, mx.BF16)
    assert split < got <= split + 10.4e6
    for layer, dtype in (((mx.SLIDING, 64, 0), mx.BF16), ((mx.FULL, 0, 0), mx.F32)):     # nothing to share, or shared beside
        assert beside_the_cache(layer, hq, 1, d, dtype) <= split + 64 * 1024
    assert beside_the_cache((mx.FULL, 0, 0), hq, 1, d, mx.BF16, chunk=1000) == got + 2 * ((1000 * d * 2 + 255) // 256 * 256)
