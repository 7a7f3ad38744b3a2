"""Host numbers that do not fit 32 bits are refused as every other bad argument is, by every call that takes sequences."""
import numpy as np
import pytest

from paper_2409_15012_b200 import build as mbuild

mbuild.build()
from paper_2409_15012_b200 import binding as mx  # noqa: E402


@pytest.mark.parametrize("big", [2 ** 31, -2 ** 31 - 1, 2 ** 40, 10 ** 30])
def test_numbers_beyond_32_bits(big):
    ctx = mx.Context([(mx.FULL, 0, 0), (mx.FULL, 0, 0)], 4, 2, 64, mx.F32, 6, 40, device=-1)
    ctx.append_kv(0, [0], [20])
    rope = mx.Rope(64)
    calls = [lambda: ctx.fork_seqs([0], [big]), lambda: ctx.fork_seqs([big], [1]), lambda: ctx.rc_decode(1, [big], None, None),
             lambda: ctx.rc_decode_shared(1, [0, big], None, None), lambda: ctx.decode_shared(1, (big,), None, None),
             lambda: ctx.get_distinct_tokens(0, [big]), lambda: ctx.get_stored(0, [big]), lambda: ctx.read_kv(0, [0], [big], [1]),
             lambda: ctx.rope_qkv(0, [big], None, rope, store=True), lambda: ctx.rope_qkv(0, [0], [big], rope, store=True),
             lambda: ctx.rope_qkv(0, [0], None, rope, store=True, first_pos=[big]), lambda: ctx.append_kv(0, [1], [big]),
             lambda: ctx.rc_prefill(1, [0], [big], None, None, None, None), lambda: ctx.rc_attend_chunk(1, [0], [big], None, None, None, None)]
    for i, call in enumerate(calls):
        with pytest.raises(mx.MixAttnError) as e:
            call()
        assert e.value.code == mx.ERR_INVALID_ARG, i
    assert [ctx.get_len(0, s) for s in range(6)] == [20, 0, 0, 0, 0, 0]
    ctx.close()


@pytest.mark.parametrize("wide", [2 ** 32, 2 ** 31, -2 ** 32 + 1])
def test_wide_arrays_do_not_wrap(wide):
    ctx = mx.Context([(mx.FULL, 0, 0), (mx.FULL, 0, 0)], 4, 2, 64, mx.F32, 6, 40, device=-1)
    at, one = np.array([wide]), np.array([1], dtype=np.int64)
    for call in (lambda: ctx.append_kv(0, at, one), lambda: ctx.append_kv(0, one, at), lambda: ctx.rc_decode(1, at, None, None),
                 lambda: ctx.rc_decode_shared(1, at, None, None), lambda: ctx.get_distinct_tokens(0, at),
                 lambda: ctx.append_kv_rope(0, at, one, None, None, 1e4)):
        with pytest.raises(mx.MixAttnError) as e:
            call()
        assert e.value.code == mx.ERR_INVALID_ARG
    ctx.append_kv(0, one, one)
    assert [ctx.get_len(0, s) for s in range(3)] == [0, 1, 0]
    ctx.close()
