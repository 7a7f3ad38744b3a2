"""Host integers handed to the binding: one entry per sequence, whole numbers, nothing dropped."""
import numpy as np
import pytest

from paper_2409_15012_b200 import build as mbuild

mbuild.build()
from paper_2409_15012_b200 import binding as mx  # noqa: E402


def context():
    ctx = mx.Context([(mx.FULL, 0, 0), (mx.FULL, 0, 0)], 4, 2, 64, mx.F32, 6, 40, device=-1)
    ctx.append_kv(0, [0], [20])
    return ctx


@pytest.mark.parametrize("src,dst", [
    (np.zeros((2, 2), dtype=np.int64), np.array([[0, 1], [2, 3]])),   # parents as [groups, beams]: flatten them first
    ([[0, 0]], [[1, 2]]), ([0], [0.7]), ([0], np.array([1.5])), ([0], np.array([2 ** 32 + 4])), (None, None), ([0], None)])
def test_what_is_not_one_whole_number_per_sequence_is_refused(src, dst):
    ctx = context()
    for call in (ctx.rc_fork_seqs, ctx.fork_seqs):
        with pytest.raises(mx.MixAttnError) as e:
            call(src, dst)
        assert e.value.code == mx.ERR_INVALID_ARG
    assert [ctx.get_len(0, s) for s in range(6)] == [20, 0, 0, 0, 0, 0]
    ctx.close()


@pytest.mark.parametrize("dst", [[1, 2], (1, 2), np.array([1, 2]), np.array([9, 1, 9, 2])[1::2], np.array([1, 2], dtype=np.uint8),
                                 [np.int64(1), np.int64(2)], [1.0, 2.0]])
def test_what_is_taken(dst):
    ctx = context()
    ctx.fork_seqs([0, 0], dst)
    assert [ctx.get_len(0, s) for s in range(6)] == [20, 20, 20, 0, 0, 0]
    ctx.fork_seqs([], np.zeros(0))
    ctx.close()


def test_sequences_have_to_be_given():
    ctx = context()
    for call in (lambda: ctx.rc_decode(1, None, None, None), lambda: ctx.read_kv(0, None), lambda: ctx.get_stored(0, None),
                 lambda: ctx.rc_prefill(1, [0], None, None, None, None, None),
                 lambda: ctx.rc_attend_chunk(1, None, [1], None, None, None, None)):
        with pytest.raises(mx.MixAttnError) as e:
            call()
        assert e.value.code == mx.ERR_INVALID_ARG
    ctx.close()


def test_lengths_have_to_match_the_sequences():
    ctx = context()
    for lens in ([5], [5, 6, 7]):       # (a shorter list would be read past its end)
        assert ctx.rc_prefill(1, [0, 1], lens, None, None, None, None) == mx.ERR_INVALID_ARG
        assert ctx.rc_attend_chunk(1, [0, 1], lens, None, None, None, None) == mx.ERR_INVALID_ARG
        assert ctx.rc_append_kv(0, [0, 1], lens, None, None) == mx.ERR_INVALID_ARG
        assert ctx.rc_append_kv_rope(0, [0, 1], lens, None, None, 1e4) == mx.ERR_INVALID_ARG
    assert ctx.get_len(0, 0) == 20
    ctx.close()
