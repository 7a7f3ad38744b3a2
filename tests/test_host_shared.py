"""The tree of shared prefixes behind mixattn_decode_shared, on a host-only context: how many distinct
tokens a call reads, against a count over (page, place) pairs taken from the block tables."""
import random

import pytest

from paper_2409_15012_b200 import build

build.build()
from paper_2409_15012_b200 import binding as mx  # noqa: E402


def context(seqs, pages, longest, layout=None):
    return mx.Context(layout or [(mx.FULL, 0, 0), (mx.FULL, 0, 0)], 4, 2, 64, mx.BF16, seqs, pages, max_seq_len=longest)


def fewest(ctx, layer, ids):
    """Every token counted once, however many sequences share it."""
    seen = set()
    for s in ids:
        table, n = ctx.get_block_table(s), ctx.get_len(layer, s)
        seen |= {(table[t // 16], t % 16) for t in range(n)}
    return len(seen)


def test_forks_of_one_prompt():
    ctx = context(6, 200, 2000)
    ctx.append_kv(0, [0], [1000])
    ctx.fork_seqs([0] * 4, [1, 2, 3, 4])
    for s in range(5):
        ctx.append_kv(0, [s], [10 * s + 1])
    ids = [4, 2, 0, 1, 3]
    assert ctx.get_distinct_tokens(1, ids) == fewest(ctx, 1, ids) == 62 * 16 + sum(8 + 10 * s + 1 for s in range(5))
    assert ctx.get_distinct_tokens(0, [2]) == ctx.get_len(0, 2)
    assert ctx.get_distinct_tokens(0, []) == 0
    assert ctx.get_distinct_tokens(0, [2, 2, 2]) == ctx.get_len(0, 2)


@pytest.mark.parametrize("length", [1, 15, 16, 127, 128, 129, 143, 144, 160])
def test_pieces_shorter_than_the_least_are_read_by_each(length):
    ctx = context(3, 60, 400)
    ctx.append_kv(0, [0], [length])
    ctx.fork_seqs([0, 0], [1, 2])
    for s in range(3):
        ctx.append_kv(0, [s], [5])
    shared = length // 16 * 16
    want = shared + 3 * (length - shared + 5) if shared >= mx.MIN_SHARED_TOKENS else 3 * (length + 5)
    assert ctx.get_distinct_tokens(0, [0, 1, 2]) == want


def test_rings_share_nothing():
    ctx = context(3, 1, 4000, [(mx.SLIDING, 64, 0)])
    ctx.append_kv(0, [0], [1000])
    ctx.fork_seqs([0, 0], [1, 2])
    assert ctx.get_distinct_tokens(0, [0, 1, 2]) == 3 * 64


def test_random_histories():
    """Forks, appends and resets in any order: never fewer tokens than there are, and exactly those where
    every shared piece is long enough."""
    for seed in range(30):
        rng = random.Random(seed)
        ctx = context(8, 2000, 3000)
        long_pieces = seed % 2 == 0
        for _ in range(40):
            what = rng.random()
            if what < 0.5:
                s = rng.randrange(8)
                n = rng.choice([128, 160, 256]) if long_pieces else rng.randrange(1, 300)
                if ctx.get_len(0, s) + n <= 3000:
                    ctx.append_kv(0, [s], [n])
            elif what < 0.9:
                dst = rng.sample(range(8), rng.randrange(1, 6))
                ctx.fork_seqs([rng.randrange(8) for _ in dst], dst)
            else:
                ctx.seq_reset(rng.randrange(8))
        ids = [s for s in range(8) if ctx.get_len(0, s) > 0]
        rng.shuffle(ids)
        got, least, most = ctx.get_distinct_tokens(1, ids), fewest(ctx, 1, ids), sum(ctx.get_len(1, s) for s in ids)
        assert least <= got <= most
        if long_pieces:
            assert got == least
        else:
            assert got <= least + 16 * 8 * 128


def test_refusals():
    ctx = context(3, 60, 400)
    ctx.append_kv(0, [0], [20])
    for layer, ids, code in ((2, [0], mx.ERR_INVALID_ARG), (-1, [0], mx.ERR_INVALID_ARG), (0, [3], mx.ERR_BAD_SEQ), (0, [-1], mx.ERR_BAD_SEQ)):
        with pytest.raises(mx.MixAttnError) as e:
            ctx.get_distinct_tokens(layer, ids)
        assert e.value.code == code
    assert mx.lib.mixattn_get_distinct_tokens(ctx.h, 0, 0, None, None) == mx.ERR_INVALID_ARG
    assert mx.lib.mixattn_set_prefix_sharing(None, 1) == mx.ERR_INVALID_ARG
    assert mx.lib.mixattn_set_share_min_bytes(None, 0) == mx.ERR_INVALID_ARG
    assert ctx.rc_decode_shared(0, [0], None, None) == mx.ERR_INVALID_ARG
    assert mx.lib.mixattn_decode_shared(ctx.h, 0, 0, None, None, None, None) == mx.ERR_CUDA     # a host-only context launches nothing
