"""Forking and reordering of sequences on host-only contexts: lengths, block tables, shared and
fresh pages and the order of the free FIFO against a plain model; refusals of the new calls."""
from collections import Counter, deque

import numpy as np
import pytest

from synth import configs as cf
from paper_2409_15012_b200 import build as mbuild

mbuild.build()
from paper_2409_15012_b200 import binding as mx  # noqa: E402

PAGE = 16


class Model:
    """Block tables per sequence, reference counts from the tables themselves, a FIFO of free pages."""

    def __init__(self, layout, seqs, pages):
        self.layout = layout
        self.owners = [l for l, (_, _, o) in enumerate(layout) if o == l]
        self.len = {o: [0] * seqs for o in self.owners}
        self.table = [[] for _ in range(seqs)]
        self.free = deque(range(pages))

    def release(self, pages, held):
        for p in pages:
            held[p] -= 1
            if held[p] == 0:
                self.free.append(p)

    def held(self):
        return Counter(p for t in self.table for p in t)

    def reset(self, s):
        self.release(self.table[s], self.held())
        self.table[s] = []
        for o in self.owners:
            self.len[o][s] = 0

    def append(self, o, ids, n_new):
        need = sum(max(0, -(-(self.len[o][s] + n) // PAGE) - len(self.table[s]))
                   for s, n in zip(ids, n_new)) if self.layout[o][0] == mx.FULL else 0
        if need > len(self.free):
            return mx.ERR_OUT_OF_PAGES
        for s, n in zip(ids, n_new):
            self.len[o][s] += n
            while self.layout[o][0] == mx.FULL and len(self.table[s]) * PAGE < self.len[o][s]:
                self.table[s].append(self.free.popleft())
        return 0

    def fork(self, src, dst):
        replaced = {d for s, d in zip(src, dst) if s != d}
        heir = {}      # an overwritten source hands over to its first copy
        for s, d in zip(src, dst):
            if s in replaced and s not in heir:
                heir[s] = d
        copies = [(s, d) for s, d in zip(src, dst) if s != d and heir.get(s) != d]
        old_t = [list(t) for t in self.table]
        old_n = {o: list(v) for o, v in self.len.items()}
        full = [o for o in self.owners if self.layout[o][0] == mx.FULL]
        shared = [min([old_n[o][s] // PAGE for o in full] + [len(old_t[s])]) for s in range(len(old_t))]
        held = self.held()
        for s, _ in copies:
            for p in old_t[s][:shared[s]]:
                held[p] += 1
        after, freed = held.copy(), 0
        dead = [d for _, d in zip(src, dst) if d in replaced and d not in heir]
        for d in dead:
            for p in old_t[d]:
                after[p] -= 1
                freed += after[p] == 0
        if sum(len(old_t[s]) - shared[s] for s, _ in copies) > len(self.free) + freed:
            return mx.ERR_OUT_OF_PAGES
        for d in dead:
            self.release(old_t[d], held)
        for s, d in zip(src, dst):
            if s != d and heir.get(s) == d:
                self.table[d] = old_t[s]
            elif s != d:
                self.table[d] = old_t[s][:shared[s]] + [self.free.popleft() for _ in old_t[s][shared[s]:]]
            for o in self.owners:
                self.len[o][d] = old_n[o][s]
        return 0


def same(ctx, m):
    assert ctx.get_n_free_pages() == len(m.free)
    for s in range(len(m.table)):
        assert ctx.get_block_table(s) == m.table[s], s
        for l, (kind, w, o) in enumerate(m.layout):
            n = m.len[o][s]
            assert ctx.get_len(l, s) == n
            if kind == mx.SLIDING:
                assert ctx.get_ring_state(l, s) == (n % w, min(n, w))
            elif n:
                assert ctx.locate(l, s, n - 1) == (m.table[s][(n - 1) // PAGE], (n - 1) % PAGE)


LAYOUTS = {
    "tiny": cf.layout_tiny(5),
    "rings_only": [(1, 7, 0), (1, 3, 1), (1, 7, 0)],
    "two_full": [(0, 0, 0), (0, 0, 1), (1, 3, 2), (0, 0, 1)],
}


@pytest.mark.parametrize("name", sorted(LAYOUTS))
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_random_forks_match_the_model(name, seed):
    layout = LAYOUTS[name]
    seqs, pages = 7, 18
    rng = np.random.default_rng(seed)
    ctx = mx.Context(layout, 4, 2, 64, mx.F32, seqs, pages, max_seq_len=100000, device=-1)
    m = Model(layout, seqs, pages)
    refused = 0
    for _ in range(300):
        op = rng.integers(0, 10)
        if op == 0:
            s = int(rng.integers(0, seqs))
            ctx.seq_reset(s)
            m.reset(s)
        elif op < 5:
            ids = rng.permutation(seqs)[: rng.integers(1, seqs + 1)].tolist()
            n_new = rng.integers(0, 30, size=len(ids)).tolist()
            for o in m.owners[: rng.integers(1, len(m.owners) + 1)]:   # (owners may lag behind one another)
                assert ctx.rc_append_kv(o, ids, n_new) == m.append(o, ids, n_new)
        else:
            n = int(rng.integers(0, seqs + 1))
            dst = rng.permutation(seqs)[:n].tolist()
            src = rng.integers(0, seqs, size=n).tolist()
            rc, want = ctx.rc_fork_seqs(src, dst), m.fork(src, dst)
            assert rc == want
            refused += rc != 0
        same(ctx, m)
    assert name != "two_full" or refused > 0
    ctx.close()


def test_reordering_a_group_moves_no_page():
    ctx = mx.Context([(0, 0, 0)], 4, 2, 64, mx.F32, 4, 40, device=-1)
    for s in range(4):
        ctx.append_kv(0, [s], [20 + s])
    before = [ctx.get_block_table(s) for s in range(4)]
    free = ctx.get_n_free_pages()
    ctx.fork_seqs([3, 0, 1, 2], [0, 1, 2, 3])
    assert [ctx.get_block_table(s) for s in range(4)] == [before[3], before[0], before[1], before[2]]
    assert [ctx.get_len(0, s) for s in range(4)] == [23, 20, 21, 22]
    assert ctx.get_n_free_pages() == free
    ctx.close()


def test_a_shared_page_is_free_when_its_last_holder_lets_go():
    ctx = mx.Context([(0, 0, 0)], 4, 2, 64, mx.F32, 4, 10, device=-1)
    ctx.append_kv(0, [0], [48])
    ctx.fork_seqs([0, 0], [1, 2])
    assert ctx.get_n_free_pages() == 7       # three full pages, shared by all
    ctx.seq_reset(0)
    ctx.seq_reset(2)
    assert ctx.get_n_free_pages() == 7
    ctx.append_kv(0, [1], [1])
    assert ctx.get_n_free_pages() == 6
    ctx.seq_reset(1)
    assert ctx.get_n_free_pages() == 10
    ctx.close()


def test_fork_refusals_change_nothing():
    ctx = mx.Context([(0, 0, 0), (1, 5, 1)], 4, 2, 64, mx.F32, 4, 3, device=-1)
    ctx.append_kv(0, [0], [33])
    assert ctx.rc_fork_seqs([0], [4]) == mx.ERR_BAD_SEQ
    assert ctx.rc_fork_seqs([-1], [1]) == mx.ERR_BAD_SEQ
    assert ctx.rc_fork_seqs([0, 0], [1, 1]) == mx.ERR_INVALID_ARG
    assert ctx.rc_fork_seqs([0, 0], [1]) == mx.ERR_INVALID_ARG
    assert mx.lib.mixattn_fork_seqs(ctx.h, 1, None, None, None) == mx.ERR_INVALID_ARG
    assert mx.lib.mixattn_fork_seqs(ctx.h, -1, None, None, None) == mx.ERR_INVALID_ARG
    assert mx.lib.mixattn_fork_seqs(None, 0, None, None, None) == mx.ERR_INVALID_ARG
    assert ctx.rc_fork_seqs([0], [1]) == mx.ERR_OUT_OF_PAGES       # the partly filled page has no room for a copy
    assert ctx.get_len(0, 1) == 0 and ctx.get_block_table(0) == [0, 1, 2] and ctx.get_n_free_pages() == 0
    assert ctx.rc_fork_seqs([], []) == 0
    ctx.fork_seqs([0, 1], [0, 2])                                  # itself, and an empty one
    assert ctx.get_block_table(0) == [0, 1, 2] and ctx.get_len(0, 2) == 0
    ctx.fork_seqs([0, 1], [1, 0])                                  # swapped without a free page
    assert ctx.get_block_table(1) == [0, 1, 2] and ctx.get_len(0, 0) == 0
    ctx.close()


def test_read_kv_refusals():
    ctx = mx.Context([(0, 0, 0), (1, 5, 1)], 4, 2, 64, mx.F32, 2, 10, device=-1)
    for o in (0, 1):
        ctx.append_kv(o, [0], [33])

    def rc(layer, ids, first, n):
        a = [None if x is None else mx._i32(x) for x in (ids, first, n)]
        return mx.lib.mixattn_read_kv(ctx.h, layer, len(ids), *[mx._p32(x) for x in a], None, None, None)

    assert rc(2, [0], None, None) == mx.ERR_INVALID_ARG
    assert rc(0, [2], None, None) == mx.ERR_BAD_SEQ
    assert rc(0, [0], [-1], [1]) == mx.ERR_INVALID_ARG
    assert rc(0, [0], [30], [4]) == mx.ERR_INVALID_ARG
    assert rc(0, [0], [34], None) == mx.ERR_INVALID_ARG
    assert rc(0, [0], [3], [-1]) == mx.ERR_INVALID_ARG
    assert rc(0, [0], [2147483647], [2147483647]) == mx.ERR_INVALID_ARG
    assert rc(1, [0], [27], [1]) == mx.ERR_INVALID_ARG             # fell out of the window
    with pytest.raises(mx.MixAttnError):
        ctx.read_kv(0, [0, 1], [0])
    assert list(ctx.get_stored(0, [0, 1])) == [33, 0] and list(ctx.get_stored(1, [0, 1])) == [5, 0]
    with pytest.raises(mx.MixAttnError):
        ctx.get_stored(0, [2])
    assert rc(1, [0], [28], [5]) == mx.ERR_CUDA                    # in order, but there is no device
    assert rc(0, [0], None, None) == mx.ERR_CUDA
    ctx.close()


def test_layer_scores_refusals():
    ctx = mx.Context([(0, 0, 0), (0, 0, 0)], 4, 2, 64, mx.F32, 2, 10, device=-1)
    for cap in (-1.0, float("nan"), float("inf"), 1e-9, 1e9):
        assert ctx.rc_set_layer_scores(0, cap) == mx.ERR_INVALID_ARG
    for bad in (-1e-3, float("nan"), float("inf"), 2000.0):
        assert ctx.rc_set_layer_scores(0, 0.0, [0.5, bad, 0.5, 0.5]) == mx.ERR_INVALID_ARG
    assert ctx.rc_set_layer_scores(0, 0.0, [0.5]) == mx.ERR_INVALID_ARG
    assert ctx.rc_set_layer_scores(2, 30.0) == mx.ERR_INVALID_ARG
    assert ctx.rc_set_layer_scores(-1, 30.0) == mx.ERR_INVALID_ARG
    assert mx.lib.mixattn_set_layer_scores(None, 0, 0.0, None) == mx.ERR_INVALID_ARG
    assert ctx.rc_set_layer_scores(1, 30.0, [0.0, 0.5, 1.0, 1024.0]) == 0
    assert ctx.rc_set_layer_scores(1) == 0
    ctx.close()
    steep = mx.Context([(0, 0, 0)], 4, 2, 64, mx.F32, 1, 10, device=-1, softmax_scale=3e38)
    assert steep.rc_set_layer_scores(0, 1e-3) == mx.ERR_INVALID_ARG
    steep.close()
    wide = mx.Context([(0, 0, 0)], 130, 2, 64, mx.F32, 1, 10, device=-1)
    assert wide.rc_set_layer_scores(0, 0.0, [0.5] * 130) == mx.ERR_UNSUPPORTED
    assert wide.rc_set_layer_scores(0, 50.0) == 0                   # a cap alone has no such limit
    wide.close()


def test_beam_select_refusals():
    ctx = mx.Context([(0, 0, 0)], 4, 2, 64, mx.F32, 1, 10, device=-1)
    p = 4096      # never read: the call is refused first

    def rc(groups=1, beams=2, vocab=100, dtype=mx.BF16, logits=p, stride=100, scores=p, finished=None, eos=0, n_out=4):
        return mx.lib.mixattn_beam_select(ctx.h, groups, beams, vocab, dtype, logits, stride, scores, finished, eos, n_out,
                                          p, p, p, None)

    for kw in (dict(groups=-1), dict(beams=0), dict(beams=65), dict(vocab=0), dict(n_out=0), dict(n_out=65), dict(dtype=2),
               dict(stride=99), dict(vocab=2 ** 31 - 1, stride=2 ** 31), dict(finished=p, eos=100), dict(finished=p, eos=-1),
               dict(groups=2 ** 31 - 1, beams=2), dict(stride=2 ** 62), dict(vocab=2 ** 30 + 1, stride=2 ** 31, beams=1)):
        assert rc(**kw) == mx.ERR_INVALID_ARG, kw
    assert rc() == mx.ERR_CUDA                # in order, but there is no device
    assert rc(finished=p, eos=99) == mx.ERR_CUDA
    ctx.close()
