"""Forked caches on a B200 away from the default stream: calls in order on one stream without a wait
between them, results allocated for the stream that writes them, and chunks over copies that have
grown apart."""
import pytest
import torch

from gpu_common import load_lib
from test_gpu_scores import check as check_scores
from test_gpu_scores import reference as attend_reference

pytestmark = pytest.mark.gpu

BUSY = 20_000_000      # cycles, about ten milliseconds


def filled(mx, seqs=5, n=300, **kw):
    ctx = mx.Context([(0, 0, 0), (1, 96, 1)], 4, 2, 128, mx.BF16, seqs, 200, max_seq_len=600, device=0, **kw)
    gen = torch.Generator("cuda").manual_seed(71)
    kv = [tuple(torch.randn(n, 2, 128, generator=gen, device="cuda").bfloat16() for _ in range(2)) for _ in (0, 1)]
    torch.cuda.synchronize()
    return ctx, kv


def test_append_fork_and_read_in_a_row_on_a_busy_stream():
    mx, _ = load_lib()
    ctx, kv = filled(mx)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(BUSY)                  # everything below is queued before any of it runs
        for o in (0, 1):
            ctx.append_kv(o, [0], [300], *kv[o], stream=stream)
        ctx.fork_seqs([0, 0, 0], [1, 2, 3], stream=stream)
        first = [ctx.read_kv(o, [3, 1], stream=stream) for o in (0, 1)]
        for o in (0, 1):
            ctx.append_kv(o, [1], [5], kv[o][0][:5].contiguous(), kv[o][1][:5].contiguous(), stream=stream)
        ctx.fork_seqs([1, 2], [2, 1], stream=stream)
        ctx.fork_seqs([2], [4], stream=stream)
        second = [ctx.read_kv(o, [4, 1, 2], stream=stream) for o in (0, 1)]
    stream.synchronize()
    for o, w in ((0, 600), (1, 96)):
        for i in (0, 1):
            x = kv[o][i]
            grown = torch.cat([x, x[:5]])[-w:]
            assert torch.equal(first[o][i], torch.cat([x[-w:]] * 2))
            assert torch.equal(second[o][i], torch.cat([grown, x[-w:], grown]))
    ctx.close()


@pytest.mark.parametrize("handle", [False, True])
def test_read_results_belong_to_the_stream_that_writes_them(handle):
    # the block of a tensor that was let go may still be written to on the stream it came from
    mx, _ = load_lib()
    ctx, kv = filled(mx)
    ctx.append_kv(0, [0], [300], *kv[0])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    torch.cuda.empty_cache()
    old = torch.empty(2, 300, 2, 128, dtype=torch.bfloat16, device="cuda")
    torch.cuda._sleep(BUSY)
    old.fill_(7)
    del old
    k, v = ctx.read_kv(0, [0], stream=stream.cuda_stream if handle else stream)
    torch.cuda.synchronize()
    assert torch.equal(k, kv[0][0]) and torch.equal(v, kv[0][1])
    ctx.close()


@pytest.mark.parametrize("handle", [False, True])
def test_selections_belong_to_the_stream_that_writes_them(handle):
    mx, _ = load_lib()
    ctx, _ = filled(mx)
    gen = torch.Generator("cuda").manual_seed(72)
    logits = torch.randn(8, 4, 1000, generator=gen, device="cuda")
    scores = torch.zeros(8, 4, device="cuda")
    want = ctx.beam_select(logits, scores, 64)
    torch.cuda.synchronize()
    want = [x.clone() for x in want]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    old = [torch.empty((3, 8, 64), dtype=torch.int32, device="cuda") for _ in range(32)]   # (whichever block comes next)
    torch.cuda._sleep(BUSY)
    for x in old:
        x.fill_(7)
    del old, x
    got = ctx.beam_select(logits, scores, 64, stream=stream.cuda_stream if handle else stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ctx.close()


def test_results_on_the_default_stream_while_another_is_current():
    mx, _ = load_lib()
    ctx, kv = filled(mx)
    ctx.append_kv(0, [0], [300], *kv[0])
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        old = torch.empty(2, 300, 2, 128, dtype=torch.bfloat16, device="cuda")
        torch.cuda._sleep(BUSY)
        old.fill_(7)
        del old
        k, v = ctx.read_kv(0, [0])
    torch.cuda.synchronize()
    assert torch.equal(k, kv[0][0]) and torch.equal(v, kv[0][1])
    ctx.close()


@pytest.mark.parametrize("direct", [True, False])
def test_chunks_over_copies_that_have_grown_apart(direct):
    mx, _ = load_lib()
    hq, hkv, d = 4, 2, 128
    ctx = mx.Context([(0, 0, 0), (1, 128, 1)], hq, hkv, d, mx.BF16, 4, 200, max_seq_len=600, device=0, chunk_scratch_tokens=4000)
    ctx.set_chunk_ring_direct(direct)
    gen = torch.Generator("cuda").manual_seed(73)
    kv = {}
    for o in (0, 1):
        k, v = (torch.randn(203, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
        ctx.append_kv(o, [2], [203], k, v)
        kv[o] = [(k, v)] * 4
    ctx.fork_seqs([2, 2, 2], [0, 1, 3])
    grow = [0, 1, 40, 150]                   # behind the shared pages, each copy's own tokens
    for o in (0, 1):
        for s, n in enumerate(grow):
            if n:
                k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
                ctx.append_kv(o, [s], [n], k, v)
                kv[o][s] = (torch.cat([kv[o][s][0], k]), torch.cat([kv[o][s][1], v]))
    lens = [33, 1, 140, 60]
    q = torch.randn(sum(lens), hq, d, generator=gen, device="cuda").bfloat16()
    k, v = (torch.randn(sum(lens), hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    for o in (0, 1):
        out = torch.empty_like(q)
        ctx.attend_chunk(o, [0, 1, 2, 3], lens, q, k, v, out)
        torch.cuda.synchronize()
        for s in range(4):
            r = slice(sum(lens[:s]), sum(lens[:s + 1]))
            K, V = torch.cat([kv[o][s][0], k[r]]), torch.cat([kv[o][s][1], v[r]])
            want, A, top = attend_reference(q[r].double(), K.double(), V.double(), torch.arange(len(K) - lens[s], len(K), device="cuda"),
                                            0.0, None, 128 if o else 0)
            check_scores(out[r], want, A, top, "bf16", d, "prompt", len(K), f"layer {o} copy {s}")
    ctx.close()
