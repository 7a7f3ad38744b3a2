"""Prompt and chunk calls on a B200 whose neighbours are not finite: what the next sequence of the
call holds, what lies in front of a chunk, and what an earlier sequence left in a ring must not
reach a sequence's outputs.  They have to be the same bits as beside finite neighbours."""
import pytest
import torch

from gpu_common import load_lib
from test_gpu_scores import SHAPES, make, slopes_of

pytestmark = pytest.mark.gpu


def normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda").bfloat16()


def spoil(x):
    x[::2] = float("inf")
    x[1::2] = float("nan")


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("heads", [(4, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("window", [0, 50, 256])
def test_the_next_prompt_of_the_call(shape, heads, window):
    mx, _ = load_lib()
    hq, hkv, d = heads
    cap, biased = SHAPES[shape]
    lens = [200, 40, 1, 330, 128, 65]
    gen = torch.Generator("cuda").manual_seed(41)
    q, k, v = normal(gen, sum(lens), hq, d), normal(gen, sum(lens), hkv, d), normal(gen, sum(lens), hkv, d)
    outs = []
    for bad in (None, 1, 3, 5):
        kb, vb = k.clone(), v.clone()
        if bad is not None:
            r = slice(sum(lens[:bad]), sum(lens[:bad + 1]))
            spoil(kb[r])
            spoil(vb[r])
        ctx = make(mx, "prompt", window, heads, "bf16", len(lens), max(lens))
        ctx.set_layer_scores(1, cap, slopes_of(hq) if biased else None)
        out = torch.zeros_like(q)
        ctx.prefill(1, list(range(len(lens))), lens, q, kb, vb, out)
        torch.cuda.synchronize()
        assert ctx.get_device_status() == 0
        outs.append((bad, out))
        ctx.close()
    want = outs[0][1]
    assert torch.isfinite(want).all()
    for bad, out in outs[1:]:
        for i in range(len(lens)):
            r = slice(sum(lens[:i]), sum(lens[:i + 1]))
            assert i == bad or torch.equal(out[r], want[r]), (bad, i)


@pytest.mark.parametrize("direct", [True, False])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("window,d", [(0, 128), (128, 128), (384, 64), (200, 128)])
def test_the_other_chunks_of_the_call(direct, shape, window, d):
    mx, _ = load_lib()
    heads = hq, hkv, d = 4, 2, d
    cap, biased = SHAPES[shape]
    prefix, lens = [300, 77, 0, 513], [20, 130, 60, 90]
    gen = torch.Generator("cuda").manual_seed(42)
    kp, vp = ([normal(gen, n, hkv, d) for n in prefix] for _ in range(2))
    q, k, v = normal(gen, sum(lens), hq, d), normal(gen, sum(lens), hkv, d), normal(gen, sum(lens), hkv, d)
    outs = []
    for bad in (None, 0, 1, 2, 3):
        ctx = make(mx, "chunk", window, heads, "bf16", len(lens), 700, chunk=4096)
        ctx.set_chunk_ring_direct(direct)
        ctx.set_layer_scores(1, cap, slopes_of(hq) if biased else None)
        kb, vb = k.clone(), v.clone()
        for i, n in enumerate(prefix):
            pair = kp[i].clone(), vp[i].clone()
            if i == bad:
                r = slice(sum(lens[:i]), sum(lens[:i + 1]))
                for x in (*pair, kb[r], vb[r]):
                    spoil(x)
            if n:
                ctx.append_kv(0, [i], [n], *pair)
        out = torch.zeros_like(q)
        ctx.attend_chunk(1, list(range(len(lens))), lens, q, kb, vb, out)
        torch.cuda.synchronize()
        assert ctx.get_device_status() == 0
        outs.append((bad, out))
        ctx.close()
    want = outs[0][1]
    assert torch.isfinite(want).all()
    for bad, out in outs[1:]:
        for i in range(len(lens)):
            r = slice(sum(lens[:i]), sum(lens[:i + 1]))
            assert i == bad or torch.equal(out[r], want[r]), (bad, i)


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("window,d", [(128, 128), (256, 64)])
@pytest.mark.parametrize("prefix", [1, 70, 127, 128, 200])
def test_what_an_earlier_sequence_left_in_the_ring(shape, window, d, prefix):
    mx, _ = load_lib()
    heads = hq, hkv, d = 4, 2, d
    cap, biased = SHAPES[shape]
    gen = torch.Generator("cuda").manual_seed(43)
    kp, vp, k, v = (normal(gen, n, hkv, d) for n in (prefix, prefix, 50, 50))
    q = normal(gen, 50, hq, d)
    outs = []
    for stale in (False, True):
        ctx = make(mx, "chunk", window, heads, "bf16", 1, 700, chunk=4096)
        ctx.set_layer_scores(1, cap, slopes_of(hq) if biased else None)
        if stale:
            bad = torch.empty(window, hkv, d, device="cuda", dtype=torch.bfloat16)
            spoil(bad)
            ctx.append_kv(0, [0], [window], bad, bad)
            ctx.seq_reset(0)
        ctx.append_kv(0, [0], [prefix], kp, vp)
        out = torch.zeros_like(q)
        ctx.attend_chunk(1, [0], [50], q, k, v, out)
        torch.cuda.synchronize()
        outs.append(out)
        ctx.close()
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("window", [0, 50])
def test_the_next_prompt_in_fp32(shape, window):
    mx, _ = load_lib()
    heads = hq, hkv, d = 4, 2, 64
    cap, biased = SHAPES[shape]
    lens = [33, 40, 70]
    gen = torch.Generator("cuda").manual_seed(44)
    q, k, v = (normal(gen, sum(lens), h, d).float() for h in (hq, hkv, hkv))
    outs = []
    for bad in (False, True):
        kb, vb = k.clone(), v.clone()
        if bad:
            spoil(kb[33:73])
            spoil(vb[33:73])
        ctx = make(mx, "prompt", window, heads, "f32", len(lens), max(lens))
        ctx.set_layer_scores(1, cap, slopes_of(hq) if biased else None)
        out = torch.zeros_like(q)
        ctx.prefill(1, [0, 1, 2], lens, q, kb, vb, out)
        torch.cuda.synchronize()
        outs.append(out)
        ctx.close()
    assert torch.isfinite(outs[0]).all()
    assert torch.equal(outs[0][:33], outs[1][:33]) and torch.equal(outs[0][73:], outs[1][73:])
