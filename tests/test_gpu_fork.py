"""Forking, reordering and reading cached sequences on a B200: contents against plain lists of the
tokens, attention over copies, and a run of selection, reordering, append and attention together."""
import numpy as np
import pytest
import torch

from gpu_common import load_lib
from test_gpu_beam import reference as select_reference
from test_gpu_scores import check as check_scores
from test_gpu_scores import on_e4m3, reference as attend_reference, slopes_of

pytestmark = pytest.mark.gpu

LAYOUTS = {
    "mixed": [(0, 0, 0), (1, 40, 1), (0, 0, 0), (1, 40, 1), (1, 64, 4), (0, 0, 5)],
    "rings": [(1, 7, 0), (1, 130, 1)],
    "paged": [(0, 0, 0)],
}


def same_contents(ctx, layout, model):
    for o in model:
        kind, window, _ = layout[o]
        seqs = list(range(len(model[o])))
        keep = [m[-window:] if kind == 1 else m for m in model[o]]
        k, v = ctx.read_kv(o, seqs)
        torch.cuda.synchronize()
        want = torch.cat([torch.stack([t[0] for t in m]) for m in keep if m]) if any(keep) else k[:0]
        assert torch.equal(k, want)
        want = torch.cat([torch.stack([t[1] for t in m]) for m in keep if m]) if any(keep) else v[:0]
        assert torch.equal(v, want)


@pytest.mark.parametrize("name", sorted(LAYOUTS))
@pytest.mark.parametrize("dtype,heads", [("bf16", (4, 2, 128)), ("bf16", (3, 3, 64)), ("f32", (4, 2, 64)), ("f32", (2, 1, 128)),
                                         ("fp8", (4, 2, 128))])
def test_random_forks_keep_contents(name, dtype, heads):
    mx, _ = load_lib()
    layout = LAYOUTS[name]
    hq, hkv, d = heads
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    seqs = 6
    ctx = mx.Context(layout, hq, hkv, d, mx.F32 if dtype == "f32" else mx.BF16, seqs, 200, max_seq_len=2000, device=0,
                     kv_format=mx.KV_FP8_E4M3 if dtype == "fp8" else mx.KV_NATIVE)
    owners = [l for l, (_, _, o) in enumerate(layout) if o == l]
    model = {o: [[] for _ in range(seqs)] for o in owners}
    gen = torch.Generator("cuda").manual_seed(21)
    rng = np.random.default_rng(5)
    for step in range(60):
        op = rng.integers(0, 10)
        if op == 0:
            s = int(rng.integers(0, seqs))
            ctx.seq_reset(s)
            for o in owners:
                model[o][s] = []
        elif op < 5:
            ids = rng.permutation(seqs)[: rng.integers(1, seqs + 1)].tolist()
            n_new = rng.integers(0, 60, size=len(ids)).tolist() if op < 4 else [1] * len(ids)
            for o in owners[: rng.integers(1, len(owners) + 1)]:
                k, v = (torch.randn(sum(n_new), hkv, d, generator=gen, device="cuda").to(dt) for _ in range(2))
                if dtype == "fp8":
                    k, v = on_e4m3(k), on_e4m3(v)
                if ctx.rc_append_kv(o, ids, None if op == 4 else n_new, k, v) != 0:
                    continue
                row = 0
                for s, n in zip(ids, n_new):
                    model[o][s] += list(zip(k[row:row + n], v[row:row + n]))
                    row += n
        else:
            n = int(rng.integers(1, seqs + 1))
            dst = rng.permutation(seqs)[:n].tolist()
            src = rng.integers(0, seqs, size=n).tolist()
            if ctx.rc_fork_seqs(src, dst) == 0:
                for o in owners:
                    old = [list(m) for m in model[o]]
                    for s, t in zip(src, dst):
                        model[o][t] = list(old[s])
        same_contents(ctx, layout, model)
    assert ctx.get_device_status() == 0
    ctx.close()


def test_many_copies_in_one_call():
    # more copies, owners and partly filled pages than one launch takes
    mx, _ = load_lib()
    layout = [(0, 0, 0), (1, 33, 1), (0, 0, 2), (1, 20, 3)]
    seqs = 150
    ctx = mx.Context(layout, 2, 1, 64, mx.BF16, seqs, 4000, max_seq_len=400, device=0)
    model = {o: [[] for _ in range(seqs)] for o in range(4)}
    gen = torch.Generator("cuda").manual_seed(22)
    for o, n in ((0, 130), (1, 50), (2, 5), (3, 19)):     # owner 2 lags: nine pages per copy are not shared
        k, v = (torch.randn(n, 1, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
        ctx.append_kv(o, [149], [n], k, v)
        model[o][149] = list(zip(k, v))
    ctx.fork_seqs([149] * 149, list(range(149)))
    for o in model:
        model[o] = [list(model[o][149]) for _ in range(seqs)]
    same_contents(ctx, layout, model)
    ctx.close()


def test_copies_grow_apart_and_attend_to_their_own_tokens():
    mx, _ = load_lib()
    layout = [(0, 0, 0), (1, 128, 1)]
    hq, hkv, d = 8, 2, 128
    ctx = mx.Context(layout, hq, hkv, d, mx.BF16, 8, 200, max_seq_len=600, device=0)
    gen = torch.Generator("cuda").manual_seed(23)
    kv = {}
    for o in (0, 1):
        k, v = (torch.randn(309, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
        ctx.append_kv(o, [3], [309], k, v)
        kv[o] = [(k, v)] * 8
    ctx.fork_seqs([3] * 7, [0, 1, 2, 4, 5, 6, 7])
    for step in range(20):
        for o in (0, 1):
            k, v = (torch.randn(8, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
            ctx.append_kv(o, list(range(8)), None, k, v)
            kv[o] = [(torch.cat([a, k[i:i + 1]]), torch.cat([b, v[i:i + 1]])) for i, (a, b) in enumerate(kv[o])]
        if step == 9:
            ctx.fork_seqs([5, 5, 0, 7], [0, 1, 7, 5])
            for o in (0, 1):
                old = list(kv[o])
                for s, t in ((5, 0), (5, 1), (0, 7), (7, 5)):
                    kv[o][t] = old[s]
    for o in (0, 1):
        q = torch.randn(8, hq, d, generator=gen, device="cuda").bfloat16()
        out = torch.empty_like(q)
        ctx.decode(o, list(range(8)), q, out)
        torch.cuda.synchronize()
        for i in range(8):
            K, V = kv[o][i]
            want, A, top = attend_reference(q[i:i + 1].double(), K.double(), V.double(),
                                            torch.tensor([len(K) - 1], device="cuda"), 0.0, None, layout[o][1])
            check_scores(out[i:i + 1], want, A, top, "bf16", d, "decode", len(K), f"layer {o} copy {i}")
    # a chunk behind the copies, rings read in place and copied
    ctx.close()


@pytest.mark.parametrize("direct", [True, False])
def test_chunks_behind_reordered_sequences(direct):
    mx, _ = load_lib()
    hq, hkv, d = 4, 2, 128
    ctx = mx.Context([(0, 0, 0), (1, 128, 1)], hq, hkv, d, mx.BF16, 3, 100, max_seq_len=600, device=0, chunk_scratch_tokens=2000)
    ctx.set_chunk_ring_direct(direct)
    ctx.set_chunk_gather_reuse(True)
    gen = torch.Generator("cuda").manual_seed(24)
    lens = [200, 150, 77]
    kv = {o: [tuple(torch.randn(n, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2)) for n in lens] for o in (0, 1)}
    for o in (0, 1):
        for s in range(3):
            ctx.append_kv(o, [s], [lens[s]], *kv[o][s])
    q = torch.randn(3 * 20, hq, d, generator=gen, device="cuda").bfloat16()
    k, v = (torch.randn(3 * 20, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    for src in ([0, 1, 2], [2, 0, 1], [0, 0, 2]):     # (the second call must not reuse the first one's copied keys)
        ctx.fork_seqs(src, [0, 1, 2])
        for o in (0, 1):
            kv[o] = [kv[o][s] for s in src]
            out = torch.empty_like(q)
            ctx.attend_chunk(o, [0, 1, 2], [20] * 3, q, k, v, out)
            torch.cuda.synchronize()
            for s in range(3):
                r = slice(20 * s, 20 * s + 20)
                K, V = torch.cat([kv[o][s][0], k[r]]), torch.cat([kv[o][s][1], v[r]])
                want, A, top = attend_reference(q[r].double(), K.double(), V.double(),
                                                torch.arange(len(K) - 20, len(K), device="cuda"), 0.0, None, 128 if o else 0)
                check_scores(out[r], want, A, top, "bf16", d, "prompt", len(K), f"layer {o} sequence {s}")
    ctx.close()


def test_ranges_and_debug_reads():
    mx, _ = load_lib()
    ctx = mx.Context([(0, 0, 0), (1, 50, 1)], 4, 2, 64, mx.BF16, 4, 100, max_seq_len=600, device=0)
    gen = torch.Generator("cuda").manual_seed(25)
    kv = {o: tuple(torch.randn(119, 2, 64, generator=gen, device="cuda").bfloat16() for _ in range(2)) for o in (0, 1)}
    for o in (0, 1):
        ctx.append_kv(o, [0], [119], *kv[o])
    ctx.fork_seqs([0, 0], [2, 3])
    for o in (0, 1):
        k, v = ctx.read_kv(o, [2, 0, 2, 1], [70, 100, 119, 0], [49, 3, 0, 0])
        torch.cuda.synchronize()
        for got, src in ((k, kv[o][0]), (v, kv[o][1])):
            assert torch.equal(got, torch.cat([src[70:119], src[100:103]]))
        a, b = ctx.debug_read_kv(o, 3, 117)
        assert torch.equal(a, kv[o][0][117].cpu()) and torch.equal(b, kv[o][1][117].cpu())
    with pytest.raises(mx.MixAttnError):
        ctx.read_kv(1, [2], [68], [3])
    ctx.close()


def test_beam_search_over_the_cache():
    """Selection, reordering, append and capped attention together: every step is checked against
    the definition over plain per-hypothesis lists of the tokens' keys and values."""
    mx, _ = load_lib()
    hq, hkv, d, vocab, groups, beams = 4, 2, 64, 501, 2, 3
    layout = [(0, 0, 0), (1, 32, 1)]
    seqs = groups * beams
    ctx = mx.Context(layout, hq, hkv, d, mx.F32, seqs, 200, max_seq_len=300, device=0)
    slopes = slopes_of(hq)
    for l in (0, 1):
        ctx.set_layer_scores(l, 15.0, slopes)
    gen = torch.Generator("cuda").manual_seed(26)
    # a model of one linear map: token -> (q, k, v) per layer, attention outputs -> logits
    emb = torch.randn(2, vocab, (hq + 2 * hkv) * d, generator=gen, device="cuda")
    head = torch.randn(2 * hq * d, vocab, generator=gen, device="cuda") * 0.2

    def qkv(o, tokens):
        x = emb[o][tokens].view(-1, hq + 2 * hkv, d)
        return [t.contiguous() for t in (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:])]

    prompts = [torch.randint(0, vocab, (n,), generator=gen, device="cuda") for n in (45, 70)]
    hyp = [[] for _ in range(seqs)]
    for g, p in enumerate(prompts):
        hyp[g * beams] = p.tolist()
        for o in (0, 1):
            _, k, v = qkv(o, p[:-1])
            ctx.append_kv(o, [g * beams], [len(p) - 1], k, v)
    ctx.fork_seqs([g * beams for g in range(groups) for _ in range(beams - 1)],
                  [g * beams + b for g in range(groups) for b in range(1, beams)])
    hyp = [list(hyp[s // beams * beams]) for s in range(seqs)]
    scores = torch.full((groups, beams), float("-inf"), device="cuda")
    scores[:, 0] = 0
    finished = torch.zeros(groups, beams, dtype=torch.uint8, device="cuda")
    eos = 7
    for step in range(30):
        tokens = torch.tensor([h[-1] for h in hyp], device="cuda")
        outs = []
        for o in (0, 1):
            q, k, v = qkv(o, tokens)
            ctx.append_kv(o, list(range(seqs)), None, k, v)
            out = torch.empty_like(q)
            ctx.decode(o, list(range(seqs)), q, out)
            for s in range(seqs):
                ids = torch.tensor(hyp[s], device="cuda")
                _, K, V = qkv(o, ids)
                want, A, top = attend_reference(q[s:s + 1].double(), K.double(), V.double(),
                                                torch.tensor([len(ids) - 1], device="cuda"), 15.0, slopes, layout[o][1])
                check_scores(out[s:s + 1], want, A, top, "f32", d, "f32", len(ids), f"step {step} layer {o} hypothesis {s}")
            outs.append(out.reshape(seqs, -1))
        logits = (torch.cat(outs, 1) @ head).view(groups, beams, vocab)
        logits[..., eos] += 2
        s_new, parent, token = ctx.beam_select(logits, scores, beams, finished=finished, eos_token=eos)
        S, B, T = select_reference(logits, scores, beams, finished, eos)
        assert (parent.cpu().numpy() == B).all() and (token.cpu().numpy() == T).all()
        src = (parent.cpu() + beams * torch.arange(groups)[:, None]).reshape(-1).tolist()
        ctx.fork_seqs(src, list(range(seqs)))
        hyp = [hyp[s] + [t] for s, t in zip(src, token.cpu().reshape(-1).tolist())]
        finished = (torch.gather(finished, 1, parent.long()).bool() | (token == eos)).to(torch.uint8)
        scores = s_new
    assert ctx.get_device_status() == 0
    ctx.close()
