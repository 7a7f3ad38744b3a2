"""Attention with capped and distance-biased scores on a B200 against the definition in 64 bits:
one query per sequence, prompts and chunks behind a cache, every storage format.

Bounds, with A = sum_j p_j |v_j| of the output element in question (p the softmax weights):
  * the output's own rounding: half a step, eps / 2 of its value;
  * bf16 prompts hold the weights as one bf16 number each: 2^-8 A (half a step, and the sum of the
    weights keeps full precision), decode holds them to 16 bits and a quantised cache as fp16:
    2^-11 A, plus half the fp16 subnormal step times the largest element (448) per key;
  * scores are fp32 numbers of magnitude s in base-2 units, made of head_dim products and a dozen
    further roundings (six of them the cap's): 2^-24 s sqrt(head_dim) for the sum's random walk, bounded here by
    2^-24 s (head_dim / 4 + 16); an error d of a score moves weights by d ln 2, the output by
    at most 2 d ln 2 A."""
import numpy as np
import pytest
import torch

from gpu_common import load_lib

pytestmark = pytest.mark.gpu

SHAPES = {"none": (0.0, False), "cap": (20.0, False), "bias": (0.0, True), "both": (30.0, True)}


def slopes_of(hq):
    return [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]


def reference(q, K, V, pos, cap, slopes, window, scale=None):
    """q [t, Hq, D] at positions pos [t], K / V [n, Hkv, D] of positions 0..n-1, all float64.
    Returns (out, A, largest |score| in base 2)."""
    t, hq, d = q.shape
    n, hkv, _ = K.shape
    scale = d ** -0.5 if scale is None else scale
    back = pos[:, None] - torch.arange(n, device=q.device)[None]
    hidden = back < 0
    if window:
        hidden |= back >= window
    out, A, top = torch.empty_like(q), torch.empty_like(q), 0.0
    for h in range(hq):
        g = h // (hq // hkv)
        s = q[:, h] @ K[:, g].T * scale
        if cap:
            s = cap * torch.tanh(s / cap)
        if slopes is not None:
            s = s - slopes[h] * back.double()
        s = s.masked_fill(hidden, float("-inf"))
        p = torch.softmax(s, dim=-1)
        out[:, h] = p @ V[:, g]
        A[:, h] = p @ V[:, g].abs()
        # (keys whose weight vanishes do not matter, however large their bias)
        near = s.masked_fill(p < 2.0 ** -40, 0.0)
        top = max(top, float(near.abs().max()) / np.log(2))
    return out, A, top


def check(got, want, A, top, dtype, d, kind, n_keys, what):
    eps = torch.finfo(got.dtype).eps / 2
    w = {"prompt": 2.0 ** -8, "decode": 2.0 ** -16, "fp8": 2.0 ** -11, "f32": 2.0 ** -23}[kind]
    score = 2.0 ** -24 * top * (d / 4 + 16) * 2 * np.log(2)
    bound = eps * want.abs() * 1.001 + (w + score) * A + 1e-30
    if kind == "fp8":
        bound = bound + n_keys * 2.0 ** -25 * 448
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all(), what
    worst = float((err / bound).max())
    assert worst <= 1, f"{what}: {worst:.3f} of the bound, max error {float(err.max()):.3e}"


def on_e4m3(x):
    top = x.abs().amax(-1, keepdim=True).float()
    scale = torch.exp2(torch.floor(torch.log2(torch.clamp(top, min=1e-30))) - 8)
    return (torch.clamp(x.float() / scale, -448, 448).to(torch.float8_e4m3fn).float() * scale).to(x.dtype)


def make(mx, kind, window, heads, dtype, seqs, longest, chunk=0, scale=0.0, layers=2):
    hq, hkv, d = heads
    layer = (mx.SLIDING, window) if window else (mx.FULL, 0)
    return mx.Context([(*layer, 0)] * layers, hq, hkv, d, mx.F32 if dtype == "f32" else mx.BF16, seqs,
                      seqs * (-(-longest // 16) + 1), max_seq_len=longest + 64, device=0, chunk_scratch_tokens=chunk,
                      kv_format=mx.KV_FP8_E4M3 if dtype == "fp8" else mx.KV_NATIVE, softmax_scale=scale)


HEADS = [(8, 2, 128), (4, 4, 64), (12, 1, 128), (20, 2, 64)]


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("dtype,heads", [("bf16", h) for h in HEADS] + [("f32", (4, 2, 64)), ("f32", (9, 1, 128)),
                                                                      ("fp8", (8, 2, 128)), ("fp8", (12, 1, 128))])
@pytest.mark.parametrize("window", [0, 70, 256])
def test_decode(shape, dtype, heads, window):
    mx, _ = load_lib()
    cap, biased = SHAPES[shape]
    hq, hkv, d = heads
    slopes = slopes_of(hq) if biased else None
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 70, 71, 141, 255, 256, 257, 700, 1025]
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    gen = torch.Generator("cuda").manual_seed(1)
    ctx = make(mx, "decode", window, heads, dtype, len(lens), max(lens))
    K, V = [], []
    for i, n in enumerate(lens):
        k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda").to(dt) for _ in range(2))
        if dtype == "fp8":
            k, v = on_e4m3(k), on_e4m3(v)
        ctx.append_kv(0, [i], [n], k, v)
        K.append(k)
        V.append(v)
    ctx.set_layer_scores(1, cap, slopes)
    q = (3 * torch.randn(len(lens), hq, d, generator=gen, device="cuda")).to(dt)
    out = torch.full_like(q, float("nan"))
    ctx.decode(1, list(range(len(lens))), q, out)
    static = torch.full_like(q, float("nan"))
    assert ctx.rc_decode_static_scratch(1, list(range(len(lens))), q, static) == 0
    torch.cuda.synchronize()
    assert ctx.get_device_status() == 0
    assert torch.equal(out, static)
    for i, n in enumerate(lens):
        want, A, top = reference(q[i:i + 1].double(), K[i].double(), V[i].double(), torch.tensor([n - 1], device="cuda"), cap,
                                 slopes, window)
        kind = {"bf16": "decode", "fp8": "fp8", "f32": "f32"}[dtype]
        check(out[i:i + 1], want, A, top, dtype, d, kind, min(n, window or n), f"len {n}")
    # plain scores again
    ctx.set_layer_scores(1)
    again = torch.empty_like(q)
    ctx.decode(1, list(range(len(lens))), q, again)
    # layer 0 keeps its plain scores
    ctx.decode(0, list(range(len(lens))), q, out)
    want, A, top = reference(q[9:10].double(), K[9].double(), V[9].double(), torch.tensor([lens[9] - 1], device="cuda"), 0.0,
                             None, window)
    check(out[9:10], want, A, top, dtype, d, {"bf16": "decode", "fp8": "fp8", "f32": "f32"}[dtype], lens[9], "plain layer")
    assert torch.equal(out, again)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("batch,n", [(1, 9000), (3, 5000), (70, 1024)])   # clusters, splits and short items
def test_decode_launch_variants(dtype, batch, n):
    mx, _ = load_lib()
    heads = hq, hkv, d = 8, 4, 128
    cap, slopes = 25.0, slopes_of(hq)
    gen = torch.Generator("cuda").manual_seed(2)
    ctx = make(mx, "decode", 0, heads, dtype, batch, n)
    k, v = (torch.randn(batch, n, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    if dtype == "fp8":
        k, v = on_e4m3(k), on_e4m3(v)
    ctx.append_kv(0, list(range(batch)), [n] * batch, k, v)
    for l in (0, 1):
        ctx.set_layer_scores(l, cap, slopes)
    q = (3 * torch.randn(batch, hq, d, generator=gen, device="cuda")).bfloat16()
    out = torch.empty_like(q)
    ctx.decode(0, list(range(batch)), q, out)
    torch.cuda.synchronize()
    for i in sorted({0, batch // 2, batch - 1}):
        want, A, top = reference(q[i:i + 1].double(), k[i].double(), v[i].double(), torch.tensor([n - 1], device="cuda"), cap,
                                 slopes, 0)
        check(out[i:i + 1], want, A, top, dtype, d, "fp8" if dtype == "fp8" else "decode", n, f"sequence {i}")
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 64])
def test_rows_behind_a_sequence_do_not_matter(dtype, window):
    # pages and ring slots behind a short sequence hold an earlier one's infinities and NaN
    mx, _ = load_lib()
    heads = hq, hkv, d = 4, 2, 128
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    ctx = make(mx, "decode", window, heads, dtype, 1, 64)
    bad = torch.full((64, hkv, d), float("nan"), device="cuda", dtype=dt)
    bad[::2] = float("inf")
    ctx.append_kv(0, [0], [64], bad, bad)
    ctx.seq_reset(0)
    gen = torch.Generator("cuda").manual_seed(3)
    n = 21
    k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda").to(dt) for _ in range(2))
    ctx.append_kv(0, [0], [n], k, v)
    ctx.set_layer_scores(1, 30.0, slopes_of(hq))
    q = torch.randn(1, hq, d, generator=gen, device="cuda").to(dt)
    out = torch.empty_like(q)
    ctx.decode(1, [0], q, out)
    torch.cuda.synchronize()
    want, A, top = reference(q.double(), k.double(), v.double(), torch.tensor([n - 1], device="cuda"), 30.0, slopes_of(hq), window)
    check(out, want, A, top, dtype, d, "f32" if dtype == "f32" else "decode", n, "stale rows")
    ctx.close()


@pytest.mark.parametrize("shape", ["cap", "bias", "both"])
@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 2, 128)), ("bf16", (4, 4, 64)), ("f32", (4, 2, 64)), ("f32", (2, 1, 128))])
@pytest.mark.parametrize("window", [0, 50, 128, 300])
def test_prompt(shape, dtype, heads, window):
    mx, _ = load_lib()
    cap, biased = SHAPES[shape]
    hq, hkv, d = heads
    slopes = slopes_of(hq) if biased else None
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    lens = [1, 127, 128, 129, 700] if dtype == "bf16" else [1, 33, 200]
    gen = torch.Generator("cuda").manual_seed(4)
    total = sum(lens)
    q = (3 * torch.randn(total, hq, d, generator=gen, device="cuda")).to(dt)
    k, v = (torch.randn(total, hkv, d, generator=gen, device="cuda").to(dt) for _ in range(2))
    ctx = make(mx, "prompt", window, heads, dtype, len(lens), max(lens))
    ctx.set_layer_scores(0, cap, slopes)
    out = torch.full_like(q, float("nan"))
    ctx.prefill(0, list(range(len(lens))), lens, q, k, v, out)
    torch.cuda.synchronize()
    assert ctx.get_device_status() == 0
    row = 0
    for n in lens:
        r = slice(row, row + n)
        want, A, top = reference(q[r].double(), k[r].double(), v[r].double(), torch.arange(n, device="cuda"), cap, slopes, window)
        check(out[r], want, A, top, dtype, d, "f32" if dtype == "f32" else "prompt", n, f"len {n}")
        row += n
    ctx.close()


@pytest.mark.parametrize("shape", ["cap", "bias", "both"])
def test_unaligned_tensors_take_the_exact_kernel(shape):
    mx, _ = load_lib()
    cap, biased = SHAPES[shape]
    hq, hkv, d, n = 4, 2, 64, 90
    gen = torch.Generator("cuda").manual_seed(8)
    flat = torch.randn(3, n * hq * d + 8, generator=gen, device="cuda").bfloat16()
    q, k, v = flat[0, 1:1 + n * hq * d].view(n, hq, d), flat[1, 3:3 + n * hkv * d].view(n, hkv, d), flat[2, 5:5 + n * hkv * d].view(n, hkv, d)
    ctx = make(mx, "prompt", 33, (hq, hkv, d), "bf16", 1, n)
    ctx.set_layer_scores(1, cap, slopes_of(hq) if biased else None)
    out = torch.full((n, hq, d), float("nan"), device="cuda", dtype=torch.bfloat16)
    ctx.prefill(1, [0], [n], q, k, v, out)      # (a layer that reads a cache: nothing is stored)
    torch.cuda.synchronize()
    want, A, top = reference(q.double(), k.double(), v.double(), torch.arange(n, device="cuda"), cap,
                             slopes_of(hq) if biased else None, 33)
    check(out, want, A, top, "bf16", d, "f32", n, "unaligned")
    ctx.close()


@pytest.mark.parametrize("direct", [True, False])
@pytest.mark.parametrize("shape", ["cap", "bias", "both"])
@pytest.mark.parametrize("window", [0, 128, 384, 200])
@pytest.mark.parametrize("d", [128, 64])
def test_chunks_behind_a_cache(direct, shape, window, d):
    mx, _ = load_lib()
    cap, biased = SHAPES[shape]
    hq, hkv = 6, 2
    heads = hq, hkv, d
    slopes = slopes_of(hq) if biased else None
    prefix, lens = [300, 0, 1000, 127], [200, 130, 1, 390]
    gen = torch.Generator("cuda").manual_seed(5)
    ctx = make(mx, "chunk", window, heads, "bf16", len(lens), 1400, chunk=4096)
    ctx.set_chunk_ring_direct(direct)
    K, V = [], []
    for i, (p, n) in enumerate(zip(prefix, lens)):
        k, v = (torch.randn(p + n, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
        if p:
            ctx.append_kv(0, [i], [p], k[:p].contiguous(), v[:p].contiguous())
        K.append(k)
        V.append(v)
    q = (3 * torch.randn(sum(lens), hq, d, generator=gen, device="cuda")).bfloat16()
    ctx.set_layer_scores(1, cap, slopes)
    out = torch.full_like(q, float("nan"))
    ctx.attend_chunk(1, list(range(len(lens))), lens, q, torch.cat([k[p:] for k, p in zip(K, prefix)]),
                     torch.cat([v[p:] for v, p in zip(V, prefix)]), out)
    torch.cuda.synchronize()
    assert ctx.get_device_status() == 0
    row = 0
    for i, (p, n) in enumerate(zip(prefix, lens)):
        r = slice(row, row + n)
        want, A, top = reference(q[r].double(), K[i].double(), V[i].double(), torch.arange(p, p + n, device="cuda"), cap, slopes,
                                 window)
        check(out[r], want, A, top, "bf16", d, "prompt", p + n, f"prefix {p} chunk {n}")
        row += n
    ctx.close()


@pytest.mark.parametrize("window", [0, 128])
def test_chunks_behind_a_quantised_cache(window):
    mx, _ = load_lib()
    hq, hkv, d = heads = 6, 2, 128
    prefix, n = 210, 150
    gen = torch.Generator("cuda").manual_seed(10)
    ctx = make(mx, "chunk", window, heads, "fp8", 1, 500, chunk=1000)
    k, v = (torch.randn(prefix + n, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    k[:prefix], v[:prefix] = on_e4m3(k[:prefix]), on_e4m3(v[:prefix])
    ctx.append_kv(0, [0], [prefix], k[:prefix].contiguous(), v[:prefix].contiguous())
    q = (3 * torch.randn(n, hq, d, generator=gen, device="cuda")).bfloat16()
    ctx.set_layer_scores(1, 25.0, slopes_of(hq))
    out = torch.full_like(q, float("nan"))
    ctx.attend_chunk(1, [0], [n], q, k[prefix:].contiguous(), v[prefix:].contiguous(), out)
    torch.cuda.synchronize()
    want, A, top = reference(q.double(), k.double(), v.double(), torch.arange(prefix, prefix + n, device="cuda"), 25.0,
                             slopes_of(hq), window)
    check(out, want, A, top, "bf16", d, "prompt", prefix + n, "quantised prefix")
    ctx.close()


@pytest.mark.parametrize("window", [0, 256])
def test_scores_far_above_the_first_tile(window):
    # scores of several hundred, which make the prompt kernel move its exponent reference; capped
    # ones of up to the cap, and steep slopes
    mx, _ = load_lib()
    heads = hq, hkv, d = 4, 2, 128
    n = 900
    gen = torch.Generator("cuda").manual_seed(6)
    q = (60 * torch.randn(n, hq, d, generator=gen, device="cuda")).bfloat16()
    k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    for cap, slopes in ((0.0, [0.0, 0.01, 1.0, 100.0]), (150.0, None), (400.0, [1024.0, 3.0, 0.0, 0.3])):
        ctx = make(mx, "prompt", window, heads, "bf16", 1, n)
        ctx.set_layer_scores(0, cap, slopes)
        out = torch.full_like(q, float("nan"))
        ctx.prefill(0, [0], [n], q, k, v, out)
        torch.cuda.synchronize()
        want, A, top = reference(q.double(), k.double(), v.double(), torch.arange(n, device="cuda"), cap, slopes, window)
        check(out, want, A, top, "bf16", d, "prompt", n, f"cap {cap}")
        ctx.decode(0, [0], q[-1:], out[-1:])
        torch.cuda.synchronize()
        check(out[-1:], want[-1:], A[-1:], top, "bf16", d, "decode", n, f"decode, cap {cap}")
        ctx.close()


def test_one_call_over_many_layers_and_a_captured_step():
    mx, _ = load_lib()
    heads = hq, hkv, d = 8, 2, 128
    n = 333
    ctx = make(mx, "decode", 0, heads, "bf16", 2, n + 8, layers=3)
    gen = torch.Generator("cuda").manual_seed(7)
    k, v = (torch.randn(2, n, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    ctx.append_kv(0, [0, 1], [n, n], k, v)
    kn, vn = (torch.randn(2, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = (2 * torch.randn(2, hq, d, generator=gen, device="cuda")).bfloat16()
    shapes = [(0.0, None), (20.0, None), (0.0, slopes_of(hq))]
    for l, (cap, s) in enumerate(shapes):
        ctx.set_layer_scores(l, cap, s)
    outs = torch.empty(3, 2, hq, d, dtype=torch.bfloat16, device="cuda")
    ctx.decode_layers(0, 3, [0, 1], ctx.pointer_table([q] * 3), ctx.pointer_table([kn, None, None]),
                      ctx.pointer_table([vn, None, None]), ctx.pointer_table(list(outs)))
    torch.cuda.synchronize()
    for l, (cap, s) in enumerate(shapes):
        for i in range(2):
            want, A, top = reference(q[i:i + 1].double(), torch.cat([k[i], kn[i:i + 1]]).double(),
                                     torch.cat([v[i], vn[i:i + 1]]).double(), torch.tensor([n], device="cuda"), cap, s, 0)
            check(outs[l, i:i + 1], want, A, top, "bf16", d, "decode", n + 1, f"layer {l}")
    # a captured call replays with new queries
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    out = torch.empty_like(q)
    qg = q.clone()
    with torch.cuda.graph(graph, stream=stream):
        ctx.decode(2, [0, 1], qg, out, stream=torch.cuda.current_stream())
    q2 = (2 * torch.randn(2, hq, d, generator=gen, device="cuda")).bfloat16()
    qg.copy_(q2)
    graph.replay()
    torch.cuda.synchronize()
    direct = torch.empty_like(q)
    ctx.decode(2, [0, 1], q2, direct)
    torch.cuda.synchronize()
    assert torch.equal(out, direct)
    ctx.close()
