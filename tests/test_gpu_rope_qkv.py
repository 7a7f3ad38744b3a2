"""Rotation of a projection's rows on a B200 against the formula in 64 bits, and what is stored against
what append_kv stores.

Bound of a rotated channel, x and y its pair's inputs: the angle, reduced to [-pi, pi], is rounded to fp32 (2^-23
at most), sine and cosine are off by at most two units in the last place (2^-23), each product and
the sum are rounded once (2^-24 each), and so is the factor's product with sine and cosine: (2^-23 + 2^-23 +
3 * 2^-24)(|x| + |y|), bounded by 2^-21 (|x| + |y|) times the factor; then half a step of the output's type."""
import math

import numpy as np
import pytest
import torch

from gpu_common import load_lib

pytestmark = pytest.mark.gpu


def turned(x, pos, rotary, halves, freq, scale):
    """(rotated x, |x| + |y| per channel) in 64 bits; x [tokens, heads, dim]."""
    x = x.double()
    angle = torch.outer(torch.as_tensor(pos, dtype=torch.float64, device="cuda"), torch.tensor(freq, dtype=torch.float64, device="cuda"))
    c, s = angle.cos()[:, None] * scale, angle.sin()[:, None] * scale
    out, size = x.clone(), torch.zeros_like(x)
    first = slice(0, rotary // 2) if halves else slice(0, rotary, 2)
    second = slice(rotary // 2, rotary) if halves else slice(1, rotary, 2)
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * c - b * s, a * s + b * c
    size[..., first] = size[..., second] = (a.abs() + b.abs()) * scale
    return out, size


def check(got, x, pos, rotary, halves, freq, scale, what=""):
    want, size = turned(x, pos, rotary, halves, freq, scale)
    bound = torch.finfo(got.dtype).eps / 2 * want.abs() * 1.001 + 2.0 ** -21 * size + 1e-38
    bound = torch.where(size == 0, torch.zeros_like(bound), bound)      # what does not turn is handed on
    assert ((got.double() - want).abs() <= bound).all(), (what, float(((got.double() - want).abs() - bound).max()))


def bits(t):
    return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def powers(rotary, theta=10000.0):
    return [theta ** (-2.0 * i / rotary) for i in range(rotary // 2)]


def make(heads, dtype, window, seqs=8, longest=600, layers=2):
    mx, _ = load_lib()
    layer = (mx.SLIDING, window) if window else (mx.FULL, 0)
    return mx, mx.Context([(*layer, 0)] * layers, *heads, mx.F32 if dtype == "f32" else mx.BF16, seqs, seqs * (longest // 16 + 2),
                          max_seq_len=longest, device=0, kv_format=mx.KV_FP8_E4M3 if dtype == "fp8" else mx.KV_NATIVE)


def projection(heads, tokens, dtype, seed=1, pad=0):
    hq, hkv, d = heads
    gen = torch.Generator("cuda").manual_seed(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    rows = torch.randn(tokens, (hq + 2 * hkv) * d + pad, generator=gen, device="cuda").to(t)
    cut = rows[:, :(hq + 2 * hkv) * d].view(tokens, hq + 2 * hkv, d) if pad == 0 else \
        rows.as_strided((tokens, hq + 2 * hkv, d), (rows.shape[1], d, 1))
    return cut[:, :hq], cut[:, hq:hq + hkv], cut[:, hq + hkv:]


FORMS = [((32, 8, 128), "bf16"), ((4, 2, 64), "bf16"), ((12, 3, 128), "fp8"), ((4, 2, 64), "f32"), ((5, 5, 128), "f32"), ((71, 1, 64), "bf16")]


@pytest.mark.parametrize("rotary", [16, 48, 64, 128])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("heads,dtype", FORMS)
def test_plain_tensors(heads, dtype, halves, rotary):
    if rotary > heads[2]:
        pytest.skip("more channels than the heads have")
    mx, ctx = make(heads, dtype, 0)
    lens, first = [1, 0, 7, 8, 9, 30, 2], [0, 5, 1000000, 31, 2047483000, 77, 3]
    tokens = sum(lens)
    q, k, v = projection(heads, tokens, dtype)
    freq = powers(rotary, 500000.0)
    pos = np.concatenate([np.arange(p, p + n) for p, n in zip(first, lens)])
    for rope, scale in ((mx.Rope(rotary, 500000.0, halves=halves), 1.0), (mx.Rope(rotary, inv_freq=freq, halves=halves, scale=1.25), 1.25)):
        qo, ko, vo = ctx.rope_qkv(0, range(7), lens, rope, q=q, k=k, v=v, first_pos=first)
        check(qo, q, pos, rotary, halves, freq, scale, "q")
        check(ko, k, pos, rotary, halves, freq, scale, "k")
        assert torch.equal(bits(vo), bits(v.contiguous()))
        only = ctx.rope_qkv(1, range(7), lens, rope, q=q, first_pos=first)
        assert torch.equal(bits(only[0]), bits(qo)) and only[1] is None and only[2] is None


@pytest.mark.parametrize("window", [0, 64, 100])
@pytest.mark.parametrize("heads,dtype", FORMS)
def test_stored_as_append_kv_stores(heads, dtype, window):
    """The same calls twice: rotated and stored in one go, or handed back and appended."""
    d = heads[2]
    mx, one = make(heads, dtype, window)
    _, two = make(heads, dtype, window)
    rope = mx.Rope(d, 10000.0, halves=True)
    ids = [3, 0, 7, 5]
    for step, lens in enumerate(([30, 1, 0, 205], None, [17, 17, 17, 17], [1, 2, 1, 0], None, [0, 130, 3, 1])):
        n = lens if lens is not None else [1] * 4
        q, k, v = projection(heads, sum(n), dtype, seed=step)
        was = [one.get_len(0, s) for s in ids]
        qo, none, _ = one.rope_qkv(0, ids, lens, rope, q=q, k=k, v=v, store=True)
        assert none is None
        pos = np.concatenate([np.arange(a, a + m) for a, m in zip(was, n)]).astype(float)
        check(qo, q, pos, d, True, powers(d), 1.0)
        q2, k2, v2 = two.rope_qkv(0, ids, lens, rope, q=q, k=k, v=v)
        assert torch.equal(bits(q2), bits(qo))
        check(k2, k, pos, d, True, powers(d), 1.0)
        two.append_kv(0, ids, lens, k2, v2)
        for s in ids:
            assert one.get_len(0, s) == two.get_len(0, s)
            assert one.get_block_table(s) == two.get_block_table(s)
        for a, b in zip(one.read_kv(1, ids), two.read_kv(1, ids)):
            assert torch.equal(bits(a), bits(b)), step
    # both ways at once, angles of other positions
    q, k, v = projection(heads, 4, dtype, seed=99)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    ko, vo = torch.empty(4, heads[1], d, device="cuda", dtype=t), torch.empty(4, heads[1], d, device="cuda", dtype=t)
    one.rope_qkv(0, ids, None, rope, q=q, k=k, v=v, store=True, first_pos=[9, 8, 7, 6], out=(None, ko, vo))
    check(ko, k, [9, 8, 7, 6], d, True, powers(d), 1.0)
    two.append_kv(0, ids, None, ko, vo)
    for a, b in zip(one.read_kv(1, ids), two.read_kv(1, ids)):
        assert torch.equal(bits(a), bits(b))


def test_interleaved_as_append_kv_rope():
    """Against the append that rotates dense keys: the angles agree to a few units of a double."""
    mx, one = make((8, 2, 128), "f32", 0)
    _, two = make((8, 2, 128), "f32", 0)
    q, k, v = projection((8, 2, 128), 300, "f32")
    one.rope_qkv(0, [1], [300], mx.Rope(128, 10000.0), k=k, v=v, store=True)
    two.append_kv_rope(0, [1], [300], k.contiguous(), v.contiguous(), 10000.0)
    a, b = one.read_kv(0, [1])[0].double(), two.read_kv(0, [1])[0].double()
    size = turned(k, np.arange(300), 128, False, powers(128), 1.0)[1]
    assert ((a - b).abs() <= 2.0 ** -20 * size).all()
    check(a.float(), k, np.arange(300), 128, False, powers(128), 1.0)


@pytest.mark.parametrize("pad", [8, 64])
def test_rows_apart(pad):
    heads = (8, 2, 64)
    mx, ctx = make(heads, "bf16", 0)
    q, k, v = projection(heads, 50, "bf16", pad=pad)
    qo, ko, vo = ctx.rope_qkv(0, [0], [50], mx.Rope(64, halves=True), q=q, k=k, v=v)
    for got, x in ((qo, q), (ko, k)):
        check(got, x, np.arange(50), 64, True, powers(64), 1.0)
    assert torch.equal(vo, v)


def test_many_sequences():
    heads = (8, 2, 64)
    mx, ctx = make(heads, "bf16", 0, seqs=300, longest=64)
    ids = list(range(299, -1, -1))
    for lens in (None, [i % 3 for i in range(300)], None):
        n = [1] * 300 if lens is None else lens
        was = [ctx.get_len(0, s) for s in ids]
        q, k, v = projection(heads, sum(n), "bf16")
        qo = ctx.rope_qkv(0, ids, lens, mx.Rope(64), q=q, k=k, v=v, store=True)[0]
        pos = np.concatenate([np.arange(a, a + m) for a, m in zip(was, n)]).astype(float)
        check(qo, q, pos, 64, False, powers(64), 1.0)
        ks, vs = ctx.read_kv(1, ids, first_pos=was, n_tokens=n)
        check(ks, k, pos, 64, False, powers(64), 1.0)
        assert torch.equal(vs, v)


def test_outputs_belong_to_the_stream():
    heads = (8, 2, 64)
    mx, ctx = make(heads, "bf16", 0)
    q, k, v = projection(heads, 600, "bf16")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20000000)
    got = ctx.rope_qkv(0, [0], [600], mx.Rope(64), q=q, k=k, v=v, stream=side)
    trash = [torch.full_like(x, 9.0) for x in got]      # on the current stream: other memory than the results'
    side.synchronize()
    check(got[0], q, np.arange(600), 64, False, powers(64), 1.0)
    assert all(bool((x == 9.0).all()) for x in trash)


def test_refusals():
    heads = (8, 2, 64)
    mx, ctx = make(heads, "bf16", 0, seqs=3, longest=64)
    q, k, v = projection(heads, 4, "bf16")

    def refused(code, layer=0, ids=(0, 1), n=(2, 2), rope=mx.Rope(64), **rest):
        rest = {"q": q, "k": k, "v": v, **rest}
        before = [ctx.get_len(0, s) for s in range(3)]
        with pytest.raises(mx.MixAttnError) as e:
            ctx.rope_qkv(layer, list(ids), None if n is None else list(n), rope, **rest)
        assert e.value.code == code
        assert [ctx.get_len(0, s) for s in range(3)] == before and ctx.get_n_free_pages() == 18

    for rope in (mx.Rope(0), mx.Rope(8), mx.Rope(72), mx.Rope(128), mx.Rope(64, 1.0), mx.Rope(64, math.inf), mx.Rope(64, math.nan),
                 mx.Rope(64, scale=-1.0), mx.Rope(64, scale=math.inf), mx.Rope(64, inv_freq=[math.nan] * 32)):
        refused(mx.ERR_INVALID_ARG, rope=rope)
    refused(mx.ERR_INVALID_ARG, layer=2)
    refused(mx.ERR_NOT_OWNER, layer=1, store=True)
    refused(mx.ERR_BAD_SEQ, ids=(0, 3))
    refused(mx.ERR_INVALID_ARG, ids=(0, 0), store=True)
    refused(mx.ERR_INVALID_ARG, n=(2, -2))
    refused(mx.ERR_INVALID_ARG, n=(2, 3))                            # other rows than the tensors have
    refused(mx.ERR_INVALID_ARG, first_pos=[-1, 0])
    refused(mx.ERR_INVALID_ARG, first_pos=[0, 2**31 - 2])
    refused(mx.ERR_INVALID_ARG, k=None, store=True)
    refused(mx.ERR_INVALID_ARG, q=q.float())
    refused(mx.ERR_INVALID_ARG, q=q.cpu())
    refused(mx.ERR_INVALID_ARG, q=k)
    refused(mx.ERR_INVALID_ARG, q=torch.empty(8, 4, 64, device="cuda", dtype=torch.bfloat16).transpose(0, 1))     # heads apart
    refused(mx.ERR_INVALID_ARG, q=torch.empty(4 * 516, device="cuda", dtype=torch.bfloat16).as_strided((4, 8, 64), (516, 64, 1)))   # 8 bytes off
    refused(mx.ERR_INVALID_ARG, q=torch.empty(4 * 512 + 4, device="cuda", dtype=torch.bfloat16)[4:].view(4, 8, 64))
    with pytest.raises(mx.MixAttnError):
        mx.Rope(64, inv_freq=[1.0])
    big = projection(heads, 65, "bf16")
    refused(mx.ERR_INVALID_ARG, ids=(0,), n=(65,), q=big[0], k=big[1], v=big[2], store=True)      # beyond the longest sequence
    assert ctx.rope_qkv(0, [], [], mx.Rope(64)) == (None, None, None)
    empty = ctx.rope_qkv(0, [0], [0], mx.Rope(64), q=q[:0])
    assert empty[0].shape == (0, 8, 64)
