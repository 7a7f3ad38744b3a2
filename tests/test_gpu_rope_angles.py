"""Angles of rotated projections up to the largest positions and frequencies that a call takes, against sines of angles
that are reduced exactly, in rational numbers.  Bounds: test_gpu_rope_qkv.py, 2^-21 (|x| + |y|) and half a step of the type."""
import math
from fractions import Fraction

import pytest
import torch

from test_gpu_rope_qkv import check, make, projection  # noqa: F401

pytestmark = pytest.mark.gpu

TWO_PI = Fraction("6.28318530717958647692528676655900576839433879875021")


def turn(pos, freq):
    """(cos, sin) of pos * freq"""
    a = pos * Fraction(freq)
    a -= round(a / TWO_PI) * TWO_PI
    return math.cos(a), math.sin(a)


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_positions_and_fast_pairs(dtype, halves):
    heads = (4, 2, 64)
    mx, ctx = make(heads, dtype, 0)
    first = [0, 131071, 999983, 1 << 24, (1 << 31) - 4, 2047483000, 1]
    freq = [1e6, 999999.7, 999900.0, 123456.789, 3.0, 1.0, 6.283185307179586, -999999.7, 1.5707963267948966, 355.0, 1e-7, 0.0, 22.0 / 7, 710.0, 98765.4321, 1e5 + 0.1]
    q, k, v = projection(heads, 3 * len(first), dtype)
    rope = mx.Rope(32, inv_freq=freq, halves=halves)
    qo, ko, _ = ctx.rope_qkv(0, range(7), [3] * 7, rope, q=q, k=k, v=v, first_pos=first)
    pos = [p + i for p in first for i in range(3)]
    cs = torch.tensor([[turn(p, f) for f in freq] for p in pos], dtype=torch.float64, device="cuda")
    c, s = cs[..., 0][:, None], cs[..., 1][:, None]
    a, b = (slice(0, 16), slice(16, 32)) if halves else (slice(0, 32, 2), slice(1, 32, 2))
    for x, got in ((q.double(), qo), (k.double(), ko)):
        want, size = x.clone(), torch.zeros_like(x)
        want[..., a], want[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
        bound = torch.finfo(got.dtype).eps / 2 * want.abs() * 1.001 + 2.0 ** -21 * size
        err = (got.double() - want).abs()
        assert (err <= bound).all(), float((err - bound).max())


def test_the_last_position():
    """2^31 - 2 is the last one; the largest frequency is 1e6."""
    heads = (4, 2, 64)
    mx, ctx = make(heads, "f32", 0)
    q = projection(heads, 2, "f32")[0]
    ctx.rope_qkv(0, [0], [2], mx.Rope(64), q=q, first_pos=[(1 << 31) - 3])
    for f, at in ((1.0, (1 << 31) - 2), (1e6 + 1, 0), (-1e6 - 1, 0), (math.inf, 0), (math.nan, 0)):
        with pytest.raises(mx.MixAttnError) as e:
            ctx.rope_qkv(0, [0], [2], mx.Rope(64, inv_freq=[1.0] * 31 + [f]), q=q, first_pos=[at])
        assert e.value.code == mx.ERR_INVALID_ARG
