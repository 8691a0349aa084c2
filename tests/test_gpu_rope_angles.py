"""Sines of far positions through the C ABI, against angles reduced in whole numbers.  The rest of a turn, at most one half turn, is
rounded to fp32 (2^-25 half turns, pi 2^-25 radians) and sincospif is good to one step (2^-24): together below 2^-22."""
from decimal import Decimal, localcontext

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def rest_of_turns(pos, freq):
    """pos * freq / (2 pi) without its whole turns: freq is a whole number of 2^-53, 1 / (2 pi) has 160 binary places."""
    with localcontext() as ctx:
        ctx.prec = 60
        per_turn = int(Decimal(2) ** 160 / (2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494")))
    steps = np.array([int(w * 2.0 ** 53) * per_turn for w in freq], object)
    assert all(w * 2.0 ** 53 == int(w * 2.0 ** 53) for w in freq)
    rest = (pos.astype(object)[:, None] * steps[None, :]) % 2 ** 213
    return (rest >> 153).astype(np.float64) * 2.0 ** -60


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("low,high,top", [(0, 5000, 1.0), (2 ** 30, 2 ** 31, 1.0), (-2 ** 31, -2 ** 30, 1.0), (2 ** 30, 2 ** 31, 65536.0)])
def test_sines_of_far_positions(low, high, top, interleaved, backward):
    import torch
    from paper_2404_15159_b200 import binding as B
    T, dim = 3000, 128
    rng = np.random.default_rng(91)
    pos = rng.integers(low, high, T)
    freq = rng.uniform(0.5, 1.0, dim // 2) * top
    x = torch.zeros(T, 1, dim, device="cuda")
    x[:, :, (slice(0, dim, 2) if interleaved else slice(0, dim // 2))] = 1.0     # the pair (1, 0) turns to (cos, sin)
    out = torch.empty_like(x)
    shape = B.make_rope_shape(T, 1, 0, dim, dim, B.MIXLORA_ROPE_INTERLEAVED if interleaved else B.MIXLORA_ROPE_HALF,
                              B.MIXLORA_DTYPE_FP32)
    call = B.mixlora_rope_backward if backward else B.mixlora_rope_forward
    call(shape, x, None, torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(freq).cuda(), out, None)
    angle = 2.0 * np.pi * rest_of_turns(pos, freq)
    got = out[:, 0].double().cpu().numpy()
    cos, sin = (got[:, 0::2], got[:, 1::2]) if interleaved else (got[:, :dim // 2], got[:, dim // 2:])
    assert np.abs(cos - np.cos(angle)).max() <= 2.0 ** -22
    assert np.abs(sin - (-1 if backward else 1) * np.sin(angle)).max() <= 2.0 ** -22
