"""Rotary positions through the C ABI against the float64 oracle.  A value is two products and a sum in fp32, each sine
within 2^-21 of the true one (a turn is reduced in 64 bits, sincospif is good to 2 steps, the rest is rounding), rounded
once to the type: |error| <= 2^-20 amplitude (|u| + |w|) + half a step of the value."""
import numpy as np
import pytest

from oracle import attention_oracle as orc
from paper_2404_15159_b200 import synth

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "fp32"])


def setup(T, hq, hk, dim, rot, bf16, seed=0, interleaved=False, amplitude=1.0, pad=0):
    import torch
    from paper_2404_15159_b200 import binding as B
    rng = np.random.default_rng(seed)
    rnd = synth.round_to_bf16 if bf16 else (lambda x: np.asarray(x, np.float32).astype(np.float64))
    act = torch.bfloat16 if bf16 else torch.float32
    q, k = rnd(rng.standard_normal((T, hq, dim))), rnd(rng.standard_normal((T, max(hk, 1), dim)))
    rows = torch.full((T, (hq + hk) * dim + pad), 7.0, dtype=act, device="cuda")
    rows[:, :hq * dim] = torch.from_numpy(q.reshape(T, -1)).cuda().to(act)
    if hk:
        rows[:, hq * dim:(hq + hk) * dim] = torch.from_numpy(k.reshape(T, -1)).cuda().to(act)
    table = torch.empty(rot // 2, dtype=torch.float64, device="cuda")
    B.mixlora_rope_frequencies(rot, 10000.0, B.MIXLORA_ROPE_SCALE_NONE, 1.0, 0.0, 0.0, 0, table)
    shape = B.make_rope_shape(T, hq, hk, dim, rot, B.MIXLORA_ROPE_INTERLEAVED if interleaved else B.MIXLORA_ROPE_HALF,
                              B.MIXLORA_DTYPE_BF16 if bf16 else B.MIXLORA_DTYPE_FP32, amplitude, q_stride=rows.stride(0),
                              k_stride=rows.stride(0))
    return B, torch, rng, q, k, rows, table, shape


def close(got, want, size, bf16):
    off = np.abs(got.double().cpu().numpy().reshape(want.shape) - want)
    bound = 2.0 ** -20 * size + (2.0 ** -8 if bf16 else 2.0 ** -24) * (np.abs(want) + 2.0 ** -20 * size)
    assert (off <= bound).all(), f"off by {(off / np.maximum(bound, 1e-300)).max():.2f} times the bound"


@TYPES
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("T,hq,hk,dim,rot", [(1, 1, 1, 8, 2), (1, 32, 8, 128, 128), (37, 5, 1, 80, 80), (130, 4, 4, 96, 48),
                                             (7, 3, 2, 64, 6), (3001, 2, 1, 128, 64), (5, 40, 0, 128, 128), (2, 2, 2, 512, 500)])
def test_against_the_oracle(T, hq, hk, dim, rot, interleaved, backward, bf16):
    B, torch, rng, q, k, rows, table, shape = setup(T, hq, hk, dim, rot, bf16, T, interleaved, 1.25, pad=8)
    pos = rng.integers(-1000, 2 ** 31 - 1, T).astype(np.int32) if T % 2 else rng.integers(0, 200000, T).astype(np.int32)
    q_out = torch.full((T, hq, dim), 7.0, dtype=rows.dtype, device="cuda")
    k_out = torch.full((T, max(hk, 1), dim), 7.0, dtype=rows.dtype, device="cuda")
    call = B.mixlora_rope_backward if backward else B.mixlora_rope_forward
    call(shape, rows, rows[:, hq * dim:] if hk else None, torch.from_numpy(pos).cuda(), table, q_out, k_out if hk else None)
    w = orc.rope_frequencies(rot, 10000.0)
    # the table is the library's own: its entries are a few 2^-53 off, which far positions multiply
    np.testing.assert_allclose(table.cpu().numpy(), w, rtol=2.0 ** -48)
    w = table.cpu().numpy()
    close(q_out, *orc.rope(q, pos, w, interleaved, 1.25, backward), bf16)
    if hk:
        close(k_out, *orc.rope(k, pos, w, interleaved, 1.25, backward), bf16)
    else:
        assert (k_out == 7.0).all()


@TYPES
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [64, 40, 6])
def test_in_place_equals_out_of_place_and_padding_is_left(rot, interleaved, bf16):
    T, hq, hk, dim = 2500, 4, 2, 64
    B, torch, rng, q, k, rows, table, shape = setup(T, hq, hk, dim, rot, bf16, 3, interleaved, pad=24)
    out = [torch.empty(T, h, dim, dtype=rows.dtype, device="cuda") for h in (hq, hk)]
    B.mixlora_rope_forward(shape, rows, rows[:, hq * dim:], None, table, *out)
    shape.q_out_stride = shape.k_out_stride = rows.stride(0)
    B.mixlora_rope_forward(shape, rows, rows[:, hq * dim:], None, table, rows, rows[:, hq * dim:])
    assert torch.equal(rows[:, :hq * dim].reshape(T, hq, dim), out[0])
    assert torch.equal(rows[:, hq * dim:(hq + hk) * dim].reshape(T, hk, dim), out[1])
    assert (rows[:, -24:] == 7.0).all()
    # and back: the gradient's way undoes a pure rotation
    B.mixlora_rope_backward(shape, rows, rows[:, hq * dim:], None, table, rows, rows[:, hq * dim:])
    back = rows[:, :hq * dim].double().cpu().numpy().reshape(T, hq, dim)
    assert np.abs(back - q).max() <= (2.0 ** -6 if bf16 else 2.0 ** -19) * np.abs(q).max()


@pytest.mark.parametrize("args", [(128, 10000.0, 0, 1.0, 0.0, 0.0, 0), (2, 10000.0, 2, 4.0, 0.0, 0.0, 0), (96, 5e5, 1, 8.0, 0.0, 0.0, 0),
                                  (128, 10000.0, 2, 4.0, 0.0, 0.0, 0), (128, 5e5, 3, 8.0, 1.0, 4.0, 8192),
                                  (512, 10000.0, 3, 2.0, 0.0, 32.0, 2048)])
def test_frequencies(args):
    import torch
    from paper_2404_15159_b200 import binding as B
    out = torch.full((args[0] // 2 + 1,), 7.0, dtype=torch.float64, device="cuda")
    B.mixlora_rope_frequencies(*args, out)
    want = orc.rope_frequencies(*args)
    np.testing.assert_allclose(out[:-1].cpu().numpy(), want, rtol=2.0 ** -46)
    assert out[-1] == 7.0


def test_no_tokens():
    B, torch, rng, q, k, rows, table, shape = setup(1, 2, 2, 64, 64, True)
    shape.tokens = 0
    out = torch.full((1, 2, 64), 7.0, dtype=rows.dtype, device="cuda")
    B.mixlora_rope_forward(shape, rows, rows[:, 128:], None, table, out, out)
    torch.cuda.synchronize()
    assert (out == 7.0).all()
