"""Pins of the attention and rotary oracle: the mask against its definition, gradients against differences, the
rotation against complex multiplication and its adjoint."""
import numpy as np
import pytest

from oracle import attention_oracle as orc


@pytest.mark.parametrize("lq,lk", [(5, 5), (1, 7), (7, 3), (4, 9)])
@pytest.mark.parametrize("causal,window,prefix", [(True, 0, 0), (False, 0, 0), (True, 3, 0), (False, 2, 0), (True, 2, 4)])
def test_visible_is_its_definition(lq, lk, causal, window, prefix):
    got = orc.visible(lq, lk, causal, window, prefix)
    for i in range(lq):
        p = lk - lq + i
        for j in range(lk):
            want = j < prefix or ((not causal or j <= p) and (window == 0 or abs(p - j) < window))
            assert got[i, j] == want


@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(window=3), dict(softcap=2.0), dict(prefix=[2, 0, 1]),
                                dict(slopes=np.array([0.5, 0.25, 0.1, 0.0])), dict(softcap=1.5, window=2, causal=False)])
def test_gradients_match_differences(kw):
    rng = np.random.default_rng(5)
    q_off, k_off = [0, 4, 4, 10], [0, 6, 8, 14]
    q, do = rng.standard_normal((10, 4, 3)), rng.standard_normal((10, 4, 3))
    k, v = rng.standard_normal((14, 2, 3)), rng.standard_normal((14, 2, 3))

    def loss(q, k, v):
        return float((orc.attention(q, k, v, q_off, k_off, **kw)["o"] * do).sum())

    got = orc.attention(q, k, v, q_off, k_off, d_o=do, **kw)
    h = 1e-5
    for n, x in (("d_q", q), ("d_k", k), ("d_v", v)):
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in x.shape)
            args = dict(q=q, k=k, v=v)
            side = []
            for step in (h, -h):
                y = x.copy()
                y[at] += step
                args[n[2:]] = y
                side.append(loss(**args))
            assert abs((side[0] - side[1]) / (2 * h) - got[n][at]) < 1e-7


def test_rows_that_see_nothing_and_rows_outside():
    rng = np.random.default_rng(6)
    q, k, v = rng.standard_normal((6, 1, 4)), rng.standard_normal((5, 1, 4)), rng.standard_normal((5, 1, 4))
    got = orc.attention(q, k, v, [0, 4], [0, 5], k_len=[2], d_o=np.ones_like(q))
    assert not got["o"][:2].any() and np.isneginf(got["lse"][0, :2]).all() and not got["d_q"][:2].any()
    assert np.isnan(got["o"][4:]).all() and np.isnan(got["d_k"][2:]).all() and np.isfinite(got["d_k"][:2]).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_complex_multiplication_and_its_adjoint(interleaved):
    rng = np.random.default_rng(7)
    x, y = rng.standard_normal((5, 2, 10)), rng.standard_normal((5, 2, 10))
    w = orc.rope_frequencies(6, 10000.0)
    pos = np.array([0, 1, -3, 1000, 7])
    got, _ = orc.rope(x, pos, w, interleaved)
    z = x[..., 0:6:2] + 1j * x[..., 1:6:2] if interleaved else x[..., :3] + 1j * x[..., 3:6]
    z = z * np.exp(1j * pos[:, None] * w)[:, None, :]
    pair = (got[..., 0:6:2], got[..., 1:6:2]) if interleaved else (got[..., :3], got[..., 3:6])
    np.testing.assert_allclose(pair[0] + 1j * pair[1], z, atol=1e-12)
    np.testing.assert_array_equal(got[..., 6:], x[..., 6:])
    back, _ = orc.rope(y, pos, w, interleaved, backward=True)
    assert abs((got * y).sum() - (x * back).sum()) < 1e-10


def test_frequencies():
    w = orc.rope_frequencies(8, 100.0)
    np.testing.assert_allclose(w, [1.0, 100.0 ** -0.25, 0.1, 100.0 ** -0.75])
    np.testing.assert_allclose(orc.rope_frequencies(8, 100.0, orc.LINEAR, 4.0), w / 4)
    ntk = orc.rope_frequencies(8, 100.0, orc.NTK, 4.0)
    assert ntk[0] == 1.0
    np.testing.assert_allclose(ntk[-1], w[-1] / 4)                 # the slowest pair is stretched fully
    parts = orc.rope_frequencies(64, 10000.0, orc.PARTS, 8.0, 1.0, 4.0, 8192)
    full = orc.rope_frequencies(64, 10000.0)
    turns = 8192 * full / (2 * np.pi)
    np.testing.assert_array_equal(parts[turns >= 4], full[turns >= 4])
    np.testing.assert_allclose(parts[turns <= 1], full[turns <= 1] / 8)
    assert (np.diff(parts) < 0).all()
