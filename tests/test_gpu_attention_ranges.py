"""Masked attention at the edges of its range: scores that jump within a tile, capped scores of every size, values that
are very large or small, what lies outside the sequences.  Cases, oracle and bounds as in test_gpu_attention.py."""
import numpy as np
import pytest

from paper_2404_15159_b200 import synth
from test_gpu_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("mask", [dict(), dict(slopes=[0.001, 0.0])], ids=str)
def test_rows_of_a_warp_rescale_at_different_places(mask, dim):
    # Even rows' scores have grown by some 2^13 in the tile before (their sums are rescaled at the next tile's start), odd
    # rows' jump by 2^140 in that tile's first 64 keys (theirs are rescaled again at once).  With a distance term the tiles
    # come last keys first.
    c = Case([300], hq=2, hk=2, dim=dim, seed=70 + dim, causal=False, **mask)
    grow, jump = (slice(192, 256), slice(0, 64)) if mask else (slice(64, 128), slice(128, 192))
    unit = 2.0 * dim ** 0.5                           # times a key's 1: a score of 2
    c.q[0::2, :, :2], c.q[1::2, :, :2] = [unit, 0.0], [0.0, unit]
    c.k[:, :, :2] = 0.0
    c.k[grow, :, 0], c.k[jump, :, 1] = 4.5, 50.0
    c.q = synth.round_to_bf16(c.q)                   # as the GPU gets them
    c.check(c.run())


def parts(c, got, b):
    """What a run gives for sequence b: its rows and its used keys."""
    rows = slice(c.q_off[b], c.q_off[b + 1])
    keys = slice(c.k_off[b], c.k_off[b] + (c.k_off[b + 1] - c.k_off[b] if c.k_len is None else c.k_len[b]))
    return {n: x[:, rows] if n == "lse" else x[keys] if n in ("d_k", "d_v") else x[rows] for n, x in got.items()}


def same(a, b):
    assert all(np.array_equal(a[n], b[n]) for n in a), [n for n in a if not np.array_equal(a[n], b[n])]


@pytest.mark.parametrize("q_len", [0, 2])
@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "fp32"])
@pytest.mark.parametrize("slopes", [None, [0.25, 0.0]], ids=str)
def test_capped_scores_are_the_same_whatever_lies_outside(slopes, bf16, q_len):
    # zeros, values whose scores lie far above the cap, and NaN: behind the used keys, and in rows of no sequence
    lens, slots, used = ([40, 150, 1], [70, 200, 130], [50, 150, 129]) if q_len == 0 else ([q_len] * 3, [70, 200, 130], [50, 150, 129])
    runs = []
    for fill in (0.0, 1000.0, np.nan):
        c = Case(lens, k_lens=slots, k_len=used, hq=2, hk=2, dim=64, seed=81, bf16=bf16, tail=70, softcap=6.0, slopes=slopes)
        for x in (c.q, c.k, c.v, c.d_o):
            x[np.isnan(x)] = fill
        runs.append(c.run(backward=q_len == 0, max_q_len=q_len))
    for got in runs[1:]:
        for b in range(3):
            same(parts(c, runs[0], b), parts(c, got, b))


@pytest.mark.parametrize("slopes", [None, [0.25, 0.0]], ids=str)
def test_capped_scores_are_the_same_whatever_the_neighbours_hold(slopes):
    runs = []
    for amp in (1.0, 64.0):
        c = Case([75, 140, 200], hq=2, hk=2, dim=64, seed=82, softcap=6.0, slopes=slopes)
        for x in (c.q, c.k, c.v, c.d_o):
            x[:75] *= amp
            x[215:] *= amp
        runs.append(c.run())
    same(parts(c, runs[0], 1), parts(c, runs[1], 1))
    assert not np.array_equal(parts(c, runs[0], 0)["o"], parts(c, runs[1], 0)["o"])


@pytest.mark.parametrize("amp", [0.2, 3.0, 30.0])
@pytest.mark.parametrize("mask", [dict(), dict(slopes=[0.25, 0.0]), dict(window=70, prefix=[20, 0])], ids=str)
def test_scores_below_around_and_far_above_the_cap(mask, amp):
    # amp 0.2: the polynomial alone; 3: both forms in a warp; 30: most scores at the cap
    c = Case([190, 300], hq=2, hk=2, dim=96, seed=83, amp=amp, softcap=4.0, **mask)
    c.check(c.run())


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "fp32"])
@pytest.mark.parametrize("softcap", [200.0, 1e4, 1e8, 1e30])
def test_caps_far_above_the_scores(softcap, bf16, few):
    # A capped score is cap2 tanh(x mul): the three factors' and two products' roundings are 5 half steps of 2^-24, the
    # polynomial is off by 2.6e-7 (4.4 of 2^-24) and rounds 3 times more at its end: 2^-20 of the score covers them.
    c = Case([2, 1, 2] if few else [60, 1, 130], k_lens=[700, 300, 130], k_len=[700, 256, 130], hq=4, hk=2, dim=128, seed=84,
             bf16=bf16, softcap=softcap, cap_rel=2.0 ** -20)
    c.check(c.run(backward=not few, max_q_len=2 if few else 0), backward=not few)


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "fp32"])
@pytest.mark.parametrize("v_size", [2.0 ** 80, 1.0, 2.0 ** -80], ids=["2^80", "1", "2^-80"])
@pytest.mark.parametrize("softcap,slopes", [(0.0, None), (0.0, [0.01, 0.0]), (60.0, None), (66.5, None), (67.0, None),
                                            (100.0, None), (60.0, [0.01, 0.0])], ids=str)
def test_small_and_large_values_under_rising_scores(softcap, slopes, v_size, bf16, few):
    # first scores of about 0 (-90 with a distance term, or minus the cap), then, for rows that see them, some of +60 and one
    # of +90: rows' weights jump by 2^86, or by 2^170 and more, and nothing of v may be lost on the way
    c = Case([2] if few else [300], k_lens=[300], hq=2, hk=2, dim=64, seed=85, bf16=bf16, softcap=softcap, slopes=slopes,
             causal=not few)
    c.q[:, :, 0] = 16.0                               # times a key's 1: a score of 2
    c.k[:, :, 0] = -200.0 if softcap else -45.0 if slopes else 0.0
    c.k[100:110, :, 0], c.k[210, :, 0] = 30.0, 45.0
    c.v *= v_size
    got = c.run(backward=not few, max_q_len=2 if few else 0)
    c.check(got, backward=not few)
    assert (np.abs(got["o"]).max(axis=(1, 2)) > v_size / 64).all()


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 30])
def test_widest_window_over_the_most_rows(window):
    # 2^30 rows stand up to 2^30 - 1 before their one key: position less window would leave 32 bits
    import torch
    from paper_2404_15159_b200 import binding as B
    rows = 2 ** 30
    x = torch.zeros(rows, 1, 8, dtype=torch.bfloat16, device="cuda")
    x[0] = torch.arange(8, device="cuda")
    o = torch.full_like(x, 100.0)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    shape = B.make_attention_shape(1, rows, rows, 1, 1, 8, causal=0, window=window)
    ws = B.alloc_attention_workspace(shape, False)
    mask = B.make_attention_mask(off, off, k_len=torch.ones(1, dtype=torch.int32, device="cuda"))
    B.mixlora_attention_forward(shape, mask, x, x, x, o, None, ws)
    assert B.mixlora_device_status(ws) == 0
    assert all(bool((part == x[0]).all()) for part in o.split(2 ** 27))
    del x, o, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "fp32"])
@pytest.mark.parametrize("seqs,q_len,hq", [(1, 1, 2), (40, 1, 4), (3, 2, 8)])
def test_few_rows_keep_weights_beyond_bf16(seqs, q_len, hq, bf16):
    # Up to 8 rows a key head.  Values that come in pairs v, -v whose weights differ by a few per cent, so that o is a small
    # part of sum p |v|: weights rounded once to bf16 would be off by 2^-8 of that sum.  They go in as two bf16 values, off by
    # half a step of the second, 2^-16; the output's own rounding is 2^-8 of o itself.
    from oracle import attention_oracle as orc
    c = Case([q_len] * seqs, k_lens=[64] * seqs, hq=hq, hk=2, dim=16, seed=86, bf16=bf16, causal=False, amp=0.5)
    c.k[1::2] = synth.round_to_bf16(c.k[0::2] + 0.03 * np.random.default_rng(5).standard_normal(c.k[0::2].shape))
    c.v[1::2] = -c.v[0::2]
    got = c.run(backward=False, max_q_len=q_len)
    want = orc.attention(c.q, c.k, c.v, c.q_off, c.k_off, causal=False, p_step=2.0 ** -16, out_step=0.0)
    bound = want["bound"]["o"] + (2.0 ** -8 if bf16 else 2.0 ** -24) * (np.abs(want["o"]) + want["bound"]["o"])
    assert (np.abs(got["o"] - want["o"]) <= bound).all()
    assert (np.abs(got["lse"] - want["lse"]) <= want["bound"]["lse"]).all()
