"""Masked attention at the edges of its range: scores that jump within a tile, capped scores of every size, values that
are very large or small, what lies outside the sequences.  Cases, oracle and bounds as in test_gpu_attention.py."""
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
