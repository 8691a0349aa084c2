"""Where the head's losses can go wrong at the edges: numbers that are none, tokens that are sure at a model's own width, both
on every side of the form for few tokens and of a tile."""
import pytest
import torch

from test_gpu_head import check, lists, rand, run, want

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
TOKENS = pytest.mark.parametrize("t", [40, 130, 300])      # few tokens, less than a tile's rows, more
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def B():
    from paper_2404_15159_b200 import binding
    return binding


def targets(kind, g, t, v):
    if kind == "labels":
        return (torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32),)
    index, logit = lists(g, t, v, 6, ragged=False)
    return (index, logit) if kind == "listed" else (index, logit, torch.logsumexp(logit, 1) + 0.3)


@TYPES
@TOKENS
@pytest.mark.parametrize("kind", ["listed", "tail"])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_the_lse_of_a_row_that_is_no_number_is_none(B, bad, kind, t, dtype):
    g, x, w = rand(40, t, 300, 64, dtype)
    args = targets(kind, g, t, 300)
    x[7, 3] = bad
    got = run(B, x, w, *args)
    torch.cuda.synchronize()
    assert got["lse"][7].isnan() and got["lse"].isnan().sum() == 1


@TOKENS
@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
def test_the_lse_of_a_listed_logit_that_is_infinite_is_no_number(B, tail, t):
    # the listed column alone has no bounds: the difference from the largest logit, inf - inf, is formed in 64 bits
    g, x, w = rand(41, t, 300, 64, torch.bfloat16)
    x[:, 3], w[5, 3] = 1.0, INF
    index = torch.tensor([[9, 5, 200]], dtype=torch.int32, device="cuda").repeat(t, 1)
    logit = torch.randn(t, 3, generator=g, device="cuda")
    got = run(B, x, w, index, logit, torch.logsumexp(logit, 1) + 0.3 if tail else None)
    torch.cuda.synchronize()
    assert got["lse"].isnan().all() and got["loss"].isnan().all()
