"""Where the head's losses can go wrong at the edges: numbers that are none, tokens that are sure at a model's own width, both
on every side of the form for few tokens and of a tile."""
import math

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


def exact_logits(z):
    """fp32 states and head whose logits are the fp32 numbers z [t, v] themselves: a token picks its column of the head."""
    t = z.shape[0]
    d = (t + 7) // 8 * 8
    x, w = torch.zeros(t, d, device="cuda"), torch.zeros(z.shape[1], d, device="cuda")
    x[torch.arange(t), torch.arange(t)] = 1.0
    w[:, :t] = z.T
    return x, w


def test_a_small_divergence_of_exact_logits_keeps_its_digits(B):
    # every column is listed, so that no sum in 32 bits takes part: loss = sum q (ln q - z + lse) of logits and probabilities in 64.
    # The exponential's series leaves out 1e-11 relatively, the logarithm's less, where |ln of a fraction| is largest, 0.49 ln 2;
    # and the loss is rounded once.
    g = torch.Generator(device="cuda").manual_seed(42)
    t, v = 56, 64
    z = -0.49 * 0.6931 * torch.randint(0, 2, (t, v), generator=g, device="cuda").float()
    z[1::3] = 3 * torch.randn(t, v, generator=g, device="cuda")[1::3]
    z[:, 0] = 0.0
    u = z + 2.0 ** -8 * torch.randn(t, v, generator=g, device="cuda")
    x, w = exact_logits(z)
    index = torch.arange(v, dtype=torch.int32, device="cuda").repeat(t, 1)
    got = run(B, x, w, index, u, grad=False)
    log_q, log_p = torch.log_softmax(u.double(), 1), torch.log_softmax(z.double(), 1)
    loss = (log_q.exp() * (log_q - log_p)).sum(1)
    assert float(loss.max()) < 1e-3
    assert bool(((got["loss"].double() - loss).abs() <= 2.0 ** -34 + 2.0 ** -24 * loss).all())
    lse = torch.logsumexp(z.double(), 1)
    assert bool(((got["lse"].double() - lse).abs() <= 2.0 ** -34 + 2.0 ** -24 * lse.abs()).all())


def test_a_loss_of_two_exact_logits_is_rounded_once(B):
    # one other column, of logit 0, whose sum is 1 without a rounding: loss = ln(1 + e^-z), its series good to 2^-32
    z = torch.cat([torch.linspace(-85.0, 85.0, 171, device="cuda"), torch.linspace(-1.0, 1.0, 165, device="cuda")])
    x, w = exact_logits(torch.stack([z, torch.zeros_like(z)], 1))
    got = run(B, x, w, torch.zeros(z.numel(), dtype=torch.int32, device="cuda"), grad=False)
    loss = torch.nn.functional.softplus(-z.double(), threshold=1000.0)
    loss = torch.where(z > 0, torch.log1p(torch.exp(-z.double())), loss)
    assert bool(((got["loss"].double() - loss).abs() <= (2.0 ** -24 + 2.0 ** -31) * loss + 2.0 ** -149).all())
    lse = torch.nn.functional.softplus(z.double(), threshold=1000.0)
    assert bool(((got["lse"].double() - lse).abs() <= (2.0 ** -24 + 2.0 ** -31) * lse + 2.0 ** -31 * z.double().abs()).all())


@TYPES
@TOKENS
@pytest.mark.parametrize("kind", ["labels", "listed", "tail"])
@pytest.mark.parametrize("softcap", [0.0, 4.0])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_a_token_that_is_no_number_says_so_and_stays_alone(B, bad, softcap, kind, t, dtype):
    # a cap makes numbers of infinite products, and an exponential a zero of those below: neither hides them
    v = 300
    g, x, w = rand(43, t, v, 64, dtype)
    args = targets(kind, g, t, v)
    x[7, 3], x[t - 1, 60] = bad, bad
    out = torch.tensor([7, t - 1], device="cuda")
    keep = torch.ones(t, dtype=torch.bool, device="cuda").index_fill(0, out, False)
    norm = torch.full((1,), float(t), device="cuda")
    got = run(B, x, w, *args, softcap=softcap, normalizer=norm)
    torch.cuda.synchronize()
    for n in ("loss", "lse", "d_x"):
        assert got[n][out].isnan().all(), n
    assert got["totals"][0].isnan() and got["totals"][1] == t
    x[out] = 0
    ref = want(x, w, *args, softcap=softcap, normalizer=float(t))
    for n in ("loss", "lse", "d_x"):
        off = (got[n].double() - ref[n]).abs()[keep]
        assert bool((off <= ref["bound"][n][keep]).all()), n


@TYPES
@TOKENS
@pytest.mark.parametrize("kind", ["labels", "listed", "tail"])
@pytest.mark.parametrize("softcap", [0.0, 4.0])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_a_head_that_is_no_number_reaches_every_token(B, bad, softcap, kind, t, dtype):
    v = 300
    g, x, w = rand(44, t, v, 64, dtype)
    args = targets(kind, g, t, v)
    args[0][:2] = 17                       # listed for some, not for others
    args[0][2] = -1                        # left out
    w[17, 5] = bad
    for grad in (True, False):
        got = run(B, x, w, *args, softcap=softcap, grad=grad)
        torch.cuda.synchronize()
        for n in ("loss", "lse", "d_x")[: 3 if grad else 2]:
            keep = torch.arange(t, device="cuda") != 2
            assert got[n][keep].isnan().all() and (got[n][2] == 0).all(), n


@TYPES
@pytest.mark.parametrize("bad", [INF, -INF])
def test_one_column_of_infinite_logits(B, bad, dtype):
    g, x, w = rand(45, 3, 1, 64, dtype)
    x[1] = torch.sign(w[0].float()).to(dtype) * bad
    got = run(B, x, w, torch.zeros(3, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert got["loss"].isnan().tolist() == [False, True, False] and got["d_x"].isnan().any(1).tolist() == [False, True, False]


# units of 2^-23 of a logit that the spans of its sum may cost it: a step of 16 products cuts off less than one unit of what has
# been added up, half of one on the average, and over a span of n steps that has grown to (n + 1) / 2 steps' worth on the average.
# Few tokens have spans of 128 products; tiles longer ones that go up and down in turns, or else 256
SPANS = {40: 8, 300: 16}               # steps of a span


def cut_off(t):
    return 0.5 * (SPANS[t] + 1) / 2 * 2.0 ** -23


@pytest.mark.parametrize("t", [40, 300])
def test_a_logit_loses_less_than_its_spans_cut_off(B, t):
    # one column: the log-sum-exp is the logit.  Its products lean one way, as those of a sure token with its label do, so that
    # what is cut off adds up; what rounds either way goes down with the number of logits (4096 products: below 2 units each).
    # Sums between two powers of two lose up to twice as much as those just below one: the widths take both
    g = torch.Generator(device="cuda").manual_seed(46)
    for d in (1024, 1104, 1536, 2560, 4096, 4416):
        off, n = 0.0, 0
        for _ in range(10):
            w = torch.randn(1, d, generator=g, device="cuda")
            x = (torch.randn(t, d, generator=g, device="cuda") + 0.3 * w).bfloat16()
            w = w.bfloat16()
            got = run(B, x, w, torch.zeros(t, dtype=torch.int32, device="cuda"), grad=False)
            z = (x.double() @ w.double().T)[:, 0]
            off += float(((got["lse"].double() - z) / z.mean()).sum())
            n += t
        assert abs(off / n) <= cut_off(t) + 2 * 2.0 ** -23 * n ** -0.5, (d, off / n * 2 ** 23)


@pytest.mark.parametrize("t", [40, 300])
def test_a_sure_token_at_a_models_width_keeps_its_loss(B, t):
    # loss = e^(lse of the others - z): relatively it is off by what the logits are off by.  The label's logit is about 30, that
    # of the columns that matter beside it about 4 (their spread is 2), with either sign of what is cut off; exponentials and
    # sums add 2^-21
    v, d = 32000, 4096
    g, x, w = rand(47, t, v, d, torch.bfloat16, 2.0)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    wl = w[labels.long()].float()
    x = (x.float() + 30.0 * wl / (wl * wl).sum(1, keepdim=True)).bfloat16()
    got = run(B, x, w, labels, grad=False)
    z = torch.empty(t, device="cuda", dtype=torch.float64)
    ref = torch.empty_like(z)
    for a in range(0, t, 50):
        all_z = x[a:a + 50].double() @ w.double().T
        z[a:a + 50] = torch.gather(all_z, 1, labels[a:a + 50].long()[:, None])[:, 0]
        others = torch.logsumexp(all_z.scatter(1, labels[a:a + 50].long()[:, None], -INF), 1)
        ref[a:a + 50] = torch.log1p(torch.exp(others - z[a:a + 50]))
    off = (got["loss"].double() - ref) / ref
    assert float(ref.max()) < 1e-2
    assert abs(float(off.mean())) <= cut_off(t) * (float(z.mean()) + 4.0) + 2.0 ** -21, float(off.mean())


@TYPES
@TOKENS
@pytest.mark.parametrize("given", [False, True], ids=["own", "given"])
@pytest.mark.parametrize("size", [2.0 ** -140, 2.0 ** 120])
def test_weights_of_any_size_divide_out(B, size, given, t, dtype):
    # one over a sum of 2^-137 is no fp32 number, and one over 2^127 has few bits; weight / normalizer is a number like any other
    g, x, w = rand(48, t, 300, 64, dtype)
    labels = torch.randint(0, 300, (t,), generator=g, device="cuda", dtype=torch.int32)
    weights = size * torch.randint(1, 4, (t,), generator=g, device="cuda").float() / (t if size > 1 else 1)
    norm = torch.tensor([size * 5], device="cuda") if given else None
    got = run(B, x, w, labels, weights=weights, normalizer=norm)
    ref = want(x, w, labels, weights=weights, normalizer=size * 5 if given else None)
    check(B, got, {n: ref[n] for n in ("loss", "lse", "d_x", "bound")})


MORE = pytest.mark.parametrize("t", [130, 300])            # the form for more than 64 tokens


@TYPES
@MORE
def test_far_logits_in_every_place_of_a_tile(B, t, dtype):
    v, d = 1500, 64
    g, x, w = rand(49, t, v, d, dtype)
    lift = torch.zeros(v, device="cuda")
    lift[100], lift[300], lift[700:760], lift[1400] = 30.0, 80.0, -90.0, 55.0
    x[:, 0] = torch.linspace(-3, 3, t, device="cuda").to(dtype)
    w[:, 0] = lift.to(dtype)
    labels = torch.tensor([100, 300, 701, 1400, 5], dtype=torch.int32, device="cuda").repeat(t)[:t].contiguous()
    check(B, run(B, x, w, labels), want(x, w, labels))
    index = torch.tensor([300, 5, 701, 1400], dtype=torch.int32, device="cuda").repeat(t, 1)
    logit = 2 * torch.randn(t, 4, generator=g, device="cuda")
    check(B, run(B, x, w, index, logit), want(x, w, index, logit))


@TYPES
@MORE
def test_a_sure_token_in_a_tile_keeps_its_small_loss_and_gradient(B, t, dtype):
    # relatively, row by row: logits of a few tens, sums of 64 products, are off by less than 2^-12 here, and what rounds the
    # gradient's factors and itself comes to less than four half steps of bf16
    v, d = 800, 64
    g, x, w = rand(50, t, v, d, dtype)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    lean = torch.linspace(0, 40, t, device="cuda")[:, None]
    wl = w[labels.long()].float()
    x = (x.float() + lean * wl / (wl * wl).sum(1, keepdim=True)).to(dtype)
    got, ref = run(B, x, w, labels), want(x, w, labels)
    check(B, got, ref)
    assert float(ref["loss"].min()) < 1e-10
    rel = ((got["loss"].double() - ref["loss"]).abs() / ref["loss"]).max()
    assert float(rel) < 2.0 ** -10
    size = ref["d_x"].abs().max(1).values
    assert float(((got["d_x"].double() - ref["d_x"]).abs().max(1).values / size).max()) < (2.0 ** -6 if dtype == torch.bfloat16 else 2.0 ** -10)


@TYPES
@MORE
def test_teacher_logits_at_the_edges_of_a_tile(B, t, dtype):
    g, x, w = rand(51, t, 300, 64, dtype)
    index, logit = lists(g, t, 300, 4, ragged=False)
    last = t - 7                          # the same edges among the first rows and the last
    for a in (0, last):
        logit[a + 1, 1:] = -INF
        logit[a + 2] = -INF               # says nothing: left out
        logit[a + 3] *= 1000
    check(B, run(B, x, w, index, logit), want(x, w, index, logit))
    t_lse = torch.logsumexp(logit, 1) + 0.1
    for a in (0, last):
        t_lse[a + 2] = 0.0                # the teacher chose none of these: everything is left over
        t_lse[a + 4] = t_lse[a + 4] - 1.0  # listed entries above one: nothing is left over
    check(B, run(B, x, w, index, logit, t_lse), want(x, w, index, logit, t_lse))
    logit[last + 5, 2] = NAN
    got = run(B, x, w, index, logit)
    torch.cuda.synchronize()
    assert got["loss"][last + 5].isnan() and got["loss"].isnan().sum() == 1 and got["d_x"].isnan().any(1).sum() == 1


@TYPES
@pytest.mark.parametrize("left_out", [False, True], ids=["all", "some"])
@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("shape,grad", [("wide", True), ("deep", True), ("deep", False)])
def test_pieces_of_every_kind(B, shape, grad, top, left_out, dtype):
    # a piece is 256 rows at the widest vocabulary, 4096 (in parts: 1280) at the greatest width; where no token is left out the rows
    # are read in place, the last piece's tiles reaching beyond the last token
    bf16 = dtype == torch.bfloat16
    t, v, d = (601, 1 << 20, 16) if shape == "wide" else (4397 if bf16 else 1399, 300, 65536)
    g, x, w = rand(52, t, v, d, dtype, 2.0)
    weights = torch.rand(t, generator=g, device="cuda") + 0.1
    out = torch.zeros(t, dtype=torch.bool, device="cuda")
    if left_out:
        out[1::3] = True
    if top:
        index = torch.randint(0, v, (t, top), generator=g, device="cuda", dtype=torch.int32)
        index[:, 1:][torch.rand(t, top - 1, generator=g, device="cuda") < 0.3] = -1
        index[out] = -1
        args = [index, 3 * torch.randn(t, top, generator=g, device="cuda")]
        args.append(torch.logsumexp(args[1], 1) + 0.4)
    else:
        labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
        args = [torch.where(out, torch.full_like(labels, -1), labels)]
    got = run(B, x, w, *args, weights=weights, grad=grad)
    torch.cuda.synchronize()
    assert B.mixlora_device_status(got["ws"]) == 0
    norm = float(weights[~out].double().sum())
    total = 0.0
    step = 50 if shape == "wide" else 400
    for a in range(0, t, step):
        rows = slice(a, a + step)
        ref = want(x[rows], w, *(v[rows] for v in args), weights=weights[rows], normalizer=norm, gradient=grad)
        total += float(ref["totals"][0])
        for n in ("loss", "lse", "d_x")[: 3 if grad else 2]:
            off = (got[n][rows].double() - ref[n]).abs()
            assert bool((off <= ref["bound"][n]).all()), (n, a)
    assert abs(float(got["totals"][0]) - total) <= 1e-5 * abs(total) and abs(float(got["totals"][1]) - norm) <= 2.0 ** -23 * norm


@TYPES
@TOKENS
@pytest.mark.parametrize("v", [5, 300])
@pytest.mark.parametrize("left", [0.01, 0.9])
def test_what_a_teacher_leaves_over_stays_beside_listed_columns_of_any_weight(B, left, v, t, dtype):
    # one listed column holds up to 2^69 times the weight of all that are not listed, and still their share of the gradient is
    # what the teacher leaves over, spread as they are
    d = 64
    g, x, w = rand(53, t, v, d, dtype)
    w[:, 0] = 0.0
    w[4, 0] = 1.0
    x[:, 0] = torch.linspace(-10.0, 46.0, t, device="cuda").to(dtype)
    index = torch.tensor([[4, 0, 2]], dtype=torch.int32, device="cuda").repeat(t, 1)
    logit = torch.randn(t, 3, generator=g, device="cuda")
    t_lse = torch.logsumexp(logit, 1) - math.log1p(-left)
    check(B, run(B, x, w, index, logit, t_lse), want(x, w, index, logit, t_lse))


@TYPES
@TOKENS
def test_a_list_of_one_entry_is_a_label(B, t, dtype):
    # to the last bit, also where the token is so sure that its loss, e^-40 and less, is no difference of logarithms any more
    v, d = 800, 64
    g, x, w = rand(54, t, v, d, dtype)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    wl = w[labels.long()].float()
    x = (x.float() + torch.linspace(0, 44, t, device="cuda")[:, None] * wl / (wl * wl).sum(1, keepdim=True)).to(dtype)
    a = run(B, x, w, labels, z_loss=1e-3)
    index = torch.full((t, 3), -1, dtype=torch.int32, device="cuda")
    index[torch.arange(t), torch.arange(t) % 3] = labels
    b = run(B, x, w, index, torch.randn(t, 3, generator=g, device="cuda"), z_loss=1e-3)
    assert all(torch.equal(a[n], b[n]) for n in ("loss", "lse", "totals", "d_x"))
    b = run(B, x, w, index, torch.randn(t, 3, generator=g, device="cuda"))
    check(B, b, want(x, w, index, torch.zeros(t, 3, device="cuda")))


@TOKENS
@pytest.mark.parametrize("softcap", [0.0, 4.0])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_no_number_is_lost_in_a_sum_of_many_spans(B, bad, softcap, t):
    # wherever in the reduction it stands: spans that go up, that go down, and the last one
    v, d = 300, 2376
    g, x, w = rand(55, t, v, d, torch.bfloat16)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    out = torch.arange(3, 3 + 12 * 3, 3, device="cuda")
    x[out, torch.arange(12, device="cuda") * 215 + 7] = bad
    got = run(B, x, w, labels, softcap=softcap, normalizer=torch.full((1,), float(t), device="cuda"))
    torch.cuda.synchronize()
    keep = torch.ones(t, dtype=torch.bool, device="cuda").index_fill(0, out, False)
    for n in ("loss", "lse", "d_x"):
        assert got[n][out].isnan().all() and not got[n][keep].isnan().any(), n
