"""The head's losses against float64, within bounds derived for each value: both types, both targets, sizes around the
tiles, lists of every kind, options, strides, what lies in rows that are left out, and numbers at the edges."""
import pytest
import torch

from oracle import head_oracle as orc

pytestmark = pytest.mark.gpu

STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of a rounding


@pytest.fixture(scope="module")
def B():
    from paper_2404_15159_b200 import binding
    return binding


def rand(seed, t, v, d, dtype, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn(v, d, generator=g, device="cuda") * spread * d ** -0.5).to(dtype)
    x = torch.randn(t, d, generator=g, device="cuda").to(dtype)
    return g, x, w


def lists(g, t, v, top, ragged=True):
    keys = torch.rand(t, v, generator=g, device="cuda")
    index = torch.topk(keys, min(top, v), 1).indices.to(torch.int32)
    if index.shape[1] < top:
        index = torch.cat([index, torch.full((t, top - index.shape[1]), -1, dtype=torch.int32, device="cuda")], 1)
    if ragged:
        kept = torch.randint(0, 2 * top, (t, 1), generator=g, device="cuda")
        index = torch.where(torch.arange(top, device="cuda")[None] >= kept, torch.full_like(index, -1), index)
    return index.contiguous(), 3 * torch.randn(t, top, generator=g, device="cuda")


def run(B, x, w, target, logit=None, t_lse=None, weights=None, normalizer=None, grad=True, ws=None, d_x=None, stream=None,
        **opt):
    t, d = x.shape
    dtype = B.MIXLORA_DTYPE_BF16 if x.dtype == torch.bfloat16 else B.MIXLORA_DTYPE_FP32
    if grad and d_x is None:
        d_x = torch.full((t, d), float("nan"), dtype=x.dtype, device=x.device)
    shape = B.make_head_shape(t, d, w.shape[0], dtype, teacher_top=0 if logit is None else target.shape[1],
                              x_stride=x.stride(0), w_stride=w.stride(0), d_x_stride=d_x.stride(0) if grad else 0, **opt)
    ws = B.alloc_head_workspace(shape, grad, device=x.device) if ws is None else ws
    o = dict(loss=torch.full((t,), float("nan"), device=x.device), lse=torch.full((t,), float("nan"), device=x.device),
             totals=torch.full((2,), float("nan"), device=x.device))
    tail = (weights, normalizer, o["loss"], o["lse"], o["totals"], d_x if grad else None, ws)
    if logit is None:
        B.mixlora_head_loss(shape, x, w, target, *tail, stream=stream)
    else:
        B.mixlora_head_distill(shape, x, w, target, logit, t_lse, *tail, stream=stream)
    if grad:
        o["d_x"] = d_x
    o["ws"] = ws
    return o


def want(x, w, target, logit=None, t_lse=None, **opt):
    rows = (orc.label_rows(target, w.shape[0]) if logit is None else
            orc.teacher(target, logit, w.shape[0], opt.get("temperature", 1.0), t_lse))
    step = STEP[x.dtype]
    # an fp32 factor is the product of a few rounded ones
    return orc.head(x, w, *rows, p_step=step if x.dtype == torch.bfloat16 else 2.0 ** -21, out_step=step, **opt)


def check(B, got, ref):
    torch.cuda.synchronize()
    assert B.mixlora_device_status(got["ws"]) == 0
    for n in ("loss", "lse", "totals", "d_x"):
        if n in got and n in ref:
            off, bound = (got[n].double() - ref[n]).abs(), ref["bound"][n]
            assert bool((off <= bound).all()), f"{n}: {float((off / bound.clamp_min(1e-300)).max()):.2f} of its bound"


SIZES = [(1, 1, 8), (1, 300, 64), (5, 2, 72), (130, 255, 64), (129, 256, 128), (300, 257, 200), (257, 1000, 264), (513, 2051, 64),
         (64, 5003, 512)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("grad", [True, False], ids=["grad", "loss"])
@pytest.mark.parametrize("t,v,d", SIZES)
def test_labels(B, t, v, d, grad, dtype):
    g, x, w = rand(1, t, v, d, dtype, 3.0)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    if t > 4:
        labels[::3] = torch.tensor([-100, v, -1, 1 << 30], device="cuda", dtype=torch.int32).repeat(t)[: (t + 2) // 3]
    check(B, run(B, x, w, labels, grad=grad), want(x, w, labels, gradient=grad))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("grad", [True, False], ids=["grad", "loss"])
@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
@pytest.mark.parametrize("t,v,d,top", [(1, 1, 8, 1), (3, 300, 64, 7), (5, 2, 72, 5), (130, 255, 64, 33), (300, 257, 200, 256),
                                       (257, 1000, 264, 20), (70, 2051, 64, 64), (33, 40, 64, 100)])
def test_lists(B, t, v, d, top, tail, grad, dtype):
    g, x, w = rand(2, t, v, d, dtype, 2.0)
    index, logit = lists(g, t, v, top)
    index[0, 0] = 0
    u = torch.logsumexp(logit, 1) + 0.7 if tail else None
    opt = dict(temperature=1.5, z_loss=0.01)
    t_lse = None if u is None else (u / 1.5).contiguous()
    check(B, run(B, x, w, index, logit, t_lse, grad=grad, **opt), want(x, w, index, logit, t_lse, gradient=grad, **opt))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("top", [0, 9])
@pytest.mark.parametrize("opt", [dict(softcap=5.0), dict(softcap=0.5, scale=2.0), dict(scale=0.25), dict(temperature=3.0),
                                 dict(z_loss=0.2, softcap=30.0, temperature=0.7, scale=1.5)])
def test_options(B, opt, top, dtype):
    t, v, d = 150, 700, 128
    g, x, w = rand(3, t, v, d, dtype, 3.0)
    weights = torch.rand(t, generator=g, device="cuda") - 0.2
    norm = torch.tensor([37.5], device="cuda")
    if top:
        index, logit = lists(g, t, v, top)
        args = (index, logit, torch.logsumexp(logit / opt.get("temperature", 1.0), 1) + 0.3)
    else:
        args = (torch.randint(-40, v, (t,), generator=g, device="cuda", dtype=torch.int32),)
    check(B, run(B, x, w, *args, weights=weights, normalizer=norm, **opt),
          want(x, w, *args, weights=weights, normalizer=37.5, **opt))


def test_order_and_repeats_of_a_list_are_free(B):
    g, x, w = rand(4, 40, 600, 64, torch.bfloat16, 2.0)
    index, logit = lists(g, 40, 600, 12, ragged=False)
    twice = torch.cat([index, index[:, :5]], 1)
    more = torch.cat([logit, torch.randn(40, 5, generator=g, device="cuda")], 1)
    order = torch.randperm(17, generator=g, device="cuda")
    a = run(B, x, w, twice, more)
    b = run(B, x, w, twice[:, order].contiguous(), more[:, order].contiguous())
    check(B, a, want(x, w, twice, more))
    check(B, b, want(x, w, twice, more))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("t", [200, 40])
def test_strided_rows_and_garbage_where_nothing_counts(B, t, dtype):
    v, d = 900, 96
    g, x, w = rand(5, t, v, d, dtype, 2.0)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    labels[torch.rand(t, generator=g, device="cuda") < 0.5] = -1
    wide_x = torch.full((t, d + 40), float("nan"), dtype=dtype, device="cuda")
    wide_w = torch.full((v, d + 8), float("nan"), dtype=dtype, device="cuda")
    wide_o = torch.full((t, d + 16), 7.0, dtype=dtype, device="cuda")
    wide_x[:, 8:d + 8], wide_w[:, :d] = x, w
    wide_x[labels < 0] = float("inf")
    got = run(B, wide_x[:, 8:d + 8], wide_w[:, :d], labels, d_x=wide_o[:, :d])
    x = torch.where((labels < 0)[:, None], torch.zeros_like(x), x)
    check(B, got, want(x, w, labels))
    assert (wide_o[:, d:] == 7.0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_a_batch_without_labels(B, dtype):
    _, x, w = rand(6, 70, 300, 64, dtype)
    got = run(B, x, w, torch.full((70,), -1, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for n in ("loss", "lse", "totals", "d_x"):
        assert (got[n] == 0).all()
    got = run(B, x, w, torch.full((70, 3), -1, dtype=torch.int32, device="cuda"), torch.zeros(70, 3, device="cuda"))
    for n in ("loss", "lse", "totals", "d_x"):
        assert (got[n] == 0).all()
    shape = B.make_head_shape(0, 64, 300)
    totals = torch.ones(2, device="cuda")
    ws = B.alloc_head_workspace(shape, True)
    B.mixlora_head_loss(shape, x, w, totals, None, None, totals, None, totals, w, ws)
    assert (totals == 0).all() and B.mixlora_device_status(ws) == 0


def test_a_normalizer_of_zero_gives_no_gradient(B):
    g, x, w = rand(7, 20, 300, 64, torch.bfloat16)
    labels = torch.randint(0, 300, (20,), generator=g, device="cuda", dtype=torch.int32)
    got = run(B, x, w, labels, weights=torch.zeros(20, device="cuda"))
    torch.cuda.synchronize()
    assert (got["d_x"] == 0).all() and (got["totals"] == 0).all() and (got["loss"] > 0).all()
    got = run(B, x, w, labels, normalizer=torch.zeros(1, device="cuda"))
    assert (got["d_x"] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_far_logits_in_every_place(B, dtype):
    # tiles of a row far apart from one another, so that their references differ, up and down; labels at the top and below
    t, v, d = 64, 1500, 64
    g, x, w = rand(8, t, v, d, dtype)
    lift = torch.zeros(v, device="cuda")
    lift[100], lift[300], lift[700:760], lift[1400] = 30.0, 80.0, -90.0, 55.0
    x[:, 0] = torch.linspace(-3, 3, t, device="cuda").to(dtype)
    w[:, 0] = lift.to(dtype)
    labels = torch.tensor([100, 300, 701, 1400, 5], dtype=torch.int32, device="cuda").repeat(t)[:t].contiguous()
    check(B, run(B, x, w, labels), want(x, w, labels))
    index = torch.tensor([300, 5, 701, 1400], dtype=torch.int32, device="cuda").repeat(t, 1)
    logit = 2 * torch.randn(t, 4, generator=g, device="cuda")
    check(B, run(B, x, w, index, logit), want(x, w, index, logit))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_a_sure_token_keeps_its_small_loss_and_gradient(B, dtype):
    t, v, d = 32, 800, 64
    g, x, w = rand(9, t, v, d, dtype)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    lean = torch.linspace(0, 40, t, device="cuda")[:, None]
    wl = w[labels.long()].float()
    x = (x.float() + lean * wl / (wl * wl).sum(1, keepdim=True)).to(dtype)
    got, ref = run(B, x, w, labels), want(x, w, labels)
    check(B, got, ref)
    assert float(ref["loss"].min()) < 1e-10         # e^-40, times 800 columns, some of which lean the same way
    # relatively, row by row: logits of a few tens are off by less than 2^-12 here
    rel = ((got["loss"].double() - ref["loss"]).abs() / ref["loss"]).max()
    assert float(rel) < 2.0 ** -10
    size = ref["d_x"].abs().max(1).values
    assert float(((got["d_x"].double() - ref["d_x"]).abs().max(1).values / size).max()) < (2.0 ** -6 if dtype == torch.bfloat16 else 2.0 ** -10)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_row_that_is_no_number_stays_alone(B, bad, dtype):
    g, x, w = rand(10, 40, 300, 64, dtype)
    labels = torch.randint(0, 300, (40,), generator=g, device="cuda", dtype=torch.int32)
    x[7, 3] = bad
    got = run(B, x, w, labels)
    keep = torch.arange(40, device="cuda") != 7
    torch.cuda.synchronize()
    assert got["loss"][7].isnan() and got["d_x"][7].isnan().any() and got["totals"][0].isnan()
    x[7] = 0
    ref = want(x, w, labels)
    for n in ("loss", "lse", "d_x"):
        off = (got[n].double() - ref[n]).abs()[keep]
        assert bool((off <= ref["bound"][n][keep]).all())


def test_teacher_logits_at_the_edges(B):
    g, x, w = rand(11, 12, 300, 64, torch.bfloat16)
    index, logit = lists(g, 12, 300, 4, ragged=False)
    inf = float("inf")
    logit[1, 1:] = -inf
    logit[2] = -inf                    # says nothing: left out
    logit[3] *= 1000
    check(B, run(B, x, w, index, logit), want(x, w, index, logit))
    t_lse = torch.logsumexp(logit, 1) + 0.1
    t_lse[2] = 0.0                     # the teacher chose none of these: everything is left over
    t_lse[4] = t_lse[4] - 1.0          # listed entries above one: nothing is left over
    check(B, run(B, x, w, index, logit, t_lse), want(x, w, index, logit, t_lse))
    logit[5, 2] = float("nan")
    got = run(B, x, w, index, logit)
    torch.cuda.synchronize()
    assert got["loss"][5].isnan() and got["loss"].isnan().sum() == 1 and got["d_x"].isnan().any(1).sum() == 1


@pytest.mark.parametrize("grad", [True, False], ids=["grad", "loss"])
@pytest.mark.parametrize("t,v,d,top,softcap", [(16, 40001, 64, 0, 0.0), (17, 19300, 1096, 0, 8.0), (32, 700, 2056, 40, 0.0),
                                               (33, 20011, 1032, 256, 5.0), (64, 40001, 136, 9, 0.0), (65, 20011, 1032, 33, 5.0),
                                               (258, 38000, 1096, 3, 0.0)])
def test_many_tiles_and_spans(B, t, v, d, top, softcap, grad):
    # more tiles than a block takes at once, more reduction than one span, on both sides of the form for few tokens
    g, x, w = rand(12, t, v, d, torch.bfloat16, 3.0)
    opt = dict(softcap=softcap, z_loss=0.001)
    if top:
        index, logit = lists(g, t, v, top)
        args = (index, logit, torch.logsumexp(logit, 1) + 0.2)
    else:
        args = (torch.randint(-v // 4, v, (t,), generator=g, device="cuda", dtype=torch.int32),)
    weights = torch.rand(t, generator=g, device="cuda")
    check(B, run(B, x, w, *args, weights=weights, grad=grad, **opt), want(x, w, *args, weights=weights, gradient=grad, **opt))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("t", [64, 65, 200, 256, 257])
def test_left_out_tokens_on_both_sides_of_a_tile(B, t, top, dtype):
    # up to a tile's rows the tokens that are left out pass through the products, behind it they do not; labels just behind the
    # vocabulary fall into its last tile
    v, d = 700, 128
    g, x, w = rand(13, t, v, d, dtype, 3.0)
    out = torch.rand(t, generator=g, device="cuda") < 0.4
    out[0] = False
    x[out] = torch.tensor([float("nan"), float("inf")], device="cuda", dtype=dtype).repeat(d // 2)
    weights = torch.rand(t, generator=g, device="cuda")
    weights[out] = float("nan")
    if top:
        index, logit = lists(g, t, v, top, ragged=False)
        index[out] = v + 1
        args = (index, logit)
    else:
        labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
        labels[out] = v + 3
        args = (labels,)
    got = run(B, x, w, *args, weights=weights)
    ref = want(torch.where(out[:, None], torch.zeros_like(x), x), w, *args, weights=torch.where(out, torch.zeros_like(weights), weights))
    check(B, got, ref)
    assert (got["d_x"][out] == 0).all() and (got["loss"][out] == 0).all()
