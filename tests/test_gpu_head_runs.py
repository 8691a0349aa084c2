"""The head's losses as a program runs them: behind the last layer of a training step, over shards of a batch, in pieces, on
several streams, captured, at far offsets, and the same bits every time."""
import numpy as np
import pytest
import torch

import helpers
from oracle import head_oracle as hd
from oracle import mixlora_oracle as orc
from paper_2404_15159_b200 import synth
from test_gpu_head import check, lists, rand, run, want

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])


@pytest.fixture(scope="module")
def B():
    from paper_2404_15159_b200 import binding
    return binding


@TYPES
@pytest.mark.parametrize("top", [0, 6], ids=["labels", "teacher"])
def test_training_step_of_a_layer_and_the_loss(B, top, dtype):
    # layer forward, loss and its gradient, layer backward down to the LoRA matrices and the layer's input, against the same
    # in float64; the norms this library's layers are held to: 1e-4 in fp32, 2e-2 in bf16 (largest error over largest value).
    # Every expert takes part in every token, so that no routing decision is near a border.
    bf16 = dtype == torch.bfloat16
    T, d, f, N, r, V, eps, alpha = 90, 128, 192, 2, 8, 777, 1e-5, 16.0
    rng = np.random.default_rng(21)
    rnd = synth.round_to_bf16 if bf16 else (lambda a: np.asarray(a, np.float32).astype(np.float64))
    t = dict(x=rnd(rng.standard_normal((T, d))), router_bias=None,
             w_router=np.asarray(rng.standard_normal((N, d)) * 0.1, np.float32).astype(np.float64))
    for n, (o, i) in dict(gate=(f, d), up=(f, d), down=(d, f)).items():
        t["w_" + n] = rnd(rng.standard_normal((o, i)) * i ** -0.5)
        t["a_" + n] = rnd(rng.standard_normal((N, r, i)) * i ** -0.5)
        t["b_" + n] = rnd(rng.standard_normal((N, o, r)) * 0.1)
    wn = rnd(1 + 0.2 * rng.standard_normal(d))
    head = rnd(rng.standard_normal((V, d)) * d ** -0.5)
    labels = rng.integers(-200, V, T)
    index, logit = rng.integers(-1, V, (T, max(top, 1))), 2 * rng.standard_normal((T, max(top, 1)))
    logit = np.asarray(logit, np.float32).astype(np.float64)

    act = {n: (None if v is None else torch.from_numpy(np.ascontiguousarray(v)).cuda().to(
        torch.float32 if n == "w_router" else dtype)) for n, v in t.items()}
    code = B.MIXLORA_DTYPE_BF16 if bf16 else B.MIXLORA_DTYPE_FP32
    shape = B.make_shape(T, d, f, N, N, r, alpha, code)
    params = B.make_params(**act)
    ws = B.alloc_workspace(shape, True)
    xn, inv, h = torch.empty_like(act["x"]), torch.empty(T, device="cuda"), torch.empty_like(act["x"])
    g_wn, g_head = (torch.from_numpy(v).cuda().to(dtype) for v in (wn, head))
    B.mixlora_layer_forward(shape, params, g_wn, eps, xn, inv, h, ws)
    g_index, g_labels = (torch.from_numpy(v).cuda().to(torch.int32).contiguous() for v in (index, labels))
    g_logit = torch.from_numpy(logit).cuda().float()
    o = run(B, h, g_head, g_index, g_logit) if top else run(B, h, g_head, g_labels)
    g = {n: torch.full(tuple(np.shape(t[n[2:]])), float("nan"), device="cuda") for n in helpers.GRAD_NAMES if n != "d_router_bias"}
    g["d_x"] = torch.empty_like(act["x"])
    B.mixlora_layer_backward(shape, params, g_wn, eps, xn, inv, o["d_x"], 0.0, ws, B.make_grads(accumulate=0, **g))
    torch.cuda.synchronize()
    assert B.mixlora_device_status(ws) == 0 and B.mixlora_device_status(o["ws"]) == 0

    p = {n: v for n, v in t.items() if n != "x"}
    wh, rest = orc.layer_forward(t["x"], p, wn, eps, N, alpha)
    rows = (hd.teacher(torch.from_numpy(index), torch.from_numpy(logit), V) if top else
            hd.label_rows(torch.from_numpy(labels), V))
    ref = hd.head(torch.from_numpy(wh), torch.from_numpy(head), *rows)
    back = orc.layer_backward(t["x"], p, wn, ref["d_x"].numpy(), rest)
    got = dict(loss=o["loss"], h=h, **g)
    wanted = dict(loss=ref["loss"].numpy(), h=wh, **{n: back[n] for n in g})
    for n, v in got.items():
        e = helpers.rel_err(v.double().cpu().numpy(), wanted[n])
        assert e <= (2e-2 if bf16 else 1e-4), f"{n}: {e:.2e}"


@TYPES
def test_shards_with_one_normalizer_add_up_to_the_batch(B, dtype):
    g, x, w = rand(31, 300, 900, 64, dtype, 2.0)
    labels = torch.randint(-300, 900, (300,), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.rand(300, generator=g, device="cuda")
    whole = want(x, w, labels, weights=weights)
    norm = whole["totals"][1:].float()
    parts = [run(B, x[a:b], w, labels[a:b].contiguous(), weights=weights[a:b].contiguous(), normalizer=norm)
             for a, b in ((0, 200), (200, 300))]
    totals = sum(p["totals"].double() for p in parts)
    assert bool(((totals - whole["totals"]).abs() <= whole["bound"]["totals"] + 2.0 ** -22 * whole["totals"].abs()).all())
    d_x = torch.cat([p["d_x"] for p in parts]).double()
    # the normalizer itself was rounded once more
    assert bool(((d_x - whole["d_x"]).abs() <= whole["bound"]["d_x"] + 2.0 ** -23 * whole["d_x"].abs()).all())


@TYPES
@pytest.mark.parametrize("grad", [True, False], ids=["grad", "loss"])
def test_a_batch_in_several_pieces(B, grad, dtype):
    # the widest vocabulary: a piece is 256 counted rows there (a third of the tokens are left out)
    t, v, d = 900, 1 << 20, 16
    g, x, w = rand(32, t, v, d, dtype, 2.0)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    labels[1::3] = -1
    got = run(B, x, w, labels, grad=grad)
    torch.cuda.synchronize()
    assert B.mixlora_device_status(got["ws"]) == 0
    count = int((labels >= 0).sum())
    total = 0.0
    for a in range(0, t, 50):
        ref = want(x[a:a + 50], w, labels[a:a + 50], normalizer=count, gradient=grad)
        total += float(ref["totals"][0])
        for n in ("loss", "lse", "d_x")[: 3 if grad else 2]:
            off = (got[n][a:a + 50].double() - ref[n]).abs()
            assert bool((off <= ref["bound"][n]).all()), n
    assert abs(float(got["totals"][0]) - total) <= 1e-5 * total and float(got["totals"][1]) == count


@TYPES
def test_rows_far_apart(B, dtype):
    # more than 2^32 bytes and 2^31 values from the first row to the last, in x, w and d_x
    t, v, d, step = 270, 300, 64, 1 << 23
    g, x, w = rand(33, t, v, d, dtype, 2.0)
    labels = torch.randint(-20, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    far = [torch.empty((n - 1) * step + d, dtype=dtype, device="cuda").as_strided((n, d), (step, 1)) for n in (t, v, t)]
    far[0].copy_(x)
    far[1].copy_(w)
    far[2].fill_(7.0)
    check(B, run(B, far[0], far[1], labels, d_x=far[2]), want(x, w, labels))
    few = 5
    check(B, run(B, far[0][-few:], far[1], labels[-few:].contiguous(), d_x=far[2][-few:]), want(x[-few:], w, labels[-few:]))


CALLS = [(40, 0, torch.bfloat16), (50, 5, torch.bfloat16), (300, 0, torch.bfloat16), (600, 7, torch.bfloat16),
         (300, 4, torch.float32)]


@pytest.mark.parametrize("t,top,dtype", CALLS)
def test_calls_on_two_streams_and_the_same_bits(B, t, top, dtype):
    g, x, w = rand(34, t, 5001, 320, dtype, 2.0)
    args = lists(g, t, 5001, top) if top else (torch.randint(-900, 5001, (t,), generator=g, device="cuda", dtype=torch.int32),)
    first = run(B, x, w, *args)
    check(B, first, want(x, w, *args))
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.empty_like(first["ws"]) for _ in streams]
    torch.cuda.synchronize()
    outs = []
    for _ in range(8):
        for s, ws in zip(streams, spaces):
            with torch.cuda.stream(s):
                outs.append(run(B, x, w, *args, ws=ws))
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(o[n], first[n]) for n in ("loss", "lse", "totals", "d_x"))


@pytest.mark.parametrize("t,top,dtype", CALLS)
def test_captured_calls_follow_their_inputs(B, t, top, dtype):
    # two captured calls with a workspace each, replayed at once; then new hidden states and targets in the same buffers
    g, x, w = rand(35, t, 3001, 256, dtype, 2.0)

    def targets():
        return list(lists(g, t, 3001, top)) if top else [torch.randint(-900, 3001, (t,), generator=g, device="cuda", dtype=torch.int32)]

    args = targets()
    run(B, x, w, *args)
    streams = [torch.cuda.Stream() for _ in range(2)]
    made = []
    torch.cuda.synchronize()
    for s in streams:
        graph = torch.cuda.CUDAGraph()
        d_x, code = torch.empty_like(x), (B.MIXLORA_DTYPE_BF16 if dtype == torch.bfloat16 else B.MIXLORA_DTYPE_FP32)
        shape = B.make_head_shape(t, 256, 3001, code, teacher_top=top)
        o = dict(loss=torch.empty(t, device="cuda"), lse=torch.empty(t, device="cuda"), totals=torch.empty(2, device="cuda"),
                 d_x=d_x, ws=B.alloc_head_workspace(shape, True))
        with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
            tail = (None, None, o["loss"], o["lse"], o["totals"], d_x, o["ws"])
            if top:
                B.mixlora_head_distill(shape, x, w, args[0], args[1], None, *tail)
            else:
                B.mixlora_head_loss(shape, x, w, args[0], *tail)
        made.append((graph, o))
    for turn in range(3):
        if turn:
            x.copy_(torch.randn(t, 256, generator=g, device="cuda"))
            for old, new in zip(args, targets()):
                old.copy_(new)
        for _, o in made:
            for n in ("loss", "lse", "totals", "d_x"):
                o[n].fill_(float("nan"))
        torch.cuda.synchronize()
        for s, (graph, _) in zip(streams, made):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        ref = want(x, w, *args)
        for _, o in made:
            check(B, o, ref)


def test_calls_of_different_shapes_share_a_workspace_in_turn(B):
    g, x, w = rand(36, 700, 4001, 128, torch.bfloat16, 2.0)
    shape = B.make_head_shape(700, 128, 4001, teacher_top=256)
    ws = B.alloc_head_workspace(shape, True)
    for t, top, grad in ((700, 0, True), (3, 0, False), (64, 9, True), (65, 256, True), (700, 3, False), (1, 0, True)):
        args = lists(g, t, 4001, top) if top else (torch.randint(0, 4001, (t,), generator=g, device="cuda", dtype=torch.int32),)
        check(B, run(B, x[:t], w, *args, ws=ws, grad=grad), want(x[:t], w, *args, gradient=grad))


@pytest.mark.parametrize("t,top,dtype", CALLS)
def test_outputs_that_nobody_wants(B, t, top, dtype):
    g, x, w = rand(37, t, 2001, 128, dtype, 2.0)
    args = lists(g, t, 2001, top) if top else (torch.randint(-900, 2001, (t,), generator=g, device="cuda", dtype=torch.int32),)
    full = run(B, x, w, *args)
    code = B.MIXLORA_DTYPE_BF16 if dtype == torch.bfloat16 else B.MIXLORA_DTYPE_FP32
    shape = B.make_head_shape(t, 128, 2001, code, teacher_top=top)
    loss, d_x, ws = torch.empty(t, device="cuda"), torch.empty_like(x), B.alloc_head_workspace(shape, True)
    tail = (None, None, loss, None, None, d_x, ws)
    if top:
        B.mixlora_head_distill(shape, x, w, args[0], args[1], None, *tail)
    else:
        B.mixlora_head_loss(shape, x, w, args[0], *tail)
    torch.cuda.synchronize()
    assert torch.equal(loss, full["loss"]) and torch.equal(d_x, full["d_x"]) and B.mixlora_device_status(ws) == 0
    # the loss alone takes the same sums; a gradient's workspace serves it too
    alone = run(B, x, w, *args, grad=False, ws=ws)
    assert all(torch.equal(alone[n], full[n]) for n in ("loss", "lse", "totals"))
