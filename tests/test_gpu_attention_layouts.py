"""Masked attention on rows that lie apart, each tensor with a stride of its own, and on several streams at once.  Cases,
oracle and bounds as in test_gpu_attention.py."""
import pytest

from test_gpu_attention import MARK, TYPES, Case

pytestmark = pytest.mark.gpu

GAPS = dict(q=8, k=24, v=40, o=16)      # values between the rows of each


def apart(x, gap, fill):
    """The rows of x with `gap` values behind each, and the buffer they lie in."""
    import torch
    buf = torch.full((x.shape[0], x[0].numel() + gap), fill, dtype=x.dtype, device="cuda")
    part = buf[:, :x[0].numel()].unflatten(1, x.shape[1:])
    part.copy_(x)
    return part, buf


def run_apart(c, backward, max_q_len=0):
    import torch
    from paper_2404_15159_b200 import binding as B
    t = c.to_gpu()
    nan = float("nan")
    q, k, v = (apart(t[n], GAPS[n], nan)[0] for n in "qkv")
    d_o = apart(t["d_o"], GAPS["o"], nan)[0]
    o, o_buf = apart(torch.full_like(t["q"], MARK), GAPS["o"], MARK)
    lse = torch.full((c.hq, c.rows), MARK, dtype=torch.float32, device="cuda")
    shape = c.shape(B, dict(q=q, k=k, v=v), max_q_len=max_q_len)
    shape.o_stride = o.stride(0)
    mask = B.make_attention_mask(t["q_off"], t["k_off"], t["k_len"], t["prefix"], t["slopes"])
    ws = B.alloc_attention_workspace(shape, backward)
    B.mixlora_attention_forward(shape, mask, q, k, v, o, lse, ws)
    got, bufs = dict(o=o, lse=lse), [(o_buf, GAPS["o"])]
    if backward:
        grads = [apart(torch.full_like(t[n], MARK), GAPS[n], MARK) for n in "qkv"]
        B.mixlora_attention_backward(shape, mask, q, k, v, o, lse, d_o, ws, *(g for g, _ in grads))
        got.update({"d_" + n: g for n, (g, _) in zip("qkv", grads)})
        bufs += [(b, GAPS[n]) for n, (_, b) in zip("qkv", grads)]
    assert B.mixlora_device_status(ws) == 0
    assert all((b[:, -gap:] == MARK).all() for b, gap in bufs), "values between the rows were written"
    return {n: x.double().cpu().numpy() for n, x in got.items()}


@TYPES
@pytest.mark.parametrize("dim", [40, 64, 80, 128])
@pytest.mark.parametrize("mask", [dict(), dict(softcap=5.0, slopes=[0.1, 0.0, 0.5, 0.02], window=60)], ids=str)
def test_a_stride_for_each_tensor(mask, dim, bf16):
    c = Case([100, 1, 190], hq=4, hk=2, dim=dim, seed=101, bf16=bf16, tail=2, **mask)
    c.check(run_apart(c, True))


@TYPES
@pytest.mark.parametrize("q_len,hq,dim", [(1, 4, 128), (3, 8, 80), (4, 16, 64)])
@pytest.mark.parametrize("seqs", [1, 60])
def test_few_rows_with_a_stride_for_each_tensor(seqs, q_len, hq, dim, bf16):
    # joined within a cluster, and, with many sequences, through partials or not at all
    lens = [700 - 11 * i for i in range(seqs)]
    c = Case([q_len] * seqs, k_lens=[701] * seqs, k_len=lens, hq=hq, hk=2, dim=dim, seed=102, bf16=bf16, tail=3)
    c.check(run_apart(c, False, max_q_len=q_len), backward=False)


@TYPES
def test_strided_rows_of_one_product_in_a_decoding_step(bf16):
    # q, k, v of the last tokens side by side in one product's rows (no cache)
    c = Case([2, 1, 2], hq=4, hk=2, dim=64, seed=103, bf16=bf16, tail=2)
    c.check(c.run(backward=False, packed=True, max_q_len=2), backward=False)


@TYPES
def test_training_steps_on_two_streams(bf16):
    import torch
    from paper_2404_15159_b200 import binding as B
    c = Case([300, 77, 200], hq=4, hk=2, dim=128, seed=104, bf16=bf16, softcap=9.0)
    t = c.to_gpu()
    shape = c.shape(B, t)
    mask = B.make_attention_mask(t["q_off"], t["k_off"])

    def buffers():
        return ([torch.zeros_like(t["q"]), torch.zeros(4, c.rows, device="cuda"), *(torch.zeros_like(t[n]) for n in "qkv")],
                B.alloc_attention_workspace(shape, True))

    def step(outs, ws, stream=None):
        B.mixlora_attention_forward(shape, mask, t["q"], t["k"], t["v"], outs[0], outs[1], ws, stream=stream)
        B.mixlora_attention_backward(shape, mask, t["q"], t["k"], t["v"], outs[0], outs[1], t["d_o"], ws, *outs[2:],
                                     stream=stream)

    want, ws = buffers()
    step(want, ws)
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = [buffers() for _ in streams]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (outs, ws) in zip(streams, work):
            step(outs, ws, s)
    torch.cuda.synchronize()
    for outs, ws in work:
        assert B.mixlora_device_status(ws) == 0
        assert all(torch.equal(x, y) for x, y in zip(outs, want))


def test_two_captured_decoding_steps_with_a_workspace_each():
    import torch
    from paper_2404_15159_b200 import binding as B
    c = Case([1] * 40, k_lens=[700] * 40, hq=32, hk=8, dim=128, seed=105)
    t = c.to_gpu()
    shape = c.shape(B, t, max_q_len=1, max_k_len=700)
    mask = B.make_attention_mask(t["q_off"], t["k_off"])
    want = torch.empty_like(t["q"])
    B.mixlora_attention_forward(shape, mask, t["q"], t["k"], t["v"], want, None, B.alloc_attention_workspace(shape, False))
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = []
    torch.cuda.synchronize()
    for s in streams:
        o, ws, graph = torch.zeros_like(want), B.alloc_attention_workspace(shape, False), torch.cuda.CUDAGraph()
        with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
            B.mixlora_attention_forward(shape, mask, t["q"], t["k"], t["v"], o, None, ws)
        work.append((o, ws, graph))
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (_, _, graph) in zip(streams, work):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o, _, _ in work)
