"""Masked attention through the C ABI against the float64 oracle: forward and backward, both types, over lengths, masks,
head layouts and strides where such kernels go wrong.  Tolerances are the oracle's own bounds (derived there) for p and
ds rounded to the operand type and outputs rounded once: half a step is 2^-8 of the value in bf16, 2^-24 in fp32."""
import numpy as np
import pytest

from oracle import attention_oracle as orc
from paper_2404_15159_b200 import synth

pytestmark = pytest.mark.gpu

MARK = 7.0      # what the outputs hold before a call: rows outside every sequence must still hold it


def offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


class Case:
    """Inputs of one problem: rows outside every sequence are NaN, and come back as they were."""

    def __init__(self, q_lens, k_lens=None, k_len=None, hq=2, hk=2, dim=64, seed=0, bf16=True, tail=0, amp=1.0, **mask):
        k_lens = q_lens if k_lens is None else k_lens
        self.q_off, self.k_off, self.k_len = offsets(q_lens), offsets(k_lens), k_len
        self.hq, self.hk, self.dim, self.bf16, self.mask, self.n = hq, hk, dim, bf16, mask, len(q_lens)
        self.rows, self.keys = int(self.q_off[-1]) + tail, int(self.k_off[-1]) + tail
        rng = np.random.default_rng(1000 + seed)
        rnd = synth.round_to_bf16 if bf16 else (lambda x: np.asarray(x, np.float32).astype(np.float64))
        make = lambda *s: rnd(rng.standard_normal(s))  # noqa: E731
        self.q, self.k = rnd(make(self.rows, hq, dim) * amp), make(self.keys, hk, dim)
        self.v, self.d_o = make(self.keys, hk, dim), make(self.rows, hq, dim)
        outside = np.ones(self.keys, bool)
        for b in range(self.n):
            used = k_lens[b] if k_len is None else min(max(k_len[b], 0), k_lens[b])
            outside[self.k_off[b]:self.k_off[b] + used] = False
        self.k[outside], self.v[outside] = np.nan, np.nan
        self.q[self.q_off[-1]:], self.d_o[self.q_off[-1]:] = np.nan, np.nan

    def want(self, backward=True):
        slopes = self.mask.get("slopes")
        step = 2.0 ** -8 if self.bf16 else 0.0
        return orc.attention(self.q, self.k, self.v, self.q_off, self.k_off, k_len=self.k_len,
                             d_o=self.d_o if backward else None, p_step=step,
                             out_step=2.0 ** -8 if self.bf16 else 2.0 ** -24,
                             **{**self.mask, "slopes": None if slopes is None else np.float32(slopes)})

    def to_gpu(self, packed=False):
        import torch
        act = torch.bfloat16 if self.bf16 else torch.float32
        put = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(act)  # noqa: E731
        t = dict(q=put(self.q), k=put(self.k), v=put(self.v), d_o=put(self.d_o))
        if packed:                                   # q, k, v side by side in the rows of one product, with a gap
            assert self.rows == self.keys
            w = (self.hq + 2 * self.hk) * self.dim + 8
            buf = torch.full((self.rows, w), float("nan"), dtype=act, device="cuda")
            a, b = self.hq * self.dim, (self.hq + self.hk) * self.dim
            parts = buf[:, :a], buf[:, a:b], buf[:, b:b + self.hk * self.dim]
            for n, p in zip("qkv", parts):
                p.copy_(t[n].reshape(self.rows, -1))
                t[n] = p
            t["buf"] = buf
        i32 = lambda x: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
        t.update(q_off=i32(self.q_off), k_off=i32(self.k_off), k_len=i32(self.k_len), prefix=i32(self.mask.get("prefix")))
        s = self.mask.get("slopes")
        t["slopes"] = None if s is None else torch.tensor(np.asarray(s), dtype=torch.float32, device="cuda")
        return t

    def shape(self, B, t, max_q_len=0, max_k_len=0):
        m = self.mask
        return B.make_attention_shape(self.n, self.rows, self.keys, self.hq, self.hk, self.dim,
                                      B.MIXLORA_DTYPE_BF16 if self.bf16 else B.MIXLORA_DTYPE_FP32, scale=m.get("scale"),
                                      causal=int(m.get("causal", True)), window=m.get("window", 0),
                                      softcap=m.get("softcap", 0.0), max_q_len=max_q_len, max_k_len=max_k_len,
                                      q_stride=t["q"].stride(0), k_stride=t["k"].stride(0), v_stride=t["v"].stride(0))

    def run(self, backward=True, packed=False, max_q_len=0, max_k_len=0):
        import torch
        from paper_2404_15159_b200 import binding as B
        t = self.to_gpu(packed)
        shape = self.shape(B, t, max_q_len, max_k_len)
        mask = B.make_attention_mask(t["q_off"], t["k_off"], t["k_len"], t["prefix"], t["slopes"])
        ws = B.alloc_attention_workspace(shape, backward)
        act = t["d_o"].dtype
        o = torch.full((self.rows, self.hq, self.dim), MARK, dtype=act, device="cuda")
        lse = torch.full((self.hq, self.rows), MARK, dtype=torch.float32, device="cuda")
        B.mixlora_attention_forward(shape, mask, t["q"], t["k"], t["v"], o, lse, ws)
        assert B.mixlora_device_status(ws) == 0
        got = dict(o=o, lse=lse)
        if backward:
            if packed:
                g = torch.full_like(t["buf"], MARK)
                a, b = self.hq * self.dim, (self.hq + self.hk) * self.dim
                grads = g[:, :a], g[:, a:b], g[:, b:b + self.hk * self.dim]
            else:
                grads = [torch.full_like(t[n], MARK) for n in "qkv"]
            # rows of o and lse outside every sequence hold anything
            o[int(self.q_off[-1]):] = float("nan")
            lse[:, int(self.q_off[-1]):] = float("nan")
            B.mixlora_attention_backward(shape, mask, t["q"], t["k"], t["v"], o, lse, t["d_o"], ws, *grads)
            assert B.mixlora_device_status(ws) == 0
            o[int(self.q_off[-1]):] = MARK
            lse[:, int(self.q_off[-1]):] = MARK
            if packed:
                assert (g[:, -8:] == MARK).all()
            got.update(d_q=grads[0].reshape(self.rows, self.hq, self.dim), d_k=grads[1].reshape(self.keys, self.hk, self.dim),
                       d_v=grads[2].reshape(self.keys, self.hk, self.dim))
        torch.cuda.synchronize()
        return {n: x.double().cpu().numpy() for n, x in got.items()}

    def check(self, got, backward=True):
        want = self.want(backward)
        for n, x in got.items():
            ref, bound = want[n], want["bound"][n]
            left = np.isnan(ref)
            assert (x[left] == MARK).all(), f"{n}: rows outside every sequence were written"
            x, ref, bound = x[~left], ref[~left], bound[~left]
            empty = np.isneginf(ref)
            assert np.isneginf(x[empty]).all(), f"{n}: rows that see nothing"
            off = np.abs(x[~empty] - ref[~empty])
            assert np.isfinite(off).all(), f"{n}: not finite"
            assert (off <= bound[~empty]).all(), \
                f"{n}: off by {off.max():.3e}, {(off / np.maximum(bound[~empty], 1e-300)).max():.2f} times its bound"


TYPES = pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "fp32"])


@TYPES
@pytest.mark.parametrize("lens", [[1], [2, 1, 1], [64], [127], [128], [129], [255, 256, 257], [0, 3, 0, 0, 130, 0], [700]])
def test_causal_lengths(lens, bf16):
    c = Case(lens, hq=4, hk=2, dim=128, seed=len(lens), bf16=bf16, tail=5)
    c.check(c.run())


@TYPES
@pytest.mark.parametrize("dim", [8, 16, 40, 64, 72, 80, 96, 120, 128])
def test_head_sizes(dim, bf16):
    c = Case([150, 70], hq=2, hk=1, dim=dim, seed=dim, bf16=bf16)
    c.check(c.run())


@TYPES
@pytest.mark.parametrize("mask", [
    dict(causal=False), dict(window=1), dict(window=50), dict(window=128), dict(causal=False, window=37),
    dict(prefix=[40, 300, 0]), dict(prefix=[130, 1000, 1], window=20), dict(causal=False, window=9, prefix=[200, 7, 3]),
    dict(softcap=5.0), dict(slopes=[0.5, 0.25, 0.0625, 0.0]), dict(softcap=20.0, slopes=[0.1, 0.0, 2.0, 0.01], window=200),
    dict(softcap=5.0, causal=False), dict(scale=0.02), dict(window=2 ** 31 - 1), dict(causal=False, window=2 ** 31 - 1)],
    ids=str)
def test_masks(mask, bf16):
    c = Case([290, 131, 33], hq=4, hk=2, dim=64, seed=3, bf16=bf16, tail=3, **mask)
    c.check(c.run())


@TYPES
@pytest.mark.parametrize("mask", [dict(), dict(causal=False), dict(window=210), dict(prefix=[500, 100]),
                                  dict(prefix=[140, 0], window=70, softcap=8.0), dict(causal=False, window=150)], ids=str)
def test_distance_over_many_tiles(mask, bf16):
    # the scores rise or fall by up to hundreds from tile to tile, in either direction, under every kind of mask
    c = Case([601, 300], k_lens=[601, 450], hq=4, hk=4, dim=96, seed=21, bf16=bf16, tail=4,
             slopes=[1.0, 0.03, -0.5, 0.0], **mask)
    c.check(c.run())


@TYPES
@pytest.mark.parametrize("hq,hk", [(1, 1), (8, 1), (6, 2), (5, 5)])
def test_shared_heads(hq, hk, bf16):
    c = Case([200, 141], hq=hq, hk=hk, dim=64, seed=hq, bf16=bf16)
    c.check(c.run())


@TYPES
@pytest.mark.parametrize("mask", [dict(), dict(causal=False), dict(window=30), dict(prefix=[3, 0, 500, 2, 1])], ids=str)
def test_more_rows_than_keys_and_more_keys_than_rows(mask, bf16):
    # the first rows of a sequence with fewer keys than rows see nothing; slots of which a part, or nothing, is used
    c = Case([140, 3, 20, 130, 7], k_lens=[300, 5, 260, 40, 0], k_len=[131, 1, 257, 40, 0], hq=2, hk=1, dim=64, seed=9,
             bf16=bf16, tail=9, **mask)
    c.check(c.run())


@TYPES
def test_strided_rows_of_one_product(bf16):
    c = Case([100, 190], hq=4, hk=2, dim=80, seed=11, bf16=bf16, tail=2)
    c.check(c.run(packed=True))


@TYPES
def test_large_scores_become_one_hot(bf16):
    # scores far apart: one key takes a row, the running maximum moves often
    c = Case([300], hq=2, hk=2, dim=64, seed=12, bf16=bf16, amp=40.0)
    c.check(c.run())


@TYPES
@pytest.mark.parametrize("hq,hk,q_len,dim", [(4, 4, 1, 128), (8, 2, 1, 64), (8, 2, 4, 128), (4, 2, 3, 80), (16, 1, 1, 96),
                                             (16, 1, 3, 64), (32, 1, 2, 128), (6, 6, 2, 8)])
@pytest.mark.parametrize("mask", [dict(), dict(window=100), dict(softcap=8.0, window=700, prefix=True), dict(slopes=True),
                                  dict(softcap=3.0, slopes=True, causal=False)], ids=str)
def test_few_rows_against_a_cache(hq, hk, q_len, dim, mask, bf16):
    slot = 1100
    k_len = [1100, 1, 0, 17, 513, 2, 1000]
    mask = dict(mask)
    if mask.get("prefix"):
        mask["prefix"] = [5, 0, 9, 30, 100, 1, 257]
    if mask.get("slopes"):
        mask["slopes"] = list(2.0 ** -(1.0 + np.arange(hq) % 8))
    c = Case([q_len] * 7, k_lens=[slot] * 7, k_len=k_len, hq=hq, hk=hk, dim=dim, seed=hq + q_len, bf16=bf16, tail=3, **mask)
    got = c.run(backward=False, max_q_len=q_len, max_k_len=slot)
    c.check(got, backward=False)
    tiled = c.run(backward=False)                     # the same rows without the promise
    c.check(tiled, backward=False)


@TYPES
@pytest.mark.parametrize("max_k_len", [0, 40, 5000])
def test_few_rows_split_over_a_long_cache(max_k_len, bf16):
    # one sequence, so that its keys are split over many blocks; sequences shorter than max_q_len, and empty ones
    c = Case([2, 0, 1], k_lens=[5000, 30, 300], k_len=[4999, 30, 300], hq=2, hk=1, dim=128, seed=21, bf16=bf16)
    c.check(c.run(backward=False, max_q_len=2, max_k_len=max_k_len), backward=False)


def test_rows_behind_max_q_len_are_left():
    c = Case([3], k_lens=[50], hq=1, hk=1, dim=64, seed=22)
    got = c.run(backward=False, max_q_len=2)
    assert (got["o"][2] == MARK).all() and (got["lse"][:, 2] == MARK).all() and (got["o"][:2] != MARK).any()


def test_no_sequences_and_no_rows():
    import torch
    from paper_2404_15159_b200 import binding as B
    x = torch.full((8, 1, 64), MARK, dtype=torch.bfloat16, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    lse = torch.full((1, 8), MARK, device="cuda")
    for n, rows in ((0, 8), (2, 0), (2, 8)):
        for few in (0, 1):
            s = B.make_attention_shape(n, rows, rows, 1, 1, 64, max_q_len=few)
            ws = B.alloc_attention_workspace(s, True)
            outs = [x.clone() for _ in range(4)]
            m = B.make_attention_mask(off, off)
            B.mixlora_attention_forward(s, m, x, x, x, outs[0], lse, ws)
            B.mixlora_attention_backward(s, m, x, x, x, x, lse, x, ws, *outs[1:])
            torch.cuda.synchronize()
            assert B.mixlora_device_status(ws) == 0
            assert all((o == MARK).all() for o in outs) and (lse == MARK).all()


def test_offsets_that_do_not_ascend_or_lie_outside_stay_inside_the_tensors():
    # no result is promised; nothing outside the outputs is touched and the call ends
    import torch
    from paper_2404_15159_b200 import binding as B
    for few in (0, 1):
        for bf16 in (True, False):
            act = torch.bfloat16 if bf16 else torch.float32
            pad = torch.full((3, 40, 2, 64), MARK, dtype=act, device="cuda")
            o, q = pad[1], torch.zeros(40, 2, 64, dtype=act, device="cuda")
            off = torch.tensor([-5, 30, 20, 2 ** 31 - 1, 7], dtype=torch.int32, device="cuda")
            k_len = torch.tensor([-1, 2 ** 31 - 1, 5, 9], dtype=torch.int32, device="cuda")
            s = B.make_attention_shape(4, 40, 40, 2, 2, 64, B.MIXLORA_DTYPE_BF16 if bf16 else B.MIXLORA_DTYPE_FP32,
                                       max_q_len=few)
            ws = B.alloc_attention_workspace(s, True)
            m = B.make_attention_mask(off, off, k_len=k_len, prefix=k_len)
            lse = torch.zeros(2, 40, device="cuda")
            B.mixlora_attention_forward(s, m, q, q, q, o, lse, ws)
            B.mixlora_attention_backward(s, m, q, q, q, q, lse, q, ws, torch.zeros_like(q), torch.zeros_like(q),
                                         torch.zeros_like(q))
            torch.cuda.synchronize()
            assert (pad[0] == MARK).all() and (pad[2] == MARK).all()


def test_same_result_every_time_and_in_a_captured_graph():
    import torch
    from paper_2404_15159_b200 import binding as B
    c = Case([300, 77, 200], hq=4, hk=2, dim=128, seed=31)
    t = c.to_gpu()
    shape = c.shape(B, t)
    mask = B.make_attention_mask(t["q_off"], t["k_off"])
    ws = B.alloc_attention_workspace(shape, True)
    outs = [torch.empty_like(t["q"]), torch.empty(4, c.rows, device="cuda"), *(torch.empty_like(t[n]) for n in "qkv")]

    def step():
        B.mixlora_attention_forward(shape, mask, t["q"], t["k"], t["v"], outs[0], outs[1], ws)
        B.mixlora_attention_backward(shape, mask, t["q"], t["k"], t["v"], outs[0], outs[1], t["d_o"], ws, *outs[2:])

    step()
    first = [x.clone() for x in outs]
    step()
    assert all(torch.equal(x, y) for x, y in zip(first, outs))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    t["q"].copy_(t["q"].flip(0))                      # new inputs in the same buffers
    graph.replay()
    torch.cuda.synchronize()
    replayed = [x.clone() for x in outs]
    assert not torch.equal(first[0], replayed[0])
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(replayed, outs))


def test_two_streams_with_a_workspace_each():
    import torch
    from paper_2404_15159_b200 import binding as B
    c = Case([1, 1, 1], k_lens=[900] * 3, k_len=[900, 3, 450], hq=8, hk=2, dim=128, seed=33)
    t = c.to_gpu()
    shape = c.shape(B, t, max_q_len=1)
    mask = B.make_attention_mask(t["q_off"], t["k_off"], t["k_len"])
    want = torch.empty_like(t["q"])
    B.mixlora_attention_forward(shape, mask, t["q"], t["k"], t["v"], want, None, B.alloc_attention_workspace(shape, False))
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = [(torch.empty_like(want), B.alloc_attention_workspace(shape, False)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (o, ws) in zip(streams, work):
            B.mixlora_attention_forward(shape, mask, t["q"], t["k"], t["v"], o, None, ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o, _ in work)


@TYPES
def test_many_short_sequences(bf16):
    # more sequences than the planning block has threads, empty ones among them
    lens = [(i * 7) % 4 for i in range(2600)]
    c = Case(lens, hq=2, hk=1, dim=16, seed=41, bf16=bf16, tail=1)
    c.check(c.run())


def test_decoding_step_in_a_captured_graph():
    import torch
    from paper_2404_15159_b200 import binding as B
    for slots, slot in ((1, 2000), (40, 700)):        # joined inside a cluster; through partials and a second launch
        c = Case([1] * slots, k_lens=[slot] * slots, k_len=[slot - 3 * (i % 50) for i in range(slots)], hq=32, hk=8, dim=128,
                 seed=50 + slots)
        t = c.to_gpu()
        shape = c.shape(B, t, max_q_len=1, max_k_len=slot)
        mask = B.make_attention_mask(t["q_off"], t["k_off"], t["k_len"])
        ws, o, lse = B.alloc_attention_workspace(shape, False), torch.empty_like(t["q"]), torch.empty(32, c.rows, device="cuda")
        step = lambda: B.mixlora_attention_forward(shape, mask, t["q"], t["k"], t["v"], o, lse, ws)  # noqa: E731
        step()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        torch.cuda.synchronize()
        # the next step: every sequence one key shorter, another query
        t["k_len"] -= 1
        t["q"].copy_(t["q"].flip(1))
        c.k_len = [n - 1 for n in c.k_len]
        c.q = c.q[:, ::-1]
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        c.check(dict(o=o.double().cpu().numpy(), lse=lse.double().cpu().numpy()), backward=False)


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "fp32"])
def test_offsets_beyond_32_bits(few, bf16):
    # the one sequence lies behind 2^31 elements of a cache (and, in bf16, behind 2^32 bytes of it)
    import torch
    from paper_2404_15159_b200 import binding as B
    hk, dim, lk, lq = 8, 128, 300, (2 if few else 70)
    far = 2 ** 31 // (hk * dim) + 5
    act = torch.bfloat16 if bf16 else torch.float32
    c = Case([lq], k_lens=[lk], hq=8, hk=hk, dim=dim, seed=61, bf16=bf16)
    t = c.to_gpu()
    big = [torch.empty(far + lk, hk, dim, dtype=act, device="cuda") for _ in range(2)]
    for x, n in zip(big, "kv"):
        x[far:] = t[n]
    off = torch.tensor([far, far + lk], dtype=torch.int32, device="cuda")
    shape = B.make_attention_shape(1, lq, far + lk, 8, hk, dim, B.MIXLORA_DTYPE_BF16 if bf16 else B.MIXLORA_DTYPE_FP32,
                                   max_q_len=lq if few else 0, max_k_len=lk)
    ws = B.alloc_attention_workspace(shape, not few)
    mask = B.make_attention_mask(t["q_off"], off)
    o, lse = torch.empty_like(t["q"]), torch.empty(8, lq, device="cuda")
    B.mixlora_attention_forward(shape, mask, t["q"], big[0], big[1], o, lse, ws)
    got = dict(o=o, lse=lse)
    if not few:
        grads = [torch.empty_like(t["q"]), torch.empty_like(big[0]), torch.empty_like(big[1])]
        B.mixlora_attention_backward(shape, mask, t["q"], big[0], big[1], o, lse, t["d_o"], ws, *grads)
        got.update(d_q=grads[0], d_k=grads[1][far:], d_v=grads[2][far:])
    torch.cuda.synchronize()
    c.check({n: x.double().cpu().numpy() for n, x in got.items()}, backward=not few)


@pytest.mark.parametrize("size", [1e3, 1e6, 1e15])
def test_scores_of_any_size_end(size):
    # up to scores whose neighbours in fp32 lie further apart than its exponents reach: the call still ends
    import torch
    from paper_2404_15159_b200 import binding as B
    n = 200
    x = torch.zeros(n, 1, 64, dtype=torch.bfloat16, device="cuda")
    x[:, 0, 0] = size
    v = torch.ones_like(x)
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    shape = B.make_attention_shape(1, n, n, 1, 1, 64)
    ws = B.alloc_attention_workspace(shape, True)
    o, lse = torch.empty_like(x), torch.empty(1, n, device="cuda")
    mask = B.make_attention_mask(off, off)
    B.mixlora_attention_forward(shape, mask, x, x, v, o, lse, ws)
    B.mixlora_attention_backward(shape, mask, x, x, v, o, lse, v, ws, *(torch.empty_like(x) for _ in range(3)))
    assert B.mixlora_device_status(ws) == 0
    if size <= 1e3:                                   # equal scores: every row is the mean of ones
        assert (o == 1).all()
