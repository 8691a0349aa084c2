"""The attention half of a MixLoRA layer as a program runs it: q, k, v projections with LoRA, rotary positions, masked
attention over a packed batch, output projection with LoRA, forward and back to the LoRA gradients and the input; and a
decoding step that appends to a cache.  Against the same run in float64, within the norms this library's layers are
held to: 1e-4 in fp32, 2e-2 in bf16 (largest error over largest value)."""
import numpy as np
import pytest

import helpers
from oracle import attention_oracle as att
from oracle import mixlora_oracle as orc
from paper_2404_15159_b200 import synth

pytestmark = pytest.mark.gpu

D_MODEL, HQ, HK, DIM, R, ALPHA = 256, 4, 2, 64, 8, 16.0
LENS = [90, 1, 133, 40]
OUT = dict(q=HQ * DIM, k=HK * DIM, v=HK * DIM, o=D_MODEL)
IN = dict(q=D_MODEL, k=D_MODEL, v=D_MODEL, o=HQ * DIM)


def inputs(bf16):
    rng = np.random.default_rng(77)
    rnd = synth.round_to_bf16 if bf16 else (lambda x: np.asarray(x, np.float32).astype(np.float64))
    T = sum(LENS)
    t = dict(x=rnd(rng.standard_normal((T, D_MODEL))), dy=rnd(rng.standard_normal((T, D_MODEL))))
    for n in "qkvo":
        t["w" + n] = rnd(rng.standard_normal((OUT[n], IN[n])) * IN[n] ** -0.5)
        t["a" + n] = rnd(rng.standard_normal((R, IN[n])) / R)
        t["b" + n] = rnd(rng.standard_normal((OUT[n], R)) * 0.05)
    return T, t


def reference(T, t, off, pos, w):
    lin = lambda n, x: orc.lora_linear_forward(x, t["w" + n], t["a" + n], t["b" + n], ALPHA)  # noqa: E731
    back = lambda n, x, dy: orc.lora_linear_backward(x, t["w" + n], t["a" + n], t["b" + n], ALPHA, dy)  # noqa: E731
    q, k, v = (lin(n, t["x"]).reshape(T, -1, DIM) for n in "qkv")
    qr, kr = att.rope(q, pos, w)[0], att.rope(k, pos, w)[0]
    o = att.attention(qr, kr, v, off, off)["o"]
    y = lin("o", o.reshape(T, -1))
    go = back("o", o.reshape(T, -1), t["dy"])
    g = att.attention(qr, kr, v, off, off, d_o=go["d_x"].reshape(T, HQ, DIM))
    dq, dk = att.rope(g["d_q"], pos, w, backward=True)[0], att.rope(g["d_k"], pos, w, backward=True)[0]
    out = dict(y=y, d_ao=go["d_a"], d_bo=go["d_b"], d_x=0.0)
    for n, d in (("q", dq), ("k", dk), ("v", g["d_v"])):
        gn = back(n, t["x"], d.reshape(T, -1))
        out["d_a" + n], out["d_b" + n] = gn["d_a"], gn["d_b"]
        out["d_x"] = out["d_x"] + gn["d_x"]
    return out


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "fp32"])
def test_training_step_of_the_attention_half(bf16):
    import torch
    from paper_2404_15159_b200 import binding as B
    T, t = inputs(bf16)
    off = np.concatenate([[0], np.cumsum(LENS)])
    pos = np.concatenate([np.arange(n) for n in LENS]).astype(np.int32)
    act = torch.bfloat16 if bf16 else torch.float32
    dtype = B.MIXLORA_DTYPE_BF16 if bf16 else B.MIXLORA_DTYPE_FP32
    g = {n: torch.from_numpy(np.ascontiguousarray(v)).cuda().to(act) for n, v in t.items()}
    lin = {n: B.make_linear_shape(T, IN[n], OUT[n], R, ALPHA, dtype) for n in "qkvo"}
    lws = {n: B.alloc_linear_workspace(s) for n, s in lin.items()}
    new = lambda width: torch.empty(T, width, dtype=act, device="cuda")  # noqa: E731
    proj = {n: new(OUT[n]) for n in "qkvo"}
    table = torch.empty(DIM // 2, dtype=torch.float64, device="cuda")
    B.mixlora_rope_frequencies(DIM, 10000.0, B.MIXLORA_ROPE_SCALE_NONE, 1.0, 0.0, 0.0, 0, table)
    rope = B.make_rope_shape(T, HQ, HK, DIM, DIM, dtype=dtype)
    shape = B.make_attention_shape(len(LENS), T, T, HQ, HK, DIM, dtype)
    d_off, d_pos = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (off, pos))
    mask = B.make_attention_mask(d_off, d_off)
    ws = B.alloc_attention_workspace(shape, True)
    o, lse = new(HQ * DIM), torch.empty(HQ, T, device="cuda")
    grads = {n: (torch.empty(R, IN[n], device="cuda"), torch.empty(OUT[n], R, device="cuda")) for n in "qkvo"}

    for n in "qkv":
        B.mixlora_lora_linear_forward(lin[n], g["x"], g["w" + n], g["a" + n], g["b" + n], proj[n], lws[n])
    B.mixlora_rope_forward(rope, proj["q"], proj["k"], d_pos, table, proj["q"], proj["k"])      # in place
    B.mixlora_attention_forward(shape, mask, proj["q"], proj["k"], proj["v"], o, lse, ws)
    B.mixlora_lora_linear_forward(lin["o"], o, g["wo"], g["ao"], g["bo"], proj["o"], lws["o"])
    d_o, d = new(HQ * DIM), {n: new(OUT[n]) for n in "qkv"}
    B.mixlora_lora_linear_backward(lin["o"], o, g["wo"], g["ao"], g["bo"], g["dy"], lws["o"], *grads["o"], d_o)
    B.mixlora_attention_backward(shape, mask, proj["q"], proj["k"], proj["v"], o, lse, d_o, ws, d["q"], d["k"], d["v"])
    B.mixlora_rope_backward(rope, d["q"], d["k"], d_pos, table, d["q"], d["k"])
    d_x = torch.zeros(T, D_MODEL, device="cuda")
    for n in "qkv":
        part = new(D_MODEL)
        B.mixlora_lora_linear_backward(lin[n], g["x"], g["w" + n], g["a" + n], g["b" + n], d[n], lws[n], *grads[n], part)
        d_x += part.float()
    torch.cuda.synchronize()
    assert B.mixlora_device_status(ws) == 0

    want = reference(T, t, off, pos, att.rope_frequencies(DIM, 10000.0))
    got = dict(y=proj["o"], d_x=d_x, **{"d_a" + n: grads[n][0] for n in "qkvo"}, **{"d_b" + n: grads[n][1] for n in "qkvo"})
    for n, x in got.items():
        e = helpers.rel_err(x.double().cpu().numpy(), want[n])
        assert e <= (2e-2 if bf16 else 1e-4), f"{n}: {e:.2e}"


def test_decoding_appends_to_a_cache_and_equals_the_whole_sequence():
    # token by token against slots of a cache, both forms of the forward call give the packed result within roundings
    import torch
    from paper_2404_15159_b200 import binding as B
    rng = np.random.default_rng(5)
    lens, slot = [37, 12, 20], 40
    T = sum(lens)
    off = np.concatenate([[0], np.cumsum(lens)])
    q, k, v = (torch.from_numpy(synth.round_to_bf16(rng.standard_normal((T, h, DIM)))).cuda().to(torch.bfloat16)
               for h in (HQ, HK, HK))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    d_off = i32(off)
    shape = B.make_attention_shape(3, T, T, HQ, HK, DIM)
    whole = torch.empty_like(q)
    B.mixlora_attention_forward(shape, B.make_attention_mask(d_off, d_off), q, k, v, whole, None,
                                B.alloc_attention_workspace(shape, False))
    cache_k = torch.full((3 * slot, HK, DIM), float("nan"), dtype=torch.bfloat16, device="cuda")
    cache_v = cache_k.clone()
    step = B.make_attention_shape(3, 3, 3 * slot, HQ, HK, DIM, max_q_len=1, max_k_len=slot)
    ws = B.alloc_attention_workspace(step, False)
    q_off, k_off = i32([0, 1, 2, 3]), i32([0, slot, 2 * slot, 3 * slot])
    for i in range(max(lens)):
        rows = [int(off[b]) + min(i, lens[b] - 1) for b in range(3)]
        used = [min(i, lens[b] - 1) + 1 for b in range(3)]
        for b in range(3):
            cache_k[b * slot + used[b] - 1] = k[rows[b]]
            cache_v[b * slot + used[b] - 1] = v[rows[b]]
        o = torch.empty(3, HQ, DIM, dtype=torch.bfloat16, device="cuda")
        k_len = i32(used)
        B.mixlora_attention_forward(step, B.make_attention_mask(q_off, k_off, k_len=k_len), q[rows].contiguous(), cache_k,
                                    cache_v, o, None, ws)
        # both round p (2^-8 of sum p |v| <= max |v|) and the output once
        limit = 2 * 2.0 ** -8 * 2 * float(v.abs().max())
        assert (o.float() - whole[rows].float()).abs().max().item() <= limit
