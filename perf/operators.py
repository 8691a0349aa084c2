"""Cases of the operators around the attention of a MixLoRA layer, for timing and comparison.

Two operators: rotary positions (`mixlora_rope_*`) and masked attention (`mixlora_attention_*`).  `run` computes
them from elementary torch operations, or, where `own` is true, with the library's calls.  `exact` computes the same
outputs in 64 bits, sequence by sequence and head by head.

A case's kind:
  rope         q and k rotated by their positions (forward, or the gradient's way back)
  attention    forward over packed sequences: output and log-sum-exp of every row
  train        forward and backward over packed sequences: output, dq, dk, dv
  decode       the last `q_len` tokens of every sequence against a cache of fixed slots, of which a part is used
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

ROPE = dict(kind="rope", dtype="bf16", tokens=1, q_heads=32, kv_heads=32, head_dim=128, rotary_dim=128, layout="half",
            backward=False, far=4096, scaling="none", factor=1.0, packed=False)
ATTN = dict(kind="attention", dtype="bf16", tokens=1, seqs=1, q_heads=32, kv_heads=32, head_dim=128, causal=True,
            window=0, softcap=0.0, slopes=False, prefix=False)
DECODE = dict(kind="decode", dtype="bf16", seqs=1, q_len=1, slot=1024, q_heads=32, kv_heads=32, head_dim=128,
              causal=True, window=0, softcap=0.0, slopes=False, prefix=False)


def listed():
    return [
        # one decoding step of eight sequences, positions far beyond the trained range, frequencies scaled by parts
        dict(ROPE, name="rope-decode-8", tokens=8, kv_heads=8, far=100000, scaling="parts", factor=8.0),
        # the training batch of the 7B block: q and k of 8192 tokens
        dict(ROPE, name="rope-train-8192", tokens=8192),
        # gradients in the fp32 check mode, 40 heads, half of each head rotated in neighbouring pairs, an odd count
        dict(ROPE, name="rope-bwd-fp32-1021", dtype="fp32", tokens=1021, q_heads=40, kv_heads=40, rotary_dim=64,
             layout="interleaved", backward=True),
        # gradients of a long batch whose q, k and v lie side by side in one product's rows
        dict(ROPE, name="rope-bwd-packed-32768", tokens=32768, kv_heads=8, backward=True, far=32768, scaling="ntk",
             factor=4.0, packed=True),
        # one token of one sequence against a cache of about a thousand
        dict(DECODE, name="decode-1x1024", slot=1024),
        # a serving batch: 64 sequences of very different lengths, four query heads to a key head
        dict(DECODE, name="decode-64x8192", seqs=64, slot=8192, kv_heads=8),
        # four tokens a sequence in the fp32 check mode, capped scores
        dict(DECODE, name="decode-fp32-7x2000", dtype="fp32", seqs=7, q_len=4, slot=2000, q_heads=16, kv_heads=8,
             head_dim=64, softcap=30.0),
        # the prompt of one long sequence
        dict(ATTN, name="prefill-8192", tokens=8192),
        # a packed batch of 24 documents, capped scores, a prefix that every token of its document sees
        dict(ATTN, name="documents-5003", tokens=5003, seqs=24, kv_heads=8, head_dim=64, softcap=50.0, prefix=True),
        # a training step's attention on the 7B block's 8192 tokens, packed from four documents
        dict(ATTN, name="train-8192", kind="train", tokens=8192, seqs=4, kv_heads=8),
        # odd length and head size, a sliding window, scores lowered with distance, capped
        dict(ATTN, name="train-2901-window", kind="train", tokens=2901, seqs=3, q_heads=20, kv_heads=20, head_dim=80,
             window=500, softcap=30.0, slopes=True),
        # the fp32 check mode, a bidirectional batch of short sequences
        dict(ATTN, name="train-fp32-700", kind="train", dtype="fp32", tokens=700, seqs=5, q_heads=8, kv_heads=4,
             head_dim=64, causal=False),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    heads, groups = rng.choice([(32, 32), (32, 8), (16, 16), (40, 40), (16, 2), (20, 4), (8, 1)])
    dim = rng.choice([128, 128, 64, 80, 96])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    kind = rng.choice(["rope", "decode", "attention", "train"])
    if kind == "rope":
        return dict(ROPE, dtype=dtype, tokens=_spread(rng, 1, 8192 if dtype == "fp32" else 16384), q_heads=heads,
                    kv_heads=groups, head_dim=dim, rotary_dim=rng.choice([dim, dim // 2]),
                    layout=rng.choice(["half", "interleaved"]), backward=rng.random() < 0.5,
                    far=_spread(rng, 100, 1000000), scaling=rng.choice(["none", "linear", "ntk", "parts"]),
                    factor=rng.choice([2.0, 4.0, 8.0]), packed=rng.random() < 0.5)
    mask = dict(window=rng.choice([0, 0, _spread(rng, 8, 2048)]), softcap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                slopes=rng.random() < 0.3, prefix=rng.random() < 0.3)
    if kind == "decode":
        seqs = _spread(rng, 1, 64)
        slot = _spread(rng, 16, min(32768, 1000000000 // (seqs * groups * dim * (4 if dtype == "fp32" else 2))))
        return dict(DECODE, dtype=dtype, seqs=seqs, q_len=rng.choice([1, 1, 1, 2, 4]), slot=slot, q_heads=heads,
                    kv_heads=groups, head_dim=dim, causal=True, **mask)
    tokens = _spread(rng, 64, 1500 if dtype == "fp32" else 6000)
    return dict(ATTN, kind=kind, dtype=dtype, tokens=tokens, seqs=rng.randint(1, max(1, tokens // 64)),
                q_heads=heads, kv_heads=groups, head_dim=dim, causal=rng.random() < 0.8, **mask)


# ---- inputs -----------------------------------------------------------------------------------------------------

def _cuts(total, parts, rng):
    """Offsets of `parts` runs that fill `total` rows, of uneven lengths."""
    w = torch.rand(parts, generator=rng, dtype=torch.float64) + 0.15
    edges = torch.round(torch.cumsum(w, 0) / w.sum() * total).to(torch.int32)
    edges[-1] = total
    return torch.cat([torch.zeros(1, dtype=torch.int32), edges])


def _inv_freq(case):
    """Radians per position of each rotated pair."""
    r, theta, f = case["rotary_dim"], 10000.0, case["factor"]
    if case["scaling"] == "ntk":
        theta *= f ** (r / max(r - 2, 1))
    w = theta ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    if case["scaling"] == "linear":
        w = w / f
    if case["scaling"] == "parts":   # slow waves are stretched, fast ones kept, those between blended
        turns = 8192.0 * w / (2 * math.pi)
        keep = torch.clamp((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        w = w * keep + w / f * (1 - keep)
    return w


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.Generator().manual_seed(seed)
    dt, hq, hk, d = DTYPES[case["dtype"]], case["q_heads"], case["kv_heads"], case["head_dim"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    s = dict(case=case)
    if case["kind"] == "rope":
        t = case["tokens"]
        if case["packed"]:
            rows = normal(t, (hq + 2 * hk) * d)
            s["q"] = rows[:, :hq * d].unflatten(1, (hq, d))
            s["k"] = rows[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
        else:
            s["q"], s["k"] = normal(t, hq, d), normal(t, hk, d)
        start = torch.randint(0, case["far"], (1,), generator=h).item()
        s["positions"] = ((start + torch.arange(t, device="cuda")) % case["far"]).to(torch.int32)
        s["inv_freq"] = _inv_freq(case)
    elif case["kind"] == "decode":
        n, lq, cap = case["seqs"], case["q_len"], case["slot"]
        used = torch.randint(max(lq, cap // 8), cap + 1, (n,), generator=h)
        if n == 1:
            used[0] = cap - torch.randint(0, max(1, cap // 16), (1,), generator=h)
        s["q"] = normal(n * lq, hq, d)
        s["k"], s["v"] = normal(n * cap, hk, d), normal(n * cap, hk, d)
        s["q_off"] = (torch.arange(n + 1) * lq).to(torch.int32).cuda()
        s["k_off"] = (torch.arange(n + 1) * cap).to(torch.int32).cuda()
        s["k_len"] = used.to(torch.int32).cuda()
        longest = cap
    else:
        t, n = case["tokens"], case["seqs"]
        s["q"], s["k"], s["v"] = normal(t, hq, d), normal(t, hk, d), normal(t, hk, d)
        if case["kind"] == "train":
            s["do"] = normal(t, hq, d)
        cuts = _cuts(t, n, h)
        s["q_off"] = s["k_off"] = cuts.cuda()
        s["k_len"] = None
        longest = int((cuts[1:] - cuts[:-1]).max())
    if case["kind"] != "rope":
        n = case["seqs"]
        s["prefix"] = None
        if case["prefix"]:
            s["prefix"] = (torch.rand(n, generator=h) * 0.3 * longest).to(torch.int32).cuda()
        s["slopes"] = None
        if case["slopes"]:
            s["slopes"] = 2.0 ** (-8.0 * (torch.arange(hq, device="cuda", dtype=torch.float32) + 1) / hq)
        s["scale"] = d ** -0.5
    if own:
        s["plan"] = _plan(s)
    return s


def _plan(s):
    """What a program keeps for this shape: the shape, output buffers, workspace, the frequencies' table."""
    from paper_2404_15159_b200 import binding as B
    c = s["case"]
    dtype = B.MIXLORA_DTYPE_BF16 if c["dtype"] == "bf16" else B.MIXLORA_DTYPE_FP32
    hq, hk, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    q, k = s["q"], s["k"]
    if c["kind"] == "rope":
        layout = B.MIXLORA_ROPE_HALF if c["layout"] == "half" else B.MIXLORA_ROPE_INTERLEAVED
        scaling = dict(none=B.MIXLORA_ROPE_SCALE_NONE, linear=B.MIXLORA_ROPE_SCALE_LINEAR, ntk=B.MIXLORA_ROPE_SCALE_NTK,
                       parts=B.MIXLORA_ROPE_SCALE_PARTS)[c["scaling"]]
        table = torch.empty(c["rotary_dim"] // 2, dtype=torch.float64, device="cuda")
        B.mixlora_rope_frequencies(c["rotary_dim"], 10000.0, scaling, c["factor"], 1.0, 4.0, 8192, table)
        shape = B.make_rope_shape(c["tokens"], hq, hk, d, c["rotary_dim"], layout, dtype, q_stride=q.stride(0),
                                  k_stride=k.stride(0), q_out_stride=hq * d, k_out_stride=hk * d)
        return dict(B=B, shape=shape, table=table, q=torch.empty(c["tokens"], hq, d, dtype=q.dtype, device="cuda"),
                    k=torch.empty(c["tokens"], hk, d, dtype=q.dtype, device="cuda"))
    decode = c["kind"] == "decode"
    shape = B.make_attention_shape(c["seqs"], q.shape[0], k.shape[0], hq, hk, d, dtype, scale=s["scale"],
                                   causal=int(c["causal"]), window=c["window"], softcap=c["softcap"],
                                   max_q_len=c["q_len"] if decode else 0, max_k_len=c["slot"] if decode else 0)
    mask = B.make_attention_mask(s["q_off"], s["k_off"], k_len=s["k_len"], prefix=s["prefix"], slopes=s["slopes"])
    plan = dict(B=B, shape=shape, mask=mask, workspace=B.alloc_attention_workspace(shape, c["kind"] == "train"),
                o=torch.empty_like(q), lse=torch.empty(hq, q.shape[0], dtype=torch.float32, device="cuda"))
    if c["kind"] == "train":
        plan.update(dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(k))
    return plan


# ---- the library's calls ----------------------------------------------------------------------------------------

def _own(s):
    p, kind = s["plan"], s["case"]["kind"]
    B = p["B"]
    if kind == "rope":
        call = B.mixlora_rope_backward if s["case"]["backward"] else B.mixlora_rope_forward
        call(p["shape"], s["q"], s["k"], s["positions"], p["table"], p["q"], p["k"])
        return dict(q=p["q"], k=p["k"])
    B.mixlora_attention_forward(p["shape"], p["mask"], s["q"], s["k"], s["v"], p["o"], p["lse"], p["workspace"])
    if kind != "train":
        return dict(o=p["o"], lse=p["lse"])
    B.mixlora_attention_backward(p["shape"], p["mask"], s["q"], s["k"], s["v"], p["o"], p["lse"], s["do"],
                                 p["workspace"], p["dq"], p["dk"], p["dv"])
    return dict(o=p["o"], dq=p["dq"], dk=p["dk"], dv=p["dv"])


# ---- the plain forms --------------------------------------------------------------------------------------------

def _rotate(x, cos, sin, case):
    r = case["rotary_dim"]
    x32 = x.float()
    a, rest = x32[..., :r], x32[..., r:]
    if case["layout"] == "half":
        u, w = a[..., :r // 2], a[..., r // 2:]
        out = torch.cat([u * cos - w * sin, w * cos + u * sin, rest], -1)
    else:
        u, w = a[..., 0::2], a[..., 1::2]
        out = torch.cat([torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2), rest], -1)
    return out.to(x.dtype)


def _plain_rope(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * s["inv_freq"][None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if c["backward"]:
        sin = -sin
    return dict(q=_rotate(s["q"], cos, sin, c), k=_rotate(s["k"], cos, sin, c))


def _scores(raw, s, slopes, q_pos, k_pos, allowed, prefix):
    """Scores with cap, bias and mask; also the cap's slope.  `raw` is scaled already; the rest broadcasts to it."""
    c = s["case"]
    slope_of_cap = None
    if c["softcap"]:
        t = torch.tanh(raw / c["softcap"])
        slope_of_cap = 1 - t * t
        raw = t * c["softcap"]
    if slopes is not None:
        raw = raw - slopes * (q_pos - k_pos).abs().float()
    near = torch.ones_like(allowed)
    if c["causal"]:
        near = near & (k_pos <= q_pos)
    if c["window"]:
        near = near & ((q_pos - k_pos).abs() < c["window"])
    if prefix is not None:
        near = near | (k_pos < prefix)
    return raw.masked_fill(~(allowed & near), float("-inf")), slope_of_cap


def _softmax(raw):
    m = raw.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(raw - m)
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, torch.ones_like(total)), (m + torch.log(total)).squeeze(-1)


def _plain_decode(s):
    c = s["case"]
    n, lq, cap, hq, hk, d = c["seqs"], c["q_len"], c["slot"], c["q_heads"], c["kv_heads"], c["head_dim"]
    gr = hq // hk
    q = s["q"].float().view(n, lq, hk, gr, d).permute(0, 2, 3, 1, 4).reshape(n, hk, gr * lq, d)
    k, v = (s[x].float().view(n, cap, hk, d).transpose(1, 2) for x in ("k", "v"))
    used = s["k_len"].long().view(n, 1, 1, 1, 1)
    k_pos = torch.arange(cap, device="cuda").view(1, 1, 1, 1, cap)
    q_pos = used - lq + torch.arange(lq, device="cuda").view(1, 1, 1, lq, 1)
    slopes = None if s["slopes"] is None else s["slopes"].view(1, hk, gr, 1, 1)
    prefix = None if s["prefix"] is None else s["prefix"].long().view(n, 1, 1, 1, 1)
    raw = (q @ k.transpose(-1, -2)).view(n, hk, gr, lq, cap) * s["scale"]
    raw, _ = _scores(raw, s, slopes, q_pos, k_pos, k_pos < used, prefix)
    p, lse = _softmax(raw)
    # a cache holds whatever was there behind the used part
    v = torch.where((k_pos < used).view(n, 1, cap, 1), v, torch.zeros_like(v))
    o = (p.view(n, hk, gr * lq, cap) @ v).view(n, hk, gr, lq, d).permute(0, 3, 1, 2, 4).reshape(n * lq, hq, d)
    return dict(o=o.to(s["q"].dtype), lse=lse.permute(1, 2, 0, 3).reshape(hq, n * lq))


def _plain_packed(s):
    c = s["case"]
    t, hq, hk, d = c["tokens"], c["q_heads"], c["kv_heads"], c["head_dim"]
    gr = hq // hk
    dt = s["q"].dtype

    def by_group(x):          # [t, hq, d] -> [hk, gr * t, d]
        return x.float().view(t, hk, gr, d).permute(1, 2, 0, 3).reshape(hk, gr * t, d)

    def by_row(x):            # [hk, gr * t, d] -> [t, hq, d]
        return x.view(hk, gr, t, d).permute(2, 0, 1, 3).reshape(t, hq, d).to(dt)

    row = torch.arange(t, device="cuda")
    seq = torch.searchsorted(s["q_off"][1:], row.to(torch.int32), right=True)
    pos = row - s["q_off"].long()[seq]
    q, k, v = by_group(s["q"]), s["k"].float().transpose(0, 1), s["v"].float().transpose(0, 1)
    slopes = None if s["slopes"] is None else s["slopes"].view(hk, gr, 1, 1)
    prefix = None if s["prefix"] is None else s["prefix"].long()[seq][:, None]
    raw = (q @ k.transpose(-1, -2)).view(hk, gr, t, t) * s["scale"]
    raw, cap = _scores(raw, s, slopes, pos[:, None], pos[None, :], seq[:, None] == seq[None, :], prefix)
    p, lse = _softmax(raw)
    del raw
    p = p.view(hk, gr * t, t)
    o = by_row(p @ v)
    if c["kind"] != "train":
        return dict(o=o, lse=lse.reshape(hq, t))
    do = by_group(s["do"])
    dv = p.transpose(-1, -2) @ do
    dp = do @ v.transpose(-1, -2)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    del dp, p
    if cap is not None:
        ds = ds * cap.view(hk, gr * t, t)
    dq, dk = (ds @ k) * s["scale"], (ds.transpose(-1, -2) @ q) * s["scale"]
    return dict(o=o, dq=by_row(dq), dk=dk.transpose(0, 1).contiguous().to(dt), dv=dv.transpose(0, 1).contiguous().to(dt))


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return _plain_rope(state) if kind == "rope" else _plain_decode(state) if kind == "decode" else _plain_packed(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def _pairs(case):
    """Visible (query, key) pairs of a head in a batch of equal sequences of this case's size."""
    if case["kind"] == "decode":
        used = case["slot"] * (31 / 32 if case["seqs"] == 1 else 9 / 16)   # the mean of the lengths that are drawn
        seen = min(used, case["window"]) if case["window"] and not case["prefix"] else used
        return case["seqs"] * case["q_len"] * seen, case["seqs"] * seen
    length = case["tokens"] / case["seqs"]
    per_row = length / 2 if case["causal"] else length
    if case["window"]:
        per_row = min(per_row, case["window"] * (1 if case["causal"] else 2))
    return case["tokens"] * per_row, case["tokens"]


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "rope":
        values = case["tokens"] * (hq + hk) * d
        return {"bytes": 2 * values * size + 4 * case["tokens"],
                "flops": 3 * case["tokens"] * (hq + hk) * case["rotary_dim"]}
    pairs, keys = _pairs(case)
    rows = case["seqs"] * case["q_len"] if case["kind"] == "decode" else case["tokens"]
    q_bytes, kv_bytes = rows * hq * d * size, keys * hk * d * size
    if case["kind"] == "train":   # q, do, o and dq; k, v, dk and dv; two products forward and five backward
        return {"bytes": 4 * q_bytes + 4 * kv_bytes, "flops": 7 * 2 * pairs * hq * d}
    return {"bytes": 2 * q_bytes + 2 * kv_bytes + 4 * rows * hq, "flops": 2 * 2 * pairs * hq * d}


# ---- the operators' definitions in 64 bits ----------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        turn = torch.exp(1j * s["positions"].double()[:, None] * s["inv_freq"])[:, None, :]
        if case["backward"]:
            turn = turn.conj()
        r = case["rotary_dim"]
        out = {}
        for name in ("q", "k"):
            y = s[name].double()
            if case["layout"] == "half":
                z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
                y[..., :r] = torch.cat([z.real, z.imag], -1)
            else:
                z = torch.complex(y[..., 0:r:2].contiguous(), y[..., 1:r:2].contiguous()) * turn
                y[..., :r] = torch.view_as_real(z).flatten(-2)
            out[name] = y
        return out
    hq, hk = case["q_heads"], case["kv_heads"]
    train = case["kind"] == "train"
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((hq, s["q"].shape[0]), float("-inf"), dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(o), *(torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in "kv")
    q_off, k_off = s["q_off"].tolist(), s["k_off"].tolist()
    for b in range(case["seqs"]):
        q0, q1, k0 = q_off[b], q_off[b + 1], k_off[b]
        n = k_off[b + 1] - k0 if s["k_len"] is None else int(s["k_len"][b])
        if q1 <= q0 or n <= 0:
            continue
        i = torch.arange(q1 - q0, device="cuda")[:, None] + (n - (q1 - q0))
        j = torch.arange(n, device="cuda")[None, :]
        seen = torch.ones(q1 - q0, n, dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen &= j <= i
        if case["window"]:
            seen &= (i - j < case["window"]) & (j - i < case["window"])
        if s["prefix"] is not None:
            seen |= j < int(s["prefix"][b])
        for h in range(hq):
            g = h // (hq // hk)
            q, k, v = s["q"][q0:q1, h].double(), s["k"][k0:k0 + n, g].double(), s["v"][k0:k0 + n, g].double()
            x = q @ k.T * s["scale"]
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
                cap = 1 - (x / case["softcap"]) ** 2
            if s["slopes"] is not None:
                x = x - s["slopes"][h].double() * (i - j).abs()
            x = torch.where(seen, x, -math.inf)
            z = torch.logsumexp(x, 1)
            p = torch.where(seen, torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[:, None]), 0.0)
            o[q0:q1, h], lse[h, q0:q1] = p @ v, z
            if train:
                do = s["do"][q0:q1, h].double()
                e = do @ v.T
                e = p * (e - (do * o[q0:q1, h]).sum(1, keepdim=True))
                if case["softcap"]:
                    e = e * cap
                dq[q0:q1, h] = e @ k * s["scale"]
                dk[k0:k0 + n, g] += e.T @ q * s["scale"]
                dv[k0:k0 + n, g] += p.T @ do
    return dict(o=o, dq=dq, dk=dk, dv=dv) if train else dict(o=o, lse=lse)
