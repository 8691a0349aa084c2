"""Cases of the losses at the end of a MixLoRA model, for timing and comparison.

Two operators, both of the product of the last hidden states with the frozen output head, whose logits are never kept:
softmax cross entropy (`mixlora_head_loss`) and distillation from a teacher's top logits (`mixlora_head_distill`), each
with its gradient towards the hidden states or without.  `run` computes them from elementary torch operations, or, where
`own` is true, with the library's calls.  `exact` computes the same outputs in 64 bits, a few rows at a time.

A case's kind:
  loss         labels; loss and log-sum-exp of every token, totals, and d_x if `grad`
  distill      `top` teacher logits a token; the same outputs
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

LOSS = dict(kind="loss", dtype="bf16", tokens=1, vocab=32000, d_model=4096, grad=False, top=0, tail=False,
            temperature=1.0, skipped=0.0, weighted=False, softcap=0.0, z_loss=0.0, scale=1.0, packed=False)
DISTILL = dict(LOSS, kind="distill", top=16)


def listed():
    return [
        # the log-probability of one token while serving the 7B block
        dict(LOSS, name="loss-1"),
        # scoring the answers of a few requests against a vocabulary that no tile divides, capped logits
        dict(LOSS, name="loss-37-odd-vocab", tokens=37, vocab=50257, d_model=1280, softcap=30.0),
        # perplexity of a batch of the 7B block, no gradient
        dict(LOSS, name="loss-4096", tokens=4096),
        # a training step on one short sequence
        dict(LOSS, name="train-512", tokens=512, grad=True, z_loss=1e-4),
        # the training batch of the 7B block: 16 sequences of 512
        dict(LOSS, name="train-8192", tokens=8192, grad=True),
        # instruction tuning at the 13B width: prompts carry no label, answers are weighted, a wide odd vocabulary
        dict(LOSS, name="train-5003-answers", tokens=5003, vocab=100003, d_model=5120, grad=True, skipped=0.6,
             weighted=True, packed=True),
        # the fp32 check mode
        dict(LOSS, name="train-fp32-700", dtype="fp32", tokens=700, vocab=8009, d_model=1024, grad=True, softcap=20.0),
        # distillation of a small batch at a raised temperature, the listed entries alone
        dict(DISTILL, name="distill-333", tokens=333, d_model=2048, grad=True, top=8, temperature=2.0),
        # distillation of a training batch from 64 entries a token, what they leave over as one more class
        dict(DISTILL, name="distill-4096-tail", tokens=4096, grad=True, top=64, tail=True, temperature=1.5,
             skipped=0.1),
        # how far a student is from its teacher on one request, no gradient
        dict(DISTILL, name="distill-eval-19", tokens=19, vocab=50257, d_model=1280, top=20, tail=True),
        # the fp32 check mode, weighted tokens
        dict(DISTILL, name="distill-fp32-257", dtype="fp32", tokens=257, vocab=5003, d_model=768, grad=True, top=5,
             tail=True, weighted=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    d = 8 * _spread(rng, 16, 160 if dtype == "fp32" else 640)
    vocab = _spread(rng, 500, 16384 if dtype == "fp32" else 131072)
    most = min(8192, 260_000_000 // vocab, 1_000_000_000_000 // (vocab * d))
    if dtype == "fp32":
        most = min(most, 1024, 6_000_000_000 // (vocab * d))
    tokens = _spread(rng, 1, max(1, most))
    base = dict(dtype=dtype, tokens=tokens, vocab=vocab, d_model=d, grad=rng.random() < 0.7,
                skipped=rng.choice([0.0, 0.0, 0.3, 0.7]), weighted=rng.random() < 0.3,
                softcap=rng.choice([0.0, 0.0, 0.0, 30.0]), z_loss=rng.choice([0.0, 0.0, 1e-4]),
                scale=rng.choice([1.0, 1.0, 0.5]), packed=rng.random() < 0.3)
    if rng.random() < 0.55:
        return dict(LOSS, **base)
    return dict(DISTILL, **base, top=_spread(rng, 1, 128), tail=rng.random() < 0.5,
                temperature=rng.choice([1.0, 2.0, 4.0]))


# ---- inputs -----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, t, v, d = DTYPES[case["dtype"]], case["tokens"], case["vocab"], case["d_model"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)

    # logits of unrelated tokens spread by 2; each token leans towards its label by 0 to 16
    w = (normal(v, d) * (2 * d ** -0.5)).to(dt)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda")
    x = (normal(t, d) + 4 * uniform(t, 1) * w[labels].float()).to(dt)
    if case["packed"]:      # hidden states that are parts of wider rows
        wide = torch.zeros(t, d + 64, dtype=dt, device="cuda")
        wide[:, :d] = x
        x = wide[:, :d]
    skip = uniform(t) < case["skipped"]
    skip[0] = False
    s = dict(case=case, x=x, w=w, weights=uniform(t) + 0.25 if case["weighted"] else None)
    if case["kind"] == "loss":
        s["labels"] = torch.where(skip, torch.full_like(labels, -100), labels).to(torch.int32)
    else:
        k = min(case["top"], v)
        index, logit, rest = [], [], []
        for a in range(0, t, 1024):     # a teacher that agrees with the student in part
            z = ((x[a:a + 1024].float() + 0.5 * normal(min(1024, t - a), d)).to(dt) @ w.T).float()
            top = torch.topk(z, k, dim=1)
            index.append(top.indices)
            logit.append(top.values)
            rest.append(torch.logsumexp(z.double() / case["temperature"], 1).float())
        index, logit = torch.cat(index), torch.cat(logit)
        # lists end early where a teacher's sampling cut them off
        kept = 1 + (uniform(t, 1) * 2 * k).long()
        gone = (torch.arange(k, device="cuda")[None, :] >= kept) | skip[:, None]
        s["index"] = torch.where(gone, torch.full_like(index, -1), index).to(torch.int32)
        s["logit"] = logit.contiguous()
        s["teacher_lse"] = torch.cat(rest) if case["tail"] else None
    if own:
        s["plan"] = _plan(s)
    return s


def _plan(s):
    """What a program keeps for this shape: the shape, the outputs and the workspace."""
    from paper_2404_15159_b200 import binding as B
    c, x = s["case"], s["x"]
    shape = B.make_head_shape(c["tokens"], c["d_model"], c["vocab"],
                              B.MIXLORA_DTYPE_BF16 if c["dtype"] == "bf16" else B.MIXLORA_DTYPE_FP32,
                              teacher_top=0 if c["kind"] == "loss" else s["index"].shape[1], scale=c["scale"],
                              softcap=c["softcap"], temperature=c["temperature"], z_loss=c["z_loss"],
                              x_stride=x.stride(0))
    f32 = dict(dtype=torch.float32, device="cuda")
    return dict(B=B, shape=shape, workspace=B.alloc_head_workspace(shape, c["grad"]),
                loss=torch.empty(c["tokens"], **f32), lse=torch.empty(c["tokens"], **f32),
                totals=torch.empty(2, **f32),
                d_x=torch.empty(c["tokens"], c["d_model"], dtype=x.dtype, device="cuda") if c["grad"] else None)


# ---- the library's calls ----------------------------------------------------------------------------------------

def _own(s):
    p = s["plan"]
    B = p["B"]
    if s["case"]["kind"] == "loss":
        B.mixlora_head_loss(p["shape"], s["x"], s["w"], s["labels"], s["weights"], None, p["loss"], p["lse"],
                            p["totals"], p["d_x"], p["workspace"])
    else:
        B.mixlora_head_distill(p["shape"], s["x"], s["w"], s["index"], s["logit"], s["teacher_lse"], s["weights"],
                               None, p["loss"], p["lse"], p["totals"], p["d_x"], p["workspace"])
    out = dict(loss=p["loss"], lse=p["lse"], totals=p["totals"])
    if p["d_x"] is not None:
        out["d_x"] = p["d_x"]
    return out


# ---- the plain forms --------------------------------------------------------------------------------------------

def _targets(s):
    """Listed columns [t, k], which of them count, their probabilities, and what they leave over."""
    c = s["case"]
    if c["kind"] == "loss":
        idx = s["labels"].long()[:, None]
        valid = (idx >= 0) & (idx < c["vocab"])
        return idx.clamp(0, c["vocab"] - 1), valid, valid.double(), None
    idx = s["index"].long()
    valid = (idx >= 0) & (idx < c["vocab"])
    u = (s["logit"].double() / c["temperature"]).masked_fill(~valid, float("-inf"))
    if s["teacher_lse"] is None:
        top = u.amax(1, keepdim=True)
        e = torch.exp(u - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        q = e / e.sum(1, keepdim=True).clamp_min(1e-300)
        return idx.clamp(0, c["vocab"] - 1), valid, q, None
    q = torch.exp(u - s["teacher_lse"].double()[:, None])
    return idx.clamp(0, c["vocab"] - 1), valid, q, (1 - q.sum(1)).clamp_min(0)


def _log_times(q):
    return torch.where(q > 0, q * torch.log(q), torch.zeros_like(q))


def _plain(s):
    c = s["case"]
    tau, zeta = c["temperature"], c["z_loss"]
    idx, valid, q, rest = _targets(s)
    counted = valid.any(1)
    w = s["w"].float()
    z = (s["x"].float() @ w.T) * c["scale"]
    if c["softcap"]:
        z = torch.tanh(z / c["softcap"]) * c["softcap"]
    listed_ = torch.zeros(z.shape, dtype=torch.int8, device="cuda").scatter_add_(1, idx, valid.to(torch.int8)) > 0
    others = (z / tau).masked_fill(listed_, float("-inf"))
    top = others.amax(1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    lo = (top.double()[:, 0] + torch.log(torch.exp(others - top).sum(1).double()))   # log-sum-exp of the columns not listed
    # from here the listed columns alone, in 64 bits: a divergence is a small difference of their terms
    zk = torch.gather(z, 1, idx).double() / tau
    slope_k = 1 - (zk * tau / c["softcap"]) ** 2 if c["softcap"] else 1.0
    zl = zk.masked_fill(~valid, float("-inf"))
    m = torch.maximum(zl.amax(1), lo)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    lse = m + torch.log(torch.exp(zl - m[:, None]).sum(1) + torch.exp(lo - m))
    p_k = torch.where(valid, torch.exp(zk - lse[:, None]), torch.zeros_like(zk))
    share = 1 + 2 * zeta * lse
    if c["kind"] == "loss":
        gap = lo - zk[:, 0]
        loss = torch.where(gap > 0, gap, torch.zeros_like(gap)) + torch.log1p(torch.exp(-gap.abs()))
        g_k = -torch.sigmoid(gap)[:, None] + 2 * zeta * lse[:, None] * p_k
    else:
        loss = (_log_times(q) - torch.where(q > 0, q * (zk - lse[:, None]), torch.zeros_like(q))).sum(1)
        g_k = share[:, None] * p_k - q
        if rest is not None:
            loss = loss + _log_times(rest) - torch.where(rest > 0, rest * (lo - lse), torch.zeros_like(rest))
            share = share - torch.where(rest > 0, rest / torch.exp(lo - lse), torch.zeros_like(rest))
    loss = loss + zeta * lse * lse
    zero = torch.zeros_like(loss)
    loss, lse_out = torch.where(counted, loss, zero), torch.where(counted, lse, zero)
    weight = counted.double() if s["weights"] is None else torch.where(counted, s["weights"].double(), zero)
    totals = torch.stack([(weight * loss).sum(), weight.sum()])
    out = dict(loss=loss.float(), lse=lse_out.float(), totals=totals.float())
    if c["grad"]:
        each = torch.where(counted, weight / totals[1] * (c["scale"] / tau), zero).float()
        p = torch.exp(others - lse.float()[:, None]) * share.float()[:, None]
        if c["softcap"]:
            p = p * (1 - (z / c["softcap"]) ** 2)
        p = p.scatter_add_(1, idx, torch.where(valid, g_k * slope_k, torch.zeros_like(g_k)).float())
        out["d_x"] = ((p @ w) * each[:, None]).masked_fill(~counted[:, None], 0.0).to(s["x"].dtype)
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    t, v, d = case["tokens"], case["vocab"], case["d_model"]
    rows = max(1.0, t * (1 - case["skipped"]))
    products = 2 if case["grad"] else 1
    lists = t * (4 if case["kind"] == "loss" else 8 * case["top"] + (4 if case["tail"] else 0))
    return {"bytes": v * d * size + rows * d * size + (t * d * size if case["grad"] else 0) + 8 * t + lists,
            "flops": products * 2.0 * rows * v * d}


# ---- the operators' definitions in 64 bits ----------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c, t, v = case, case["tokens"], case["vocab"]
    tau, zeta, cap = c["temperature"], c["z_loss"], c["softcap"]
    w = s["w"].double()
    loss = torch.zeros(t, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(loss)
    weight = torch.zeros_like(loss)
    given = torch.ones_like(loss) if s["weights"] is None else s["weights"].double()
    columns = s["labels"].long()[:, None] if c["kind"] == "loss" else s["index"].long()
    inside = (columns >= 0) & (columns < v)
    some = inside.any(1)
    weight[some] = given[some]
    total = weight.sum()
    d_x = torch.zeros(t, c["d_model"], dtype=torch.float64, device="cuda") if c["grad"] else None
    step = max(1, 60_000_000 // v)
    for a in range(0, t, step):
        rows = torch.nonzero(some[a:a + step])[:, 0] + a
        if rows.numel() == 0:
            continue
        raw = s["x"][rows].double() @ w.T * c["scale"]
        u = cap * torch.tanh(raw / cap) if cap else raw
        z = u / tau
        log_z = torch.logsumexp(z, 1, keepdim=True)
        log_p = z - log_z
        # the target as a row over the whole vocabulary, and which of its columns are listed
        target = torch.zeros_like(z)
        named = torch.zeros(z.shape, dtype=torch.bool, device="cuda")
        r, k = torch.nonzero(inside[rows], as_tuple=True)
        cols = columns[rows][r, k]
        if c["kind"] == "loss":
            prob = torch.ones(r.numel(), dtype=torch.float64, device="cuda")
        else:
            prob = torch.exp(s["logit"][rows].double()[r, k] / tau -
                             (s["teacher_lse"][rows].double()[r] if c["tail"] else 0.0))
        target.index_put_((r, cols), prob, accumulate=True)
        named[r, cols] = True
        if c["kind"] == "distill" and not c["tail"]:
            target = target / target.sum(1, keepdim=True)
        grad = torch.exp(log_p) * target.sum(1, keepdim=True) - target
        one = torch.special.xlogy(target, target).sum(1) - (target * log_p).sum(1)
        if c["tail"]:
            left = (1 - target.sum(1)).clamp_min(0.0)
            log_rest = torch.logsumexp(log_p.masked_fill(named, -math.inf), 1)
            one = one + torch.special.xlogy(left, left) - torch.where(left > 0, left * log_rest, 0.0)
            inner = torch.exp(log_p - log_rest[:, None]).masked_fill(named, 0.0)
            grad = grad + left[:, None] * (torch.exp(log_p) - inner)
        loss[rows] = one + zeta * log_z[:, 0] ** 2
        lse[rows] = log_z[:, 0]
        if d_x is not None:
            grad = grad + 2 * zeta * log_z * torch.exp(log_p)
            if cap:
                grad = grad * (1 - (u / cap) ** 2)
            d_x[rows] = grad @ w * (weight[rows] / total * c["scale"] / tau)[:, None]
    out = dict(loss=loss, lse=lse, totals=torch.stack([(weight * loss).sum(), total]))
    if d_x is not None:
        out["d_x"] = d_x
    return out
