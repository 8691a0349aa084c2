"""Float64 numpy reference of the rotary positions and the masked attention, sequence by sequence and head by head,
with bounds on how far a kernel that rounds its operands may be off (test infrastructure only)."""
from __future__ import annotations

import numpy as np

NONE, LINEAR, NTK, PARTS = range(4)
TINY = 2.0 ** -126


def rope_frequencies(rotary_dim, theta, scaling=NONE, factor=1.0, low_turns=1.0, high_turns=4.0, original=8192):
    i = np.arange(rotary_dim // 2, dtype=np.float64)
    if scaling == NTK:
        theta = theta * factor ** (rotary_dim / max(rotary_dim - 2, 1))
    w = theta ** (-2.0 * i / rotary_dim)
    if scaling == LINEAR:
        w = w / factor
    if scaling == PARTS:
        turns = original * w / (2.0 * np.pi)
        out = np.empty_like(w)
        for n, t in enumerate(turns):
            if t <= low_turns:
                out[n] = w[n] / factor
            elif t >= high_turns:
                out[n] = w[n]
            else:
                share = (t - low_turns) / (high_turns - low_turns)
                out[n] = share * w[n] + (1.0 - share) * w[n] / factor
        w = out
    return w


def rope(x, positions, inv_freq, interleaved=False, amplitude=1.0, backward=False):
    """x [tokens, heads, head_dim]; returns the turned values and |u| + |w| of each value's pair."""
    r = 2 * len(inv_freq)
    angle = np.asarray(positions, np.float64)[:, None] * inv_freq[None, :]
    cos, sin = amplitude * np.cos(angle)[:, None, :], amplitude * np.sin(angle)[:, None, :]
    if backward:
        sin = -sin
    y, size = np.array(x, np.float64), np.abs(np.array(x, np.float64))
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    u, w = np.array(x[..., a], np.float64), np.array(x[..., b], np.float64)
    y[..., a], y[..., b] = u * cos - w * sin, w * cos + u * sin
    size[..., a] = size[..., b] = abs(amplitude) * (np.abs(u) + np.abs(w))
    return y, size


def visible(lq, lk, causal=True, window=0, prefix=0):
    """[lq, lk] truth values: which key each query row sees (the last row stands at the last key)."""
    p = np.arange(lq)[:, None] + (lk - lq)
    j = np.arange(lk)[None, :]
    near = np.ones((lq, lk), bool)
    if causal:
        near &= j <= p
    if window:
        near &= np.abs(p - j) < window
    return near | (j < prefix)


def attention(q, k, v, q_off, k_off, k_len=None, prefix=None, slopes=None, scale=None, causal=True, window=0,
              softcap=0.0, d_o=None, p_step=0.0, out_step=2.0 ** -24, cap_rel=None):
    """Outputs and, with d_o, gradients, as a dict; `bound` holds for each how far a kernel may be off that forms scores
    and sums in fp32, rounds p and ds relatively by `p_step`, and its outputs (o before the backward pass too) by
    `out_step`.  Rows outside every sequence are NaN in both.

    The bounds: a score is a sum of D products in fp32, off by at most (D + 4) 2^-24 sum |q k| scale (the last factors'
    roundings included), a cap or a distance adds a few 2^-22 of its size (with `cap_rel` a cap adds that part of the
    score instead: for caps far above the scores); p is off relatively by twice the row's largest score error (its own
    and, through the sum, the others'), by n 2^-24 for the sum of n terms and by a few 2^-22 for the exponential:
    together `rel`.  fp32 (and bf16, which has its range) ends at 2^-126: a p, a ds, a product
    of theirs or an output below that may become zero, which is off by at most 2^-126 itself (`TINY`) and by
    that times the other factor in the sums it enters.  Everything below is the product rule over those."""
    hq, hk, dim = q.shape[1], k.shape[1], q.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    nan = np.nan
    out = dict(o=np.full(q.shape, nan), lse=np.full((hq, q.shape[0]), nan))
    bound = dict(o=np.full(q.shape, nan), lse=np.full((hq, q.shape[0]), nan))
    if d_o is not None:
        for n, like in (("d_q", q), ("d_k", k), ("d_v", v)):
            out[n], bound[n] = np.full(like.shape, nan), np.full(like.shape, nan)
    for b in range(len(q_off) - 1):
        q0, lq, k0, cap_rows = q_off[b], q_off[b + 1] - q_off[b], k_off[b], k_off[b + 1] - k_off[b]
        lk = cap_rows if k_len is None else min(max(int(k_len[b]), 0), cap_rows)
        qs, ks = slice(q0, q0 + lq), slice(k0, k0 + lk)
        seen = visible(lq, lk, causal, window, 0 if prefix is None else min(max(int(prefix[b]), 0), lk))
        dist = np.abs(np.arange(lq)[:, None] + (lk - lq) - np.arange(lk)[None, :])
        if d_o is not None:
            for n in ("d_k", "d_v"):
                out[n][ks], bound[n][ks] = 0.0, 0.0
        for h in range(hq):
            g = h // (hq // hk)
            Q, K, V = (np.asarray(x, np.float64) for x in (q[qs, h], k[ks, g], v[ks, g]))
            s = Q @ K.T * scale
            err = (dim + 4) * 2.0 ** -24 * (np.abs(Q) @ np.abs(K).T) * scale
            cap = np.ones_like(s)
            if softcap:
                t = np.tanh(s / softcap)
                cap = 1.0 - t * t
                s = softcap * t
                err = err + (softcap * 2.0 ** -20 if cap_rel is None else cap_rel * np.abs(s))
            if slopes is not None:
                s = s - float(slopes[h]) * dist
                err = err + 2.0 ** -22 * np.abs(s)
            err = err + 2.0 ** -22 * np.abs(s)
            s = np.where(seen, s, -np.inf)
            any_seen = seen.any(1)
            m = np.where(any_seen, s.max(1, initial=-np.inf), 0.0)
            e = np.where(seen, np.exp(s - m[:, None]), 0.0)
            l = e.sum(1)
            p = e / np.where(l > 0, l, 1.0)[:, None]
            with np.errstate(divide="ignore"):
                lse = np.where(any_seen, m + np.log(np.where(l > 0, l, 1.0)), -np.inf)
            worst = np.where(seen, err, 0.0).max(1, initial=0.0)
            rel = (2 * worst + (lk + dim + 16) * 2.0 ** -24 + 2.0 ** -20)[:, None]
            o, size = p @ V, p @ np.abs(V)
            o_bound = (rel + p_step) * size + out_step * (1 + rel + p_step) * size
            o_bound = o_bound + 2 * TINY * (1 + np.abs(V).sum(0, keepdims=True) + lk)
            out["o"][qs, h], bound["o"][qs, h] = o, o_bound
            out["lse"][h, qs] = lse
            bound["lse"][h, qs] = rel[:, 0] + 2.0 ** -22 * np.abs(np.where(any_seen, lse, 0.0))
            if d_o is None:
                continue
            G = np.asarray(d_o[qs, h], np.float64)
            dp, dp_size = G @ V.T, np.abs(G) @ np.abs(V).T
            delta, delta_size = (G * o).sum(1, keepdims=True), (np.abs(G) * np.abs(o)).sum(1, keepdims=True)
            delta_err = (np.abs(G) * o_bound).sum(1, keepdims=True) + (dim + 4) * 2.0 ** -24 * delta_size
            ds = p * (dp - delta) * cap
            ds_err = (p * (delta_err + (dim + 4) * 2.0 ** -24 * dp_size) + (rel + 2.0 ** -18 * bool(softcap)) * p *
                      (np.abs(dp - delta) + delta_err))
            ds_err = ds_err + p_step * (np.abs(ds) + ds_err) + 2 * TINY * (1 + np.abs(dp - delta) + delta_err)
            sums = 2.0 ** -24 * (max(lk, lq) * (hq // hk) + 16)     # a gradient's own sum in fp32

            def note(name, at, value, size_, err_, add):
                b_ = err_ + sums * size_ + 2 * TINY * (1 + max(lk, lq))
                if add:                                             # shared heads: rounded once, counted below
                    out[name][at] += value
                    bound[name][at] += b_
                else:
                    out[name][at], bound[name][at] = value, b_

            note("d_q", (qs, h), ds @ K * scale, np.abs(ds) @ np.abs(K) * scale, ds_err @ np.abs(K) * scale, False)
            note("d_k", (ks, g), ds.T @ Q * scale, np.abs(ds).T @ np.abs(Q) * scale, ds_err.T @ np.abs(Q) * scale, True)
            note("d_v", (ks, g), p.T @ G, p.T @ np.abs(G), ((rel + p_step) * p + 2 * TINY).T @ np.abs(G), True)
    for n in ("d_q", "d_k", "d_v"):
        if n in bound:
            bound[n] = bound[n] + out_step * (np.abs(out[n]) + bound[n])
    out["bound"] = bound
    return out
