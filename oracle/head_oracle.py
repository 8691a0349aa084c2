"""Float64 reference of the losses on the output head, row by row over the whole vocabulary, with bounds on how far a kernel
that rounds its operands may be off (test infrastructure only; torch tensors of any device)."""
from __future__ import annotations

import torch

TINY = 2.0 ** -126


def teacher(index, logit, vocab, temperature=1.0, teacher_lse=None):
    """Rows over the whole vocabulary: target probabilities, which columns are listed, what is left over, and which tokens
    count."""
    idx, u = index.long(), logit.double() / temperature
    t, k = idx.shape
    inside = (idx >= 0) & (idx < vocab)
    target = torch.zeros(t, vocab, dtype=torch.float64, device=idx.device)
    named = torch.zeros(t, vocab, dtype=torch.bool, device=idx.device)
    counted = inside.any(1)
    for i in range(t):
        cols, vals = idx[i][inside[i]], u[i][inside[i]]
        if cols.numel() == 0:
            continue
        if teacher_lse is None:
            if bool((vals == -float("inf")).all()):
                counted[i] = False
                continue
            q = torch.softmax(vals, 0)
        else:
            q = torch.exp(vals - teacher_lse[i].double())
        target[i].index_put_((cols,), q, accumulate=True)
        named[i, cols] = True
    rest = torch.zeros(t, dtype=torch.float64, device=idx.device)
    if teacher_lse is not None:
        rest = (1.0 - target.sum(1)).clamp_min(0.0)
        rest = torch.where(named.all(1) | ~counted, torch.zeros_like(rest), rest)
    return target, named, rest, counted


def label_rows(labels, vocab):
    y = labels.long()
    counted = (y >= 0) & (y < vocab)
    target = torch.zeros(y.numel(), vocab, dtype=torch.float64, device=y.device)
    rows = torch.nonzero(counted)[:, 0]
    target[rows, y[rows]] = 1.0
    return target, target > 0, torch.zeros(y.numel(), dtype=torch.float64, device=y.device), counted


def head(x, w, target, named, rest, counted, scale=1.0, softcap=0.0, temperature=1.0, z_loss=0.0, weights=None,
         normalizer=None, p_step=0.0, out_step=2.0 ** -24, gradient=True):
    """Outputs, and in `bound` how far off a kernel may be that sums logits in fp32 and rounds the factors of the gradient's
    product relatively by `p_step` (those that are not listed up to twice) and d_x by `out_step`.

    A logit is a sum of d products, each addition off by at most 2^-23 (nearest or truncated) of what is summed, and a few
    roundings; a cap adds 2^-21 of the logit (tanh) and passes the rest on.  `far` is a row's largest such error.  A
    probability is off relatively by twice `far`, by the sum over the vocabulary and by the exponential (2^-20 together with
    the roundings around them): `rel`.  Everything below is the product rule over those; fp32 ends at 2^-126, which is
    TINY."""
    f64 = torch.float64
    x, w = x.to(f64), w.to(f64)
    t, d = x.shape
    v = w.shape[0]
    raw = x @ w.T * scale
    err = (d + 8) * 2.0 ** -23 * (x.abs() @ w.abs().T) * scale
    slope, slope_err = torch.ones_like(raw), torch.zeros_like(raw)
    if softcap:
        th = torch.tanh(raw / softcap)
        slope = 1 - th * th
        slope_err = 2 * (err / softcap) + 2.0 ** -20
        raw = softcap * th
        err = err + 2.0 ** -21 * raw.abs()
    z = raw / temperature
    err = err / temperature + 2.0 ** -21 * z.abs()
    far = err.max(1).values
    rel = 2 * far + (v + 64) * 2.0 ** -24 + 2.0 ** -20
    lse = torch.logsumexp(z, 1)
    log_p = z - lse[:, None]
    p = torch.exp(log_p)
    # ln of what the listed columns leave to the student, without a difference from one
    log_rest = torch.logsumexp(log_p.masked_fill(named, -float("inf")), 1)
    cross = torch.where(target > 0, target * (torch.log(target.clamp_min(1e-300)) - log_p), torch.zeros_like(z)).sum(1)
    one_hot = (named.sum(1) == 1) & (target.sum(1) == 1.0) & (rest == 0)
    z_named = z.masked_fill(~named, -float("inf")).max(1).values
    gap = lse + log_rest - z_named
    soft = torch.clamp_min(gap, 0.0) + torch.log1p(torch.exp(-gap.abs()))
    loss = torch.where(one_hot, soft, cross)
    some = rest > 0
    loss = loss + torch.where(some, rest * (torch.log(rest.clamp_min(1e-300)) - log_rest), torch.zeros_like(rest))
    loss = loss + z_loss * lse ** 2
    zero = torch.zeros_like(loss)
    miss = torch.sigmoid(gap)
    loss_bound = torch.where(one_hot, miss * torch.exp(rel) * rel, (target.sum(1) + rest) * rel)
    loss_bound = loss_bound + z_loss * (2 * lse.abs() + rel) * rel + 2.0 ** -22 * loss.abs() + TINY
    lse_bound = rel + 2.0 ** -23 * lse.abs()
    weight = torch.ones_like(loss) if weights is None else weights.to(f64)
    weight = torch.where(counted, weight, zero)
    loss, lse_out = torch.where(counted, loss, zero), torch.where(counted, lse, zero)
    total = weight.sum()
    out = dict(loss=loss, lse=lse_out, totals=torch.stack([(weight * loss).sum(), total]))
    bound = dict(loss=torch.where(counted, loss_bound, zero), lse=torch.where(counted, lse_bound, zero),
                 totals=torch.stack([(weight.abs() * (loss_bound + 2.0 ** -23 * loss.abs())).sum() +
                                     2.0 ** -23 * (weight * loss).sum().abs(), 2.0 ** -23 * weight.abs().sum() + TINY]))
    if gradient:
        norm = total if normalizer is None else normalizer
        each = weight / norm * (scale / temperature) if norm != 0 else zero
        curl = 2 * z_loss * lse
        part = torch.where(some, rest / torch.exp(log_rest).clamp_min(1e-300), zero)
        share = (target.sum(1) + rest + curl - part)[:, None]
        g = torch.where(named, (target.sum(1) + rest + curl)[:, None] * p - target, share * p)
        g = torch.where(one_hot[:, None] & named, -miss[:, None] + curl[:, None] * p, g)
        size = (1 + curl.abs() + part)[:, None] * rel[:, None] + 2 * z_loss * rel[:, None] + 2.0 ** -30 * (1 + part)[:, None]
        g_err = torch.where(named, (1 + curl.abs())[:, None] * p * rel[:, None] + 2 * z_loss * p * rel[:, None] +
                            2.0 ** -22 * (target + p), size * p)
        tight = miss[:, None] * (rel[:, None] + 2.0 ** -22) + (curl.abs() + 2 * z_loss)[:, None] * p * rel[:, None]
        g_err = torch.where(one_hot[:, None] & named, tight, g_err)
        g_err = g_err * (slope + slope_err) + g.abs() * slope_err
        g = g * slope
        # a column that is not listed is rounded itself, and its row's factor may be moved by as much again
        g_err = g_err + torch.where(named, p_step, 2 * p_step + p_step ** 2) * (g.abs() + g_err) + 2.0 ** -60 * p.max(1, keepdim=True).values + TINY
        d_x = each[:, None] * (g @ w)
        size = g.abs() @ w.abs()
        b = each.abs()[:, None] * (g_err @ w.abs() + (v + 32) * 2.0 ** -23 * (size + g_err @ w.abs()))
        bound["d_x"] = torch.where(counted[:, None], b + out_step * (d_x.abs() + b) + TINY, torch.zeros_like(b))
        out["d_x"] = torch.where(counted[:, None], d_x, torch.zeros_like(d_x))
    out["bound"] = bound
    return out
