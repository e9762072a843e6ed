"""Float64 oracle of the training losses and of the optimiser step (numpy, host
only; shares nothing with the library's kernels).

A token's log-probability is l = z_y - log sum exp(z), z = x / T.  A loss that
depends on the logits through l alone has d loss / d x_v = (d loss / d l)
(onehot_y(v) - p_v) / T.
"""
from __future__ import annotations

import numpy as np

SIGMOID, SQUARED, HINGE = 0, 1, 2


def rows(x, chosen, temperature=1.0):
    """(l [n], p [n][V]) of logit rows; a row with NaN or +inf, or without a
    finite logit, and one whose token is outside the vocabulary has l = NaN."""
    x = np.asarray(x, np.float64)
    chosen = np.asarray(chosen, np.int64)
    n, V = x.shape
    l, p = np.full(n, np.nan), np.full((n, V), np.nan)
    for t in range(n):
        if np.isnan(x[t]).any() or not np.isfinite(x[t].max()):
            continue
        z = (x[t] - x[t].max()) / temperature
        e = np.exp(z)
        p[t] = e / e.sum()
        if 0 <= chosen[t] < V:
            l[t] = z[chosen[t]] - np.log(e.sum())
    return l, p


def counted(n, mask, offsets):
    """(request of each row, -1 where the row does not count; counted rows of
    each request).  Without offsets all rows are request 0.  A row is looked up by
    bisection: the last request that begins at or before it, if its bounds hold the row
    and lie in the batch."""
    req = np.full(n, -1, np.int64)
    off = [0, n] if offsets is None else [int(v) for v in offsets]
    for t in range(n):
        first, end = 0, len(off) - 1  # the request is in [first, end)
        while end - first > 1:
            mid = (first + end) // 2
            if off[mid] <= t:
                first = mid
            else:
                end = mid
        a, b = off[first], off[first + 1]
        if 0 <= a <= t < b <= n and (mask is None or mask[t]):
            req[t] = first
    count = np.array([(req == r).sum() for r in range(len(off) - 1)], np.int64)
    return req, count


def _grad(p, chosen, slope, req, temperature, grad_scale):
    n, V = p.shape
    g = np.zeros((n, V))
    for t in range(n):
        if req[t] < 0 or slope[t] == 0:  # (a row that has no part in the loss may hold NaN)
            continue
        one = np.zeros(V)
        if 0 <= chosen[t] < V:
            one[chosen[t]] = 1.0
        g[t] = slope[t] * (one - p[t]) * (grad_scale / temperature)
    return g


def policy(x, chosen, advantage, old_logp=None, ref_logp=None, mask=None, offsets=None,
           clip_low=0.2, clip_high=0.2, kl_coef=0.0, temperature=1.0, requests=False,
           per_request=False, grad_scale=1.0):
    """(statistics [6], logp [n], gradient [n][V]) of the clipped policy loss."""
    n = len(chosen)
    l, p = rows(x, chosen, temperature)
    req, count = counted(n, mask, offsets)
    stats, slope = np.zeros(6), np.zeros(n)
    for t in range(n):
        if req[t] < 0:
            continue
        w = (1.0 / ((count > 0).sum() * count[req[t]])) if requests else 1.0 / count.sum()
        A = float(advantage[req[t]] if per_request else advantage[t])
        d = 0.0 * l[t] if old_logp is None else l[t] - float(old_logp[t])
        r = np.exp(d)
        free, cut = r * A, min(max(r, 1.0 - clip_low), 1.0 + clip_high) * A
        if np.isnan(r):
            cut = r
        clipped = cut < free
        surrogate = cut if clipped else free
        kl = 0.0
        slope[t] = w * (0.0 if clipped else -free)
        if ref_logp is not None:
            q = float(ref_logp[t]) - l[t]
            kl = np.expm1(q) - q
            if kl_coef != 0.0:
                slope[t] += w * kl_coef * -np.expm1(q)
        loss = -surrogate + (kl_coef * kl if kl_coef != 0.0 else 0.0)
        stats += w * np.array([loss, surrogate, kl, r, float(clipped), np.expm1(d) - d])
    logp = np.where(req >= 0, l, 0.0)
    return stats, logp, _grad(p, chosen, slope, req, temperature, grad_scale)


def preference(x, chosen, offsets, ref_logp=None, mask=None, beta=0.1, loss=SIGMOID,
               label_smoothing=0.0, margin=0.0, length_norm=False, temperature=1.0,
               grad_scale=1.0):
    """(statistics [5], log ratios [n_req], logp [n], gradient [n][V]) of the
    loss of paired log ratios, requests 2i preferred over 2i + 1."""
    n = len(chosen)
    l, p = rows(x, chosen, temperature)
    req, count = counted(n, mask, offsets)
    s = np.zeros(len(count))
    for t in range(n):
        if req[t] >= 0:
            s[req[t]] += l[t] - (0.0 if ref_logp is None else float(ref_logp[t]))
    if length_norm:
        s = s / np.maximum(count, 1)
    pairs = [i for i in range(0, len(count), 2) if count[i] > 0 and count[i + 1] > 0]
    stats, side = np.zeros(5), np.zeros(len(count))
    for i in pairs:
        d = s[i] - s[i + 1]
        h = beta * d - margin
        if loss == SIGMOID:
            f = sum(w * np.logaddexp(0, z) for w, z in ((1 - label_smoothing, -h),
                                                        (label_smoothing, h)) if w != 0)
            slope = beta * (label_smoothing * np.exp(-np.logaddexp(0, -h))
                            - (1 - label_smoothing) * np.exp(-np.logaddexp(0, h)))
        elif loss == SQUARED:
            f, slope = (d - 0.5 / beta) ** 2, 2 * (d - 0.5 / beta)
        else:
            f, slope = (h, h) if np.isnan(h) else (max(0.0, 1 - h), -beta if h < 1 else 0.0)
        stats += np.array([f, float(d > 0), h, beta * s[i], beta * s[i + 1]]) / len(pairs)
        for r, sign in ((i, 1.0), (i + 1, -1.0)):
            side[r] = sign * slope / len(pairs) / (count[r] if length_norm else 1)
    slope = np.where(req >= 0, side[np.maximum(req, 0)], 0.0)
    logp = np.where(req >= 0, l, 0.0)
    return stats, s, logp, _grad(p, chosen, slope, req, temperature, grad_scale)


# ---- the optimiser step --------------------------------------------------------------------


def adamw(p, g, m, v, lr, beta1, beta2, eps, step, weight_decay=0.0, grad_scale=1.0):
    """(p, m, v) after one AdamW step of one tensor."""
    p, g, m, v = (np.asarray(t, np.float64) for t in (p, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mhat, vhat = m / (1 - beta1 ** step), v / (1 - beta2 ** step)
    return p - lr * (mhat / (np.sqrt(vhat) + eps) + weight_decay * p), m, v


def held8(codes, scale, signed, block=256):
    """The values of 8-bit codes under their blocks' scales."""
    q = np.asarray(codes, np.float64)
    s = np.repeat(np.asarray(scale, np.float64), block)[:q.size]
    return q * np.abs(q) / 127.0 ** 2 * s if signed else q ** 4 / 255.0 ** 4 * s


def codes8(x, signed, block=256):
    """(unrounded codes, scales) of values in blocks: the root of the ratio to
    the block's largest magnitude, times 127 with a sign, or 255."""
    x = np.asarray(x, np.float64)
    scale = np.array([np.abs(x[i:i + block]).max() for i in range(0, x.size, block)])
    s = np.repeat(np.where(scale > 0, scale, 1.0), block)[:x.size]
    r = np.sqrt(np.abs(x) / s)
    return (np.sign(x) * r * 127.0 if signed else np.sqrt(r) * 255.0), scale
