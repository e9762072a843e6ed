"""Float64 oracle of the rows' first logits, of the loss of a list of a large model's first
tokens, and of the norm before the LM head (numpy, host only; shares nothing with the library's kernels).
"""
from __future__ import annotations

import numpy as np

from .loss import counted

FORWARD, REVERSE = 0, 1
CLASS, NONE = 0, 1
BIG = 1e9  # x / T from here on is infinite
RHO = 2.0 ** -24


def _logits(x, temperature):
    x = np.array(x, np.float64)
    big = float(np.float32(BIG * temperature))
    with np.errstate(invalid="ignore"):
        x[x >= big] = np.inf
        x[x <= -big] = -np.inf
    return x


def _logsumexp(z):
    top = z.max(initial=-np.inf)
    return top + np.log(np.exp(z - top).sum()) if np.isfinite(top) else top


def top_logits(x, k, temperature=1.0):
    """(ids [n][k], log-probabilities [n][k]): value descending, index ascending."""
    x = _logits(x, temperature)
    n, V = x.shape
    ids, logp = np.full((n, k), -1, np.int64), np.full((n, k), -np.inf)
    for t in range(n):
        if np.isnan(x[t]).any() or not np.isfinite(x[t].max()):
            logp[t] = np.nan
            continue
        order = np.argsort(-x[t], kind="stable")[:k]
        order = order[np.isfinite(x[t][order])]
        ids[t, :len(order)] = order
        logp[t, :len(order)] = x[t][order] / temperature - _logsumexp(x[t] / temperature)
    return ids, logp


def _row(z, ids, sent, y, loss, rest, ce_on):
    """One row: (KL, CE, mass of p, mass of q, a over the entries, b, whether the row is
    wrong).  Entries: distinct ids in the vocabulary."""
    V = len(z)
    lse = _logsumexp(z)
    l = z - lse
    out = np.ones(V, bool)
    out[ids] = False
    ce = -l[y] if ce_on else 0.0
    p, q, ls = np.exp(sent), np.exp(l[ids]), l[ids]
    mass_p, mass_q = p.sum(), q.sum()
    kl, a, b = 0.0, np.zeros(len(ids)), 0.0
    size_a, size_b, size = np.zeros(len(ids)), 0.0, 0.0
    if len(ids):
        l_sigma = _logsumexp(l[out]) if out.any() else -np.inf
        klass = rest == CLASS and l_sigma > -np.inf
        sigma, rho = np.exp(l_sigma), max(1.0 - mass_p, RHO)
        if rest == NONE:
            sent = sent - _logsumexp(sent)
            p = np.exp(sent)
        if loss == FORWARD:
            with np.errstate(invalid="ignore"):
                terms = np.where(p > 0, p * (sent - ls), 0.0)
            a, size_a = -p, p
            size = (p * (np.abs(sent) + np.where(p > 0, np.abs(ls), 0))).sum()
            kl = terms.sum()
            if klass:
                kl += rho * (np.log(rho) - l_sigma)
                b, size_b = -rho, rho
                size += rho * (abs(np.log(rho)) + abs(l_sigma))
        else:
            if rest == NONE:
                if not np.isfinite(ls).any():
                    return None
                ls = ls - _logsumexp(ls)
                q = np.exp(ls)
            with np.errstate(invalid="ignore"):
                f = np.where(q > 0, ls - sent, 0.0)
            kl = (q * f).sum()
            size = (q * (1.0 + np.abs(f) + np.abs(sent))).sum()
            if klass:
                kl += sigma * (l_sigma - np.log(rho))
                size += sigma * (1.0 + abs(l_sigma) + 2 * abs(np.log(rho)))
            a, size_a = q * (f - kl), q * (1.0 + np.abs(f) + abs(kl) + np.abs(sent))
            if klass:
                b = sigma * (l_sigma - np.log(rho) - kl)
                size_b = sigma * (1.0 + abs(l_sigma) + 2 * abs(np.log(rho)) + abs(kl))
    return kl, ce, mass_p, mass_q, a, b, size, size_a, size_b, l, out


def distill(x, ids, sent, chosen=None, mask=None, offsets=None, kl_coef=1.0, ce_coef=0.0,
            temperature=1.0, loss=FORWARD, rest=CLASS, requests=False, grad_scale=1.0):
    """(statistics [5], KL [n], gradient [n][V], and what roundings are relative to: the
    sizes of KL's terms [n] and of the gradient's [n][V])."""
    x = _logits(x, temperature)
    n, V = x.shape
    req, count = counted(n, mask, offsets)
    stats, kls = np.zeros(5), np.zeros(n)
    grad, sizes, gsize = np.zeros((n, V)), np.zeros(n), np.zeros((n, V))
    for t in range(n):
        if req[t] < 0:
            continue
        w = (1.0 / ((count > 0).sum() * count[req[t]])) if requests else 1.0 / count.sum()
        on = (np.asarray(ids[t]) != -1) & (np.asarray(sent[t]) != -np.inf)
        s, p = np.asarray(ids[t], np.int64)[on], np.asarray(sent[t], np.float64)[on]
        y = -1 if chosen is None else int(chosen[t])
        wrong = ((s < 0).any() or (s >= V).any() or len(set(s.tolist())) < len(s)
                 or (chosen is not None and not 0 <= y < V) or np.isnan(p).any()
                 or (p == np.inf).any() or np.isnan(x[t]).any() or not np.isfinite(x[t].max()))
        r = None if wrong else _row(x[t] / temperature, s, p, y, loss, rest, chosen is not None)
        if r is None:
            kls[t] = np.nan
            grad[t] = np.nan
            stats += np.nan
            continue
        kl, ce, mass_p, mass_q, a, b, size, size_a, size_b, l, out = r
        kls[t], sizes[t] = kl, size
        total = (kl_coef * kl if kl_coef else 0.0) + (ce_coef * ce if ce_coef else 0.0)
        stats += w * np.array([total, kl, ce, mass_p, mass_q])
        q = np.exp(l)
        A = kl_coef * (a.sum() + b) - (ce_coef if chosen is not None else 0.0)
        g, gs = -A * q, abs(A) * q
        g[s] += kl_coef * a
        gs[s] += kl_coef * size_a
        if b or size_b:
            share = np.where(out, np.exp(l - _logsumexp(l[out])), 0.0)
            g += kl_coef * b * share
            gs += kl_coef * size_b * share
        if chosen is not None:
            g[y] -= ce_coef
            gs[y] += ce_coef
        grad[t] = g * (w * grad_scale / temperature)
        gsize[t] = gs * abs(w * grad_scale / temperature)
    return stats, kls, grad, sizes, gsize


def norm(h, weight, bias=None, eps=1e-5, rms=False):
    """(y, mean or None, 1 / deviation) of rows."""
    h, weight = np.asarray(h, np.float64), np.asarray(weight, np.float64)
    mean = np.zeros(len(h)) if rms else h.mean(axis=1)
    mid = h - mean[:, None]
    rstd = 1.0 / np.sqrt((mid ** 2).mean(axis=1) + eps)
    y = mid * rstd[:, None] * weight
    return (y if bias is None else y + np.asarray(bias, np.float64)), (None if rms else mean), rstd


def norm_backward(dy, h, weight, mean, rstd, dtotal=None, rms=False):
    """(dx, dweight, dbias) from given moments."""
    dy, h, weight = (np.asarray(t, np.float64) for t in (dy, h, weight))
    hat = (h if rms else h - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    g = dy * weight
    dx = g - hat * (g * hat).mean(axis=1, keepdims=True)
    if not rms:
        dx = dx - g.mean(axis=1, keepdims=True)
    dx = dx * np.asarray(rstd, np.float64)[:, None]
    return (dx if dtotal is None else dx + np.asarray(dtotal, np.float64)), (dy * hat).sum(0), dy.sum(0)
