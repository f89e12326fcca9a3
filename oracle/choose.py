"""Oracle of the drawn actions, the top logits and the student's loss (test
infrastructure only): the definitions in numpy doubles, row by row.  The GPU
library is a separate implementation of them.
"""
from __future__ import annotations

import math

import numpy as np


def order(z):
    """Columns in a row's order: larger logits first, equal ones by column;
    those of -inf left out."""
    z = np.asarray(z, np.float64) + 0.0
    at = np.lexsort((np.arange(len(z)), -z))
    return at[z[at] > -np.inf]


def left_out(z):
    z = np.asarray(z, np.float64)
    return bool(np.isnan(z).any() or not np.isfinite(z.max()))


def kept_columns(z, T, top_k=0, top_p=1.0, min_p=0.0):
    """(columns that a row keeps, in its order; how near top_p's border is to
    one of the sums, relative to their total)."""
    z = np.asarray(z, np.float64)
    at = order(z)
    e = np.exp((z[at] - z[at[0]]) / T)
    if 0 < top_k < len(z):
        at, e = at[:top_k], e[:top_k]
    length, near = len(at), np.inf
    if top_p < 1.0:
        sums = np.array([math.fsum(e[:i]) for i in range(len(e) + 1)]) if len(e) <= 64 else \
            np.concatenate([[0.0], np.cumsum(e)])
        P = top_p * sums[-1]
        length = int(np.sum(sums[:-1] < P))
        near = float(np.abs(sums[1:] - P).min() / sums[-1])
    if min_p > 0.0:
        length = min(length, int(np.sum(z[at] - z[at[0]] >= T * math.log(min_p))))
    return at[:length], near


def sample(z, u, T, top_k=0, top_p=1.0, min_p=0.0):
    """(actions, log-probabilities under z, how near each draw is to a border,
    relative to the sums it is drawn from)."""
    z = np.asarray(z, np.float32)
    n, C = z.shape
    action, logp, near = np.full(n, -1), np.zeros(n), np.full(n, np.inf)
    for i in range(n):
        if left_out(z[i]):
            continue
        zi = z[i].astype(np.float64)
        if T == 0:
            a = order(zi)[0]
        else:
            at, near[i] = kept_columns(zi, T, top_k, top_p, min_p)
            at = np.sort(at)
            sums = np.cumsum(np.exp((zi[at] - zi.max()) / T))
            x = float(u[i]) if u[i] > 0 else 0.0
            x = min(x, 1 - 2.0 ** -24) * sums[-1]
            a = at[np.argmax(sums > x)]
            gap = np.abs(sums[:-1] - x).min() / sums[-1] if len(at) > 1 else np.inf
            near[i] = min(near[i], gap)
        action[i] = a
        logp[i] = zi[a] - zi.max() - np.log(np.exp(zi - zi.max()).sum())
    return action, logp, near


def top_logits(z, k, T):
    z = np.asarray(z, np.float32)
    n, C = z.shape
    index, logq, rest = np.full((n, k), -1), np.full((n, k), -np.inf), np.zeros(n)
    for i in range(n):
        if left_out(z[i]):
            continue
        x = z[i].astype(np.float64)
        at = order(x)
        d = (x - x.max()) / T
        e = np.exp(d)
        m = min(k, len(at))
        index[i, :m] = at[:m]
        logq[i, :m] = d[at[:m]] - np.log(e.sum())
        rest[i] = e[at[m:]].sum() / e.sum()
    return index, logq, rest


def distill(z, index, logq, rest, weight, T):
    """dict of out, kl, dZ, live."""
    z = np.asarray(z, np.float64)
    n, C = z.shape
    w = np.full(n, 1.0 / max(n, 1)) if weight is None else np.asarray(weight, np.float64)
    kl, dz, live = np.zeros(n), np.zeros((n, C)), np.zeros(n, bool)
    with np.errstate(all="ignore"):
        for i in range(n):
            cols, lq = [], []
            for c, v in zip(index[i], logq[i]):
                if 0 <= c < C and c not in cols:
                    cols.append(int(c))
                    lq.append(float(v))
            if not cols or np.all(z[i] == -np.inf):
                continue
            r = 0.0 if rest is None or rest[i] <= 0 else float(rest[i])
            lq = np.array(lq + [np.log(r)])
            if np.all(lq == -np.inf):
                continue
            live[i] = True
            q = np.exp(lq - np.nanmax(lq))
            q = q / q.sum()
            lnq = lq - np.nanmax(lq) - np.log(np.exp(lq - np.nanmax(lq)).sum())
            x = z[i] / T
            top = np.nanmax(x)
            lnp = x - top - np.log(np.exp(x - top).sum())
            p = np.exp(lnp)
            other = np.ones(C, bool)
            other[cols] = False
            lo = lnp[other].max() if other.any() else -np.inf
            ln_other = lo + np.log(np.exp(lnp[other] - lo).sum()) if lo > -np.inf else -np.inf
            terms = np.append(lnp[cols], ln_other)
            kl[i] = T * T * sum(qj * (a - b) for qj, a, b in zip(q, lnq, terms) if qj != 0)
            g = p.copy()
            if q[-1] > 0 and ln_other > -np.inf:
                g[other] -= q[-1] * np.exp(lnp[other] - ln_other)
            for c, qj in zip(cols, q):
                g[c] = p[c] - qj
            if w[i] != 0:
                dz[i] = w[i] * T * g
        out = float(np.sum(np.where(live & (w != 0), w * kl, 0.0)))
    return dict(out=out, kl=kl, dZ=dz, live=live)
