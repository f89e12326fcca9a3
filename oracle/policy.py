"""Oracle of the policy loss, the gradient norm and AdamW (test
infrastructure only): the definitions in numpy doubles, row by row and
element by element.  The GPU library is a separate implementation of them.
"""
from __future__ import annotations

import numpy as np

from .frontier import GOLDEN, M64, splitmix_output

BLOCK = 256
TINY = 2.0 ** -126


def action_logp(z, action):
    """(log-probabilities, rows that take part): 0 for rows whose action is
    outside [0, C), -inf for rows without any logit above -inf."""
    z = np.asarray(z, np.float64)
    n, C = z.shape
    lp, live = np.zeros(n), np.zeros(n, bool)
    for i in range(n):
        a = int(action[i])
        if not 0 <= a < C:
            continue
        if np.all(z[i] == -np.inf):
            lp[i] = -np.inf
            continue
        live[i] = True
        top = np.max(z[i])
        with np.errstate(invalid="ignore", over="ignore"):
            lp[i] = z[i, a] - top - np.log(np.sum(np.exp(z[i] - top)))
    return lp, live


def policy_loss(z, action, adv, old=None, ref=None, weight=None, lo=0.2, hi=0.2, beta=0.0):
    """dict of out (3), logp, dZ, and per row slope (w dl/dlp), rho, kl, cut."""
    z = np.asarray(z, np.float64)
    n, C = z.shape
    lp, live = action_logp(z, action)
    w = np.full(n, 1.0 / max(n, 1)) if weight is None else np.asarray(weight, np.float64)
    out, dz = np.zeros(3), np.zeros((n, C))
    slope, rho, kl, cut = np.zeros(n), np.ones(n), np.zeros(n), np.zeros(n, bool)
    with np.errstate(all="ignore"):
        for i in range(n):
            if not live[i] or w[i] == 0:
                continue
            A = float(adv[i])
            rho[i] = 1.0 if old is None else np.exp(lp[i] - float(old[i]))
            clipped = np.clip(rho[i], 1.0 - lo, 1.0 + hi)
            cut[i] = rho[i] * A > clipped * A
            li = -(clipped * A if cut[i] else rho[i] * A)
            s = 0.0 if cut[i] else -A * rho[i]
            if ref is not None:
                d = float(ref[i]) - lp[i]
                kl[i] = d if d == np.inf else np.expm1(d) - d
                if beta:
                    li += beta * kl[i]
                    s -= beta * np.expm1(d)
            slope[i] = w[i] * s
            out += w[i] * np.array([li, kl[i], float(cut[i])])
            if slope[i] == 0:
                continue
            top = np.max(z[i])
            e = np.exp(z[i] - top)
            dz[i] = -slope[i] * e / e.sum()
            dz[i, int(action[i])] += slope[i]
    return dict(out=out, logp=lp, dZ=dz, slope=slope, rho=rho, kl=kl, cut=cut, live=live, w=w)


def grad_norm(grads):
    return float(np.sqrt(sum(float(np.sum(np.asarray(g, np.float64) ** 2)) for g in grads)))


# ------------------------------------------------------------- 8-bit values

def _values(man, emin, count):
    return np.array([(c % (1 << man)) * 2.0 ** (emin - man) if c >> man == 0 else
                     (1 + (c % (1 << man)) / (1 << man)) * 2.0 ** ((c >> man) - 1 + emin)
                     for c in range(count)])


E4M3 = _values(3, -6, 127)   # codes 0 .. 126 of OCP e4m3: up to 448
E5M2 = _values(2, -14, 124)  # codes 0 .. 123 of OCP e5m2: up to 57344


def decode(code, scale, grid):
    code = np.asarray(code, np.int64)
    x = grid[np.minimum(code & 127, len(grid) - 1)] * np.where(code > 127, -1.0, 1.0)
    return x * np.repeat(np.asarray(scale, np.float64), BLOCK)[: len(code)]


def scales(x, grid):
    """Unrounded scale of every block of 256 (at least 2^-126)."""
    pad = np.zeros(-(-len(x) // BLOCK) * BLOCK)
    pad[: len(x)] = np.abs(x)
    return np.maximum(pad.reshape(-1, BLOCK).max(1) / grid[-1], TINY)


def encode(x, scale, grid, r, never_zero):
    """(codes, distance of the rounding's decision from its border) given the
    scales: up where frac + (r + 1/2) / 2^16 >= 1."""
    y = np.abs(x) / np.repeat(np.asarray(scale, np.float64), BLOCK)[: len(x)]
    at = np.clip(np.searchsorted(grid, y, side="right") - 1, 0, len(grid) - 2)
    reach = (y - grid[at]) / (grid[at + 1] - grid[at]) + (r + 0.5) / 65536.0
    code = np.minimum(at + (reach >= 1.0), len(grid) - 1)
    if never_zero:
        code = np.where((y > 0) & (code == 0), 1, code)
    return code + np.where(x < 0, 128, 0), np.abs(reach - 1.0)


def random_bits(seed, t, first_block, count):
    """32 bits for each element of a tensor whose predecessors hold
    first_block blocks of 256."""
    base = splitmix_output(seed & M64, t)
    k = np.arange(first_block * BLOCK // 2, first_block * BLOCK // 2 + (count + 1) // 2 + 1,
                  dtype=np.uint64)
    with np.errstate(over="ignore"):
        z = np.uint64(base) + (k + np.uint64(1)) * np.uint64(GOLDEN)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    both = np.stack([z & np.uint64(0xFFFFFFFF), z >> np.uint64(32)], 1).reshape(-1)
    return both[:count].astype(np.int64)


def adamw(w, g, m, v, lr, b1, b2, eps, t, decay, k=1.0):
    """(W, m, v) of step t, unrounded."""
    w, g, m, v = (np.asarray(a, np.float64) for a in (w, g, m, v))
    g = k * g
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    step = (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return (1 - lr * decay) * w - lr * step, m, v
