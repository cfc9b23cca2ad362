"""Plain definitions, in 64 bits, of the operators at a model's two ends: matrices in
blocks of 4-bit floating point, verification of drafted tokens, embedding and its
gradient (numpy).  Shares nothing with the HIP path."""
from __future__ import annotations

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
U = 2.0 ** -24                      # unit roundoff of fp32


# ---- blocks of 4-bit floating point ---------------------------------------------------
def mx4_values(q, scales):
    """[rows, K] that codes [rows, K/2] and scales [rows, K/32] stand for."""
    q = np.asarray(q)
    code = np.empty((q.shape[0], 2 * q.shape[1]), dtype=np.int64)
    code[:, 0::2], code[:, 1::2] = q & 15, q >> 4
    s = np.asarray(scales).astype(np.int64)
    unit = np.where(s == 255, math.nan, np.ldexp(1.0, s - 127))
    sign = np.where(code & 8, -1.0, 1.0)
    return sign * GRID[code & 7] * np.repeat(unit, 32, axis=1)


def mx4_quantise(x):
    """(codes [rows, K/2], scales [rows, K/32]) of x, by comparison with the borders
    between neighbouring values."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(x.shape[0], -1, 32)
    bad = ~np.isfinite(b).all(axis=2)
    most = np.abs(np.where(np.isfinite(b), b, 0.0)).max(axis=2) if b.shape[1] else np.zeros(b.shape[:2])
    _, e = np.frexp(most)               # most = f 2^e with f in [1/2, 1)
    e = np.where(most > 0, np.maximum(e - 3, -127), -127)
    a = np.abs(b) / np.ldexp(1.0, e)[:, :, None]
    code = np.zeros(b.shape, dtype=np.int64)
    for j in range(1, 8):
        border = (GRID[j - 1] + GRID[j]) / 2
        up = a >= border if j % 2 == 0 else a > border      # the even one of two as near
        code = np.where(up, j, code)
    code = np.where(np.signbit(b), code | 8, code)
    code = np.where(bad[:, :, None], 0, code).reshape(x.shape)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), scales


# ---- drafted tokens -------------------------------------------------------------------
def softmax(x, scale):
    """(p, log p, largest) of a row, None where it has no distribution."""
    x = np.asarray(x, dtype=np.float64)
    m = np.max(x)
    if np.isnan(x).any() or np.isinf(m):
        return None
    d = (x - m) * scale
    lp = d - math.log(np.exp(d).sum())
    return np.exp(lp), lp, m


def first_largest(x):
    return int(np.flatnonzero(x == x.max())[0])


class Verdict:
    """What a sequence may give: ``tokens`` for certain, then either nothing more is
    certain (a decision within the fp32 error of its border: ``open``), or the last
    token is one of ``last``."""

    def __init__(self):
        self.tokens, self.logprob, self.last, self.open = [], [], None, False


def eps(lp):
    """Relative error of a probability computed in fp32: that of its exponent in base 2
    (a rounding of x c and one of the product with the largest logit, of at most 32 and
    the logit's own size each), the exponential's and the reciprocal's, and half of the
    sums' 2e-5."""
    return (np.abs(lp) * 1.45 + 80.0) * 2 * U + 1e-5


def verify(rows, drafts, ids, uniforms, noise, scale, draft_scale):
    """One sequence: target rows [k + 1, V], draft rows [k, V] or None, ids [k]; noise None:
    greedy."""
    v, i = Verdict(), 0
    k = len(ids)
    while True:
        d = int(ids[i]) if i < k else -1
        t = softmax(rows[i], scale)
        if t is None:
            v.last = {-1: 0.0}
            return v
        p, lp, _ = t
        if noise is None:
            best = first_largest(np.asarray(rows[i], dtype=np.float64))
            if d < 0 or d != best:
                v.last = {best: float(lp[best])}
                return v
            v.tokens.append(d)
            v.logprob.append(float(lp[d]))
            i += 1
            continue
        q = None
        if d >= 0:
            q = np.zeros_like(p)
            lq = np.zeros_like(p)
            if drafts is None:
                if d < len(q):
                    q[d] = 1.0
            else:
                s = softmax(drafts[i], draft_scale)
                q = None if s is None else s[0]
                lq = None if s is None else s[1]
            ok = False
            if d < len(p) and (drafts is None or q is not None):
                a, b = float(uniforms[i]) * q[d], p[d]
                if a != b and abs(a - b) <= 4e-5 * max(a, b):
                    v.open = True
                    return v
                ok = a < b
            if ok:
                v.tokens.append(d)
                v.logprob.append(float(lp[d]))
                i += 1
                continue
        e = np.asarray(noise, dtype=np.float64)
        w, err = p, eps(np.where(p > 0, lp, 0.0)) * p
        if q is not None:
            w = np.maximum(p - q, 0.0)
            if drafts is not None:
                err = err + eps(np.where(q > 0, lq, 0.0)) * q
            else:
                err = np.where(q > 0, 0.0, err)         # the token itself is out
            if not (w > 0).any():
                w = p
            elif (w <= err).all():
                v.open = True
                return v
        least = ((w - err) / e).max()
        v.last = {int(c): float(lp[c]) for c in np.flatnonzero(((w + err) / e >= least) & (w + err > 0))}
        return v


# ---- embedding --------------------------------------------------------------------------
def embedding_grad(tokens, drows, first, rows, scale):
    """(dtable, sum of magnitudes, number of terms) of the shard's rows."""
    d = np.asarray(drows, dtype=np.float64)
    g = np.zeros((rows, d.shape[1]))
    size = np.zeros_like(g)
    count = np.zeros(rows, dtype=np.int64)
    for t, id_ in enumerate(np.asarray(tokens)):
        v = int(id_) - first
        if id_ >= 0 and 0 <= v < rows:
            g[v] += d[t]
            size[v] += np.abs(d[t])
            count[v] += 1
    return g * scale, size * abs(scale), count
