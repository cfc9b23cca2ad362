"""Plain 64-bit definitions of the output head's operators (numpy, one row at a
time), and the error bounds of computing them in fp32.  Shares nothing with the
HIP path."""
from __future__ import annotations

import math

import numpy as np

U = 2.0 ** -24                      # unit roundoff of fp32
INF = math.inf


def row_sums(x, scale):
    """(m, log s, p, logp) of one row: the largest logit, log sum exp(scale (x - m)), the
    probabilities and their logs; empty rows have m = -inf, log s = 0, p = 0."""
    x = np.asarray(x, dtype=np.float64)
    m = np.max(x) if not np.isnan(x).any() else math.nan
    if m == -INF:
        return m, 0.0, np.zeros_like(x), np.full_like(x, -INF)
    with np.errstate(invalid="ignore", over="ignore"):
        d = (x - m) * scale
        e = np.exp(d)
        log_s = math.log(e.sum()) if not np.isnan(e).any() else math.nan
        return m, log_s, np.exp(d - log_s), d - log_s


def top_order(x):
    """Ids by descending logit (NaN first), equal ones ascending."""
    x = np.asarray(x, dtype=np.float64) + 0.0
    key = np.where(np.isnan(x), np.inf, x)
    nan = np.isnan(x)
    return np.lexsort((np.arange(x.size), -key, ~nan))


def token_logprobs(x, target, scale, top=0):
    """(logprob, entropy, (m, log s), top ids, top logprobs) of one row."""
    m, log_s, p, logp = row_sums(x, scale)
    empty = m == -INF
    entropy = 0.0 if empty else -float(np.sum(np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0)))
    if np.isnan(log_s):
        entropy = math.nan
    lp = 0.0 if target < 0 else math.nan if target >= len(x) else float(logp[target])
    ids = top_order(x)[:top]
    return lp, entropy, (m, log_s), ids, logp[ids]


def token_logprobs_grad(x, target, scale, g_logprob, g_entropy, g_lse):
    m, log_s, p, logp = row_sums(x, scale)
    if m == -INF:
        return np.zeros_like(p)
    g = g_logprob if target >= 0 else 0.0
    H = -np.sum(np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0))
    d = p * (g_lse - g) - np.where(p > 0, p * (np.where(p > 0, logp, 0.0) + H), 0.0) * g_entropy
    if target >= 0:
        d[target] += g
    return d * scale


def teacher(ids, values, scale, rest):
    """(q, q_rest) of one row's list."""
    values = np.asarray(values, dtype=np.float64)
    there = np.asarray(ids) >= 0
    q = np.zeros(len(ids))
    if not there.any():
        return q, 0.0
    if rest:
        q[there] = np.exp(values[there])
        return q, max(0.0, 1.0 - float(q.sum()))
    v = values[there] * scale
    if np.max(v) == -INF:
        return q, 0.0
    e = np.exp(v - np.max(v))
    q[there] = e / e.sum()
    return q, 0.0


def distill(x, ids, values, scale, rest):
    """(loss, gradient of the loss) of one row."""
    x = np.asarray(x, dtype=np.float64)
    ids = np.asarray(ids)
    if (ids >= len(x)).any():
        return math.nan, np.full(len(x), math.nan)
    q, q_rest = teacher(ids, values, scale, rest)
    there = ids >= 0
    m, log_s, p, logp = row_sums(x, scale)
    if not there.any():
        return 0.0, np.zeros(len(x))
    loss = 0.0
    for j in range(len(ids)):
        if q[j] > 0:
            loss += q[j] * (math.log(q[j]) - logp[ids[j]])
    outside = np.ones(len(x), dtype=bool)
    outside[ids[there]] = False
    xr = np.where(outside, x, -INF)
    mr = np.max(xr)
    if mr == -INF:
        q_rest = 0.0
    grad = p * (q.sum() + q_rest)
    if mr != -INF:
        er = np.where(outside, np.exp((np.where(outside, x, mr) - mr) * scale), 0.0)
        if q_rest > 0:
            loss += q_rest * (math.log(q_rest) - ((mr - m) * scale + math.log(er.sum()) - log_s))
            grad = grad - q_rest * er / er.sum()
    np.subtract.at(grad, ids[there], q[there])
    return loss, (np.zeros(len(x)) if m == -INF else grad * scale)


def log_bound(x, scale):
    """Bound of the absolute error of log s and of a log probability in fp32.

    An exponent scale (x - m) log2(e) of size R has three roundings (the difference,
    the scaled constant, the product), so exp is off by a relative 3 R u and its own 2
    ulp; no partial sum is a chain of more than 512 + 16 additions, each off by u of a
    sum of positive terms; log and the final difference add 4 u (1 + the value).  Terms
    beyond R = 104 are below the smallest number."""
    x = np.asarray(x, dtype=np.float64)
    fin = x[np.isfinite(x)]
    n = len(x)
    spread = min(104.0, float((fin.max() - fin.min()) * scale)) if fin.size else 0.0
    return U * (3 * 1.5 * spread + 4 + min(n, 512) + 16 + 4 * (1 + math.log(n)))


def value_bound(x, scale, value):
    """Bound of a log probability: the sums', and the roundings of the value's own size."""
    return log_bound(x, scale) + (6 * U * abs(value) if math.isfinite(value) else 0.0)


def half_ulp(v, dtype):
    """Half a unit in the last place of v in the output type."""
    p, emin = {"bf16": (8, -126), "f16": (11, -14), "f32": (24, -126)}[dtype]
    v = np.abs(np.asarray(v, dtype=np.float64))
    e = np.floor(np.log2(np.where(v > 0, v, 1.0)))
    e = np.where(v > 0, e, emin)
    return np.exp2(np.maximum(e, emin) - p)


# fp32 results below the smallest normal number may be flushed (2^-126), and so may a
# probability that small before it is multiplied with gradients of up to 2^10.
TINY = 2.0 ** -116
