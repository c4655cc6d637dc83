"""The operators on a caller's tensors by their definitions, in 64 bits on the
host (numpy): the matrix product with its epilogue, log probabilities with
entropy and alternatives, and distillation from a teacher's top classes.
Nothing here is shared with the HIP path."""
import math

import numpy as np


def _erf(x):
    return np.vectorize(math.erf, otypes=[np.float64])(x)


def activation(v, act):
    """0 none, 1 relu, 2 gelu (v * normal distribution function), 3 silu."""
    if act == 1:
        return np.where(v > 0, v, 0.0)
    if act == 2:
        return 0.5 * v * (1.0 + _erf(v / math.sqrt(2.0)))
    if act == 3:
        with np.errstate(over="ignore"):
            return v / (1.0 + np.exp(-v))
    return v


def linear(x, w, bias=None, res=None, act=0, res_first=0):
    """(y, size): size is the sum of the magnitudes that enter each output."""
    x, w = x.astype(np.float64), w.astype(np.float64)
    v, size = x @ w.T, np.abs(x) @ np.abs(w).T
    for t in ([bias] if bias is not None else []) + ([res] if res is not None else []):
        size = size + np.abs(t.astype(np.float64))
    if bias is not None:
        v = v + bias.astype(np.float64)
    if res is not None and res_first:
        v = v + res.astype(np.float64)
    v = activation(v, act)
    if res is not None and not res_first:
        v = v + res.astype(np.float64)
    return v, size


def log_softmax(z, temperature=1.0):
    """ln p of each row; a class at -inf has -inf, as has every class of a row
    of nothing else; NaN or +inf in a row makes its other classes NaN."""
    z = z.astype(np.float64) / temperature
    out = np.empty_like(z)
    for r in range(z.shape[0]):
        row = z[r]
        if np.isnan(row).any() or np.isposinf(row).any():
            out[r] = np.where(np.isneginf(row), -np.inf, np.nan)
        elif np.isneginf(row).all():
            out[r] = -np.inf
        else:
            m = row.max()
            out[r] = row - m - math.log(np.exp(row - m).sum())
    return out


def logprob(z, classes, top):
    """dict(logp [R][T], entropy [R], top_ids [R][top], top_logp [R][top])."""
    rows, n = z.shape
    lp = log_softmax(z)
    logp = np.full(classes.shape, -np.inf)
    ids = np.full((rows, top), -1, np.int32)
    best = np.full((rows, top), -np.inf)
    entropy = np.empty(rows)
    for r in range(rows):
        for i, c in enumerate(classes[r]):
            if 0 <= c < n:
                logp[r, i] = lp[r, c]
        p = np.exp(lp[r])
        entropy[r] = np.nan if np.isnan(p).any() else -sum(p[p > 0] * lp[r][p > 0])
        alive = [c for c in np.argsort(-np.where(np.isnan(z[r]), -np.inf, z[r]), kind="stable")[:top]
                 if z[r, c] > -np.inf]
        ids[r, :len(alive)] = alive
        best[r, :len(alive)] = lp[r, alive]
    return dict(logp=logp, entropy=entropy, top_ids=ids, top_logp=best)


def teacher(ids, u, classes, temperature):
    """q of a row's entries (0 for one that is left out) and whether the row
    has any mass."""
    u = np.where((ids >= 0) & (ids < classes), u.astype(np.float64), -np.inf)
    if np.isneginf(u).all():
        return np.zeros(len(u)), False
    if np.isnan(u).any() or np.isposinf(u).any():
        return np.where(np.isneginf(u), 0.0, np.nan), True
    e = np.exp((u - u.max()) / temperature)
    return e / e.sum(), True


def distill(z, ids, u, temperature, weight=None):
    """dict(loss [R], stats [R][2], grad [R][C], p [R][C], q [R][K])."""
    rows, n = z.shape
    lp = log_softmax(z, temperature)
    out = dict(loss=np.zeros(rows), stats=np.empty((rows, 2)), grad=np.zeros((rows, n)), p=np.exp(lp),
               q=np.zeros(ids.shape))
    for r in range(rows):
        row = z[r].astype(np.float64)
        if np.isnan(row).any():
            out["stats"][r] = np.nan
        elif np.isposinf(row).any():
            out["stats"][r] = np.inf, np.nan
        elif np.isneginf(row).all():
            out["stats"][r] = -np.inf, 0.0
        else:
            out["stats"][r] = row.max(), math.log(np.exp((row - row.max()) / temperature).sum())
        q, mass = teacher(ids[r], u[r], n, temperature)
        if not mass:
            continue
        out["q"][r] = q
        g = out["p"][r].copy()
        for j, c in enumerate(ids[r]):
            if 0 <= c < n and not q[j] == 0.0:
                out["loss"][r] += q[j] * (math.log(q[j]) - lp[r, c])
                g[c] -= q[j]
        out["grad"][r] = g * ((1.0 if weight is None else float(weight[r])) / temperature)
    return out
