"""Float64 CPU oracle for the most likely actions, the loss over them, and orthogonalised updates.

TEST INFRASTRUCTURE ONLY: imported by tests/; shares no code with the HIP path.  Every function is the definition written out.
"""
from __future__ import annotations

import numpy as np


def log_softmax(z, T=1.0, lowest=None):
    """Log probabilities of a row; NaN where a logit is NaN or +inf, or nothing is allowed.  `lowest`: the lowest value of the
    logits' type, which stands for -inf where its probability is below 2^-150 of the largest."""
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or np.isposinf(z).any() or np.isneginf(z).all():
        return np.full(len(z), np.nan)
    d = (z - z.max()) / T
    if lowest is not None:
        d[(z == lowest) & (d < -150.0 * np.log(2.0))] = -np.inf
    return d - np.log(np.exp(d).sum())


def top(z, k, T=1.0, lowest=None):
    """(indexes, their log probabilities, entropies) of rows without NaN: largest logits first, equal ones by index."""
    z = np.asarray(z, np.float64)
    ids = np.argsort(-z, axis=1, kind="stable")[:, :k]
    every = np.array([log_softmax(r, T, lowest) for r in z]).reshape(z.shape)
    with np.errstate(invalid="ignore"):
        p = np.exp(every)
        H = -np.where(p == 0.0, 0.0, p * np.where(p == 0.0, 0.0, every)).sum(1)
    return ids, np.take_along_axis(every, ids, 1), every, H


def distill(z, ids, lq, rows, tail=True, T=1.0, reduction="rows", n_seqs=1, grad_scale=1.0, lowest=None):
    z, lq = np.asarray(z, np.float64), np.asarray(lq, np.float64)
    n, V = z.shape
    seq, counts = rows
    length = np.bincount(seq[counts], minlength=n_seqs)
    grad, values, coeff, stats = np.zeros((n, V)), np.zeros(n), np.zeros(ids.shape), np.zeros(3)
    w = np.zeros(n)
    size = np.zeros(n)                                    # how far an error of the unlisted sum reaches into the value
    factor = np.zeros((n, 2))                             # F, r / p_rest
    for i in np.flatnonzero(counts):
        w[i] = {"sum": 1.0, "rows": 1.0 / counts.sum(), "seqs": 1.0 / (length[seq[i]] * (length > 0).sum())}[reduction]
        if np.isneginf(z[i]).all():
            continue
        every = log_softmax(z[i], T, lowest)
        p = np.exp(every)
        use = [j for j in range(ids.shape[1]) if 0 <= ids[i, j] < V and not np.isneginf(lq[i, j]) and not np.isneginf(every[ids[i, j]])]
        listed = np.zeros(V, bool)
        q = np.zeros(V)
        for j in use:
            listed[ids[i, j]] = True
            q[ids[i, j]] += np.exp(lq[i, j])
            values[i] += np.exp(lq[i, j]) * (lq[i, j] - every[ids[i, j]])
            coeff[i, j] = grad_scale * w[i] / T * np.exp(lq[i, j])
        mass, rest = q.sum(), p[~listed].sum()
        others = np.where(listed, -np.inf, every)         # in logarithms: exp(-800) is 0, what it is a part of need not be
        log_rest = others.max() + np.log(np.exp(others - others.max()).sum()) if not np.isneginf(others).all() else -np.inf
        r = max(0.0, 1.0 - mass) if tail and log_rest > -np.inf else 0.0
        if r > 0.0:
            values[i] += r * (np.log(r) - log_rest)
        F = mass + r
        grad[i] = grad_scale * w[i] / T * np.where(listed, F * p - q, F * p - (r * np.exp(others - log_rest) if r > 0.0 else 0.0))
        stats += w[i] * np.array([values[i], mass, p[listed].sum()])
        size[i], factor[i] = max(rest * mass, r, abs(F * rest - r)), (F, r * np.exp(min(-log_rest, 700.0)) if r > 0.0 else 0.0)
    return dict(stats=stats, grad=grad, values=values, coeff=coeff, w=w, size=size, factor=factor, counts=counts)


def orthogonal(g, momentum=None, beta=0.95, nesterov=True, iteration=((3.4445, -4.7750, 2.0315),) * 5, eps=1e-7):
    """(factor, new momentum, iterates)"""
    g = np.asarray(g, np.float64)
    m = u = None
    if momentum is not None:
        m = beta * np.asarray(momentum, np.float64) + g
        u = g + beta * m if nesterov else m
    else:
        u = g
    norm = np.sqrt((u ** 2).sum()) + eps
    x = u / norm if norm > 0.0 else u
    xs = [x]
    for a, b, c in iteration:                             # on the side that the kernels do not take, too
        y = x.T @ x
        x = a * x + x @ (b * y + c * y @ y)
        xs.append(x)
    return x, m, xs
