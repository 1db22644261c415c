"""Float64 CPU oracle for the losses on rows of logits and for gradient clipping.

TEST INFRASTRUCTURE ONLY: imported by tests/; shares no code with the HIP path.

Every function is the definition written out: probabilities by softmax of the given logits, the
loss as a sum over rows or pairs, its derivative by the chain rule through log pi(a) and the
entropy.  `rows_of` lists which sequence a row belongs to and whether it counts.
"""
from __future__ import annotations

import numpy as np


def rows_of(n, n_seqs=1, order="by_seq", bounds=None, mask=None):
    """(sequence of every row, whether it counts)."""
    seq, counts = np.zeros(n, np.int64), np.zeros(n, bool)
    for s in range(n_seqs):
        if order == "packed":
            at = np.arange(bounds[s], bounds[s + 1])
        else:
            steps = n // n_seqs
            every = np.arange(steps)
            at = s * steps + every if order == "by_seq" else every * n_seqs + s
            seq[at] = s
            at = at[:steps if bounds is None else bounds[s]]
        seq[at] = s
        counts[at] = True
    if mask is not None:
        counts &= np.asarray(mask) != 0
    return seq, counts


def softmax_rows(logits, actions, counts=None, lowest=None):
    """log probabilities [n, V], those of the actions and the entropies; rows that do not count are zero.
    A row adds something (`live`) if its action exists and has a probability.  `lowest`: the lowest value of the logits'
    type, which stands for -inf where its probability relative to the largest logit's is below 2^-150."""
    z = np.asarray(logits, np.float64)
    n, V = z.shape
    counts = np.ones(n, bool) if counts is None else counts
    every, l, H, live = np.full((n, V), -np.inf), np.zeros(n), np.zeros(n), np.zeros(n, bool)
    for i in np.flatnonzero(counts):
        if np.isnan(z[i]).any() or np.isposinf(z[i]).any():
            every[i], l[i], H[i], live[i] = np.nan, np.nan, np.nan, 0 <= actions[i] < V
            continue
        if np.isneginf(z[i]).all():
            l[i] = H[i] = np.nan
            continue
        d = z[i] - z[i].max()
        if lowest is not None:
            d[(z[i] == lowest) & (d < -150.0 * np.log(2.0))] = -np.inf
        every[i] = d - np.log(np.exp(d).sum())
        p = np.exp(every[i])
        H[i] = -np.sum(p[p > 0] * every[i][p > 0])
        l[i] = every[i][actions[i]] if 0 <= actions[i] < V else np.nan
        live[i] = 0 <= actions[i] < V and l[i] > -np.inf
    return every, l, H, live


def logits_gradient(every, actions, H, live, d_l, d_H):
    """d / d logits of a sum whose derivatives by l and H of every row are d_l and d_H."""
    g = np.zeros_like(every)
    for i in np.flatnonzero(live):
        if np.isnan(every[i]).any():
            g[i] = np.nan
            continue
        p = np.exp(every[i])
        some = p > 0
        g[i] = -d_l[i] * p
        g[i][some] -= d_H[i] * p[some] * (every[i][some] + H[i])
        g[i][actions[i]] += d_l[i]
    return g


def policy_loss(logits, actions, advantages, rows=None, old=None, ref=None, clip_low=0.2, clip_high=0.2, kl_coeff=0.0,
                entropy_coeff=0.0, reduction="rows", per_seq=False, grad_scale=1.0, n_seqs=1, lowest=None):
    n = len(actions)
    seq, counts = rows if rows is not None else (np.zeros(n, np.int64), np.ones(n, bool))
    every, l, H, live = softmax_rows(logits, actions, counts, lowest)
    length = np.bincount(seq[counts], minlength=n_seqs)
    w = np.zeros(n)
    for i in np.flatnonzero(counts):
        w[i] = {"sum": 1.0, "rows": 1.0 / counts.sum(), "seqs": 1.0 / (length[seq[i]] * (length > 0).sum())}[reduction]
    stats, d_l, d_H = np.zeros(5), np.zeros(n), np.zeros(n)
    for i in np.flatnonzero(live):
        A = float(advantages[seq[i] if per_seq else i])
        r = np.exp(l[i] - float(old[i])) if old is not None else 1.0 + 0.0 * l[i]
        held = np.minimum(np.maximum(r, 1.0 - clip_low), 1.0 + clip_high)
        cut = held * A < r * A
        kl = dkl = 0.0
        if ref is not None:
            d = float(ref[i]) - l[i]
            kl, dkl = np.exp(d) - d - 1.0, 1.0 - np.exp(d)
        stats[1:] += w[i] * np.array([-min(r * A, held * A) if r == r else np.nan, kl, H[i], float(cut)])
        d_l[i] = w[i] * ((0.0 if cut else -A * r) + kl_coeff * dkl)
        d_H[i] = -w[i] * entropy_coeff
    stats[0] = stats[1] + (kl_coeff if ref is not None else 0.0) * stats[2] - entropy_coeff * stats[3]
    d_l, d_H = grad_scale * d_l, grad_scale * d_H
    return dict(stats=stats, grad=logits_gradient(every, actions, H, live, d_l, d_H), logp=l, entropy=H, coeff=-d_l,
                entropy_coeff=-d_H, every=every, live=live, w=w)


def preference_loss(logits, actions, rows, n_seqs, pairs=None, ref=None, beta=0.1, smoothing=0.0, average=False,
                    grad_scale=1.0, lowest=None):
    n = len(actions)
    seq, counts = rows
    every, l, H, live = softmax_rows(logits, actions, counts, lowest)
    length = np.bincount(seq[counts], minlength=n_seqs)
    per = np.where(average & (length > 0), 1.0 / np.maximum(length, 1), 1.0)
    total, ratio = np.zeros(n_seqs), np.zeros(n_seqs)
    for i in np.flatnonzero(live):
        total[seq[i]] += l[i] * per[seq[i]]
        ratio[seq[i]] += (l[i] - (float(ref[i]) if ref is not None else 0.0)) * per[seq[i]]
    if pairs is None:
        pairs = np.arange(n_seqs).reshape(-1, 2)
    margins, loss, right, valid, d = np.full(len(pairs), np.nan), 0.0, 0, 0, np.zeros(n_seqs)
    for k, (a, b) in enumerate(pairs):
        if not (0 <= a < n_seqs and 0 <= b < n_seqs):
            continue
        m = margins[k] = beta * (ratio[a] - ratio[b])
        loss += sum(w * np.logaddexp(0.0, x) for w, x in ((1.0 - smoothing, -m), (smoothing, m)) if w != 0.0)
        right += m > 0
        valid += 1
        g = 1.0 / (1.0 + np.exp(-m)) - 1.0 + smoothing
        d[a] += beta * g
        d[b] -= beta * g
    if valid:
        loss, right, d = loss / valid, right / valid, d / valid
    d_l = np.where(live, grad_scale * d[seq] * per[seq], 0.0)
    return dict(stats=np.array([loss, right], float), grad=logits_gradient(every, actions, H, live, d_l, np.zeros(n)),
                logp=l, margins=margins, seq_logp=total, coeff=-d_l, every=every, live=live)


def clip(grads, max_norm):
    """(norm, clipped gradients) in float64."""
    norm = np.sqrt(sum(float(np.sum(np.asarray(g, np.float64) ** 2)) for g in grads))
    f = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, [np.asarray(g, np.float64) * f for g in grads]
