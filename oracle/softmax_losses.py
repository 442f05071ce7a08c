"""The softmax layer beyond cross-entropy, in float64 from the definitions (numpy, CPU).

With u = z W^T + b the logits of M frames, p = softmax(u) and s the loss scale.  A label of NO_LABEL, and an entry of a
teacher's list of class NO_LABEL or value -inf, counts for nothing.
"""
from __future__ import annotations

import numpy as np

NO_LABEL = -1


def _log_softmax(u):
    top = u.max(axis=1, keepdims=True)
    return u - top - np.log(np.exp(u - top).sum(axis=1, keepdims=True))


def _rows(W, b, z, counts):
    """Logits and their log-softmax, of the frames that count only (whatever z holds in the others)."""
    z = np.where(counts[:, None], np.asarray(z, np.float64), 0.0)
    u = z @ np.asarray(W, np.float64).T + np.asarray(b, np.float64)
    return z, u, _log_softmax(u)


def logprob(W, b, z, labels):
    """log p[label] of every frame, 0 without a label."""
    labels = np.asarray(labels).reshape(-1)
    live = labels != NO_LABEL
    _, _, lp = _rows(W, b, z, live)
    return np.where(live, lp[np.arange(len(labels)), np.where(live, labels, 0)], 0.0)


def topk(u, K):
    """Values and classes of the K largest of every row: by falling value, equal ones by rising class, NaN last."""
    values, classes = [], []
    for row in u:
        order = sorted(range(len(row)), key=lambda v: (np.isnan(row[v]), -row[v] if not np.isnan(row[v]) else 0.0, v))[:K]
        classes.append(order)
        values.append(row[order])
    return np.array(values), np.array(classes, dtype=np.int32)


def teacher_distribution(values, classes, V, temperature):
    """q [M][V] and the frames that have one."""
    M, K = classes.shape
    used = (classes != NO_LABEL) & (values != -np.inf)
    q = np.zeros((M, V))
    for m in range(M):
        k = np.flatnonzero(used[m])
        if len(k):
            e = np.exp(values[m, k].astype(np.float64) / temperature - (values[m, k].astype(np.float64) / temperature).max())
            np.add.at(q[m], classes[m, k], e / e.sum())
    return q, used.any(axis=1)


def entropy_terms(values, classes, temperature):
    """sum_k q_k log q_k of every frame, over its entries (a class that stands there twice is two of them)."""
    out = np.zeros(len(values))
    for m in range(len(values)):
        v = values[m][(classes[m] != NO_LABEL) & (values[m] != -np.inf)].astype(np.float64) / temperature
        if len(v):
            q = np.exp(v - v.max())
            q /= q.sum()
            out[m] = np.sum(np.where(q > 0, q * np.log(np.where(q > 0, q, 1.0)), 0.0))
    return out


def _gradients(W, z, du):
    return du @ np.asarray(W, np.float64), du.T @ z, du.sum(axis=0)


def distill(W, b, z, labels, values, classes, s, temperature, hard, soft):
    """(loss, dz [M][Z], dW [V][Z], db [V]); labels None: none."""
    M, V = len(z), len(b)
    values, classes = np.asarray(values).reshape(M, -1), np.asarray(classes).reshape(M, -1)
    labels = np.full(M, NO_LABEL) if labels is None or hard == 0 else np.asarray(labels).reshape(-1)
    q, some = teacher_distribution(values, classes, V, temperature)
    live = labels != NO_LABEL
    z, u, lp = _rows(W, b, z, live | some)
    lpt = _log_softmax(u / temperature)
    hot = np.zeros((M, V))
    hot[np.flatnonzero(live), labels[live]] = 1.0
    loss = hard * -(hot * lp).sum() + soft * temperature ** 2 * (entropy_terms(values, classes, temperature) - (q * lpt).sum(axis=1)).sum()
    du = hard * (np.exp(lp) * live[:, None] - hot) + soft * temperature * (np.exp(lpt) * some[:, None] - q)
    return (s * loss, *_gradients(W, z, s * du))


def policy(W, b, z, labels, advantage, old, ref, s, clip_low, clip_high, kl):
    """(loss, logp [M], dz, dW, db); old None: ratio 1, ref None: no KL term."""
    labels = np.asarray(labels).reshape(-1)
    M, V = len(z), len(b)
    live = labels != NO_LABEL
    z, _, lp_all = _rows(W, b, z, live)
    hot = np.zeros((M, V))
    hot[np.flatnonzero(live), labels[live]] = 1.0
    lp = (hot * lp_all).sum(axis=1)
    pick = lambda a: np.where(live, np.asarray(a, np.float64).reshape(-1), 0.0)  # noqa: E731
    A = pick(advantage)
    r = np.ones(M) if old is None else np.exp(lp - pick(old))
    inner, outer = r * A, np.clip(r, 1 - clip_low, 1 + clip_high) * A
    loss = -np.minimum(inner, outer)
    g = np.where(inner <= outer, -inner, 0.0)
    if ref is not None:
        d = pick(ref) - lp
        loss = loss + kl * (np.exp(d) - d - 1)
        g = g + kl * (1 - np.exp(d))
    du = s * np.where(live, g, 0.0)[:, None] * (hot - np.exp(lp_all))
    return (s * loss[live].sum(), np.where(live, lp, 0.0), *_gradients(W, z, du))
