"""The losses over a vocabulary (include/zl_loss.h) in fp64 NumPy, row by row from
their definitions: labels, a teacher's top logits with or without the rest of its
distribution, and the top logits of a row."""
import numpy as np


def lse(v):
    """log sum exp of a vector; -inf of nothing."""
    v = np.asarray(v, np.float64)
    m = v.max() if v.size else -np.inf
    return m + np.log(np.exp(v - m).sum()) if np.isfinite(m) else m


def top_logits(x, k, tau=1.0):
    """(ids, values, rest): the k largest of every row, ties to the lower column, NaN
    first; rest: log sum exp(x / tau) of the others."""
    x = np.asarray(x, np.float64)
    T, V = x.shape
    ids, values, rest = np.zeros((T, k), np.int32), np.zeros((T, k)), np.zeros(T)
    for t in range(T):
        order = np.lexsort((np.arange(V), np.where(np.isnan(x[t]), -np.inf, -x[t]), ~np.isnan(x[t])))
        ids[t], values[t] = order[:k], x[t][order[:k]]
        rest[t] = lse(x[t][order[k:]] / tau)
    return ids, values, rest


def weights(labels, ids, alpha):
    """(a, b) of a CE + b tau^2 KL."""
    if labels is None:
        return 0.0, 1.0
    return (1.0, 0.0) if ids is None else (alpha, 1.0 - alpha)


def teacher_row(V, ids, values, rest, tau):
    """The teacher's outcomes of one row: (columns, probabilities, the rest's), or None."""
    seen, at, t = set(), [], []
    for i, v in zip(ids, values):
        if 0 <= i < V and int(i) not in seen:
            seen.add(int(i))
            at.append(int(i))
            t.append(float(v) / tau)
    u = -np.inf if rest is None else float(rest)
    if not at or max(t + [u]) == -np.inf:
        return None
    L = lse(np.array(t + [u]))
    return np.array(at), np.exp(np.array(t) - L), np.exp(u - L)


def loss(z, labels=None, ids=None, values=None, rest=None, alpha=0.5, tau=1.0, grad=True):
    """(loss [T], stats [T, 4], dloss/dz [T, V] or None) of logits z [T, V]."""
    z = np.asarray(z, np.float64)
    T, V = z.shape
    a, b = weights(labels, ids, alpha)
    out, stats, dz = np.zeros(T), np.zeros((T, 4)), np.zeros((T, V)) if grad else None
    for t in range(T):
        y = -1 if labels is None else int(labels[t])
        if 0 <= y < V:
            l = lse(z[t])
            stats[t, 0], stats[t, 3] = l, z[t, y]
            out[t] += a * (l - z[t, y])
            if grad:
                g = np.exp(z[t] - l)
                g[y] = np.expm1(z[t, y] - l)
                dz[t] += a * g
        row = None if ids is None else teacher_row(V, ids[t], values[t], None if rest is None else rest[t], tau)
        if row is None:
            continue
        at, p, r = row
        u = z[t] / tau
        l = lse(u)
        named = np.zeros(V, bool)
        named[at] = True
        target = np.zeros(V)
        target[at] = p
        q = np.exp(u - l)
        on = p > 0
        kl = (p[on] * (np.log(p[on]) - (u[at][on] - l))).sum()
        stats[t, 1] = l
        if rest is not None:
            o = lse(u[~named])
            stats[t, 2] = o
            if r > 0:
                kl += r * (np.log(r) - (o - l))
            if o > -np.inf:
                target[~named] = r * np.exp(u[~named] - o)
        out[t] += b * tau * tau * kl
        if grad:
            dz[t] += b * tau * (q - target)
    return out, stats, dz


def head(x, w, labels=None, ids=None, values=None, rest=None, alpha=0.5, tau=1.0, dloss=None):
    """(loss, stats [T, 4 + k], dx, dw) of logits x w^T, of sum(dloss * loss)."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    z = x @ w.T
    out, stats, dz = loss(z, labels, ids, values, rest, alpha, tau)
    if ids is not None:
        V = z.shape[1]
        more = np.zeros(ids.shape)
        for t in range(z.shape[0]):
            seen = set()
            for j, i in enumerate(ids[t]):
                if 0 <= i < V and int(i) not in seen:
                    seen.add(int(i))
                    more[t, j] = z[t, i]
        stats = np.concatenate([stats, more], 1)
    if dloss is not None:
        dz = dz * np.asarray(dloss, np.float64)[:, None]
    return out, stats, dz @ w, dz.T @ x
