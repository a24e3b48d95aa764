"""The layer of experts in 64 bits, from the definitions (numpy; test infrastructure only)."""
import numpy as np


def route(logits, k, renorm):
    """ids, weights, offsets, tokens, slots of polydl_route."""
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    rank = np.where(np.isnan(x), np.inf, x)
    # NaN before +infinity, then the value, then the index
    ids = np.full((T, k), -1, np.int64)
    w = np.zeros((T, k))
    for t in range(T):
        order = sorted(range(E), key=lambda e: (not np.isnan(x[t, e]), -rank[t, e], e))
        order = [e for e in order if x[t, e] != -np.inf][:k]
        ids[t, :len(order)] = order
        if not order:
            continue
        with np.errstate(invalid="ignore"):
            z = np.exp(x[t] - x[t, order[0]])
        w[t, :len(order)] = z[order] / (z[order].sum() if renorm else z.sum())
    return (ids, w) + plan(ids, E)


def plan(ids, E):
    """offsets, tokens, slots of given choices."""
    T, k = ids.shape
    flat = np.where(ids.reshape(-1) < 0, E, ids.reshape(-1))
    order = np.argsort(flat, kind="stable")
    offsets = np.zeros(E + 1, np.int64)
    offsets[1:] = np.cumsum(np.bincount(flat, minlength=E + 1)[:E])
    slots = np.empty(T * k, np.int64)
    slots[order] = np.arange(T * k)
    tokens = np.where(np.arange(T * k) < offsets[E], order // k, -1)
    return offsets, tokens, np.where(ids < 0, -1, slots.reshape(T, k))


def route_bwd(logits, ids, weights, dweights, renorm):
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    g, p = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        for j, e in enumerate(ids[t]):
            if e >= 0:
                g[t, e] += dweights[t, j]
                if renorm:
                    p[t, e] = weights[t, j]
        if not renorm and np.any(x[t] != -np.inf):
            z = np.exp(x[t] - x[t].max())
            p[t] = z / z.sum()
    return p * (g - (p * g).sum(1, keepdims=True))


def act(v, name):
    return v if name is None else np.maximum(v, 0) if name == "relu" else np.clip(v, 0, 6)


def gathered(x, rows):
    """x[rows], zeros for rows that are none."""
    if rows is None:
        return x
    there = (rows >= 0) & (rows < x.shape[0])
    return np.where(there[:, None], x[np.where(there, rows, 0)], 0.0)


def w4_weights(q, scales, zeros, N, K, group):
    """[E][N][K] in 64 bits from the packed layout, place by place."""
    n, k = np.arange(N)[:, None], np.arange(K)[None, :]
    nibble = (k % 8) // 2 + 4 * (k % 2)
    byte = q[:, n // 16, k // 128, n % 16 + 16 * (k % 32 // 8), 4 * (k % 128 // 32) + nibble // 2].astype(np.int64)
    code = np.where(nibble % 2 == 1, byte >> 4, byte & 15)
    z = 8 if zeros is None else zeros[:, n // 16, k // group, n % 16].astype(np.int64)
    return scales[:, n // 16, k // group, n % 16].astype(np.float64) * (code - z)
