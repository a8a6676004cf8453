"""Plain NumPy forms, in 64 bits and from the definitions, of rotation by position, attention with its gradients, and a cache of pages.
Test infrastructure only."""
import numpy as np


def rotate(x, positions, frequencies, neighbours, inverse=False):
    """x (tokens, heads, head)."""
    half = len(frequencies)
    angle = positions.astype(np.float64)[:, None, None] * frequencies.astype(np.float64)
    c, s = np.cos(angle), np.sin(angle) * (-1 if inverse else 1)
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if neighbours else (x[..., :half], x[..., half:2 * half])
    y = x.copy()
    if neighbours:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * c - b * s, a * s + b * c
    else:
        y[..., :half], y[..., half:2 * half] = a * c - b * s, a * s + b * c
    return y


def causal(queries, keys):
    """(queries, keys): which keys a query sees; the last query sees the last key."""
    return np.arange(keys)[None, :] <= np.arange(queries)[:, None] + (keys - queries)


def attention(q, k, v, seen, scale):
    """One head: (o, lse, p); rows that see nothing are zeros, their lse minus infinity; rows that see scores, but none above minus infinity, have NaN
    for weights.  What is not seen takes no part, whatever it is."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.where(seen, (q @ k.T) * scale, -np.inf)
    top = s.max(axis=1, initial=-np.inf, keepdims=True)
    e = np.where(seen, np.exp(s - np.where(np.isinf(top), 0, top)), 0.0)
    total = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        lse = (np.log(total) + np.where(np.isinf(top), 0, top))[:, 0]
        p = np.where(seen, e / total, 0.0)
    return weighted(p, v, seen), lse, p


def weighted(w, x, seen):
    """w x, where what is not seen takes no part, infinities and NaN included."""
    if np.isfinite(x).all():
        return w @ x
    out = np.zeros((w.shape[0], x.shape[1]))
    with np.errstate(invalid="ignore"):
        for i in range(w.shape[0]):
            out[i] = w[i, seen[i]] @ x[seen[i]]
    return out


def gradients(do, q, k, v, o, lse, seen, scale):
    """One head: (dq, dk, dv, p, ds) from the forward pass's outputs."""
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.where(seen, np.exp((q @ k.T) * scale - lse[:, None]), 0.0)
        ds = np.where(seen, p * (do @ v.T - (do * o).sum(axis=1, keepdims=True)) * scale, 0.0)
    return weighted(ds, k, seen), weighted(ds.T, q, seen.T), weighted(p.T, do, seen.T), p, ds


def spans(ends):
    return list(zip(ends, ends[1:]))


def place(table, page_size, j):
    """(page, place in it) of place j of a sequence; (-1, 0) where its table has none."""
    if j < 0 or j // page_size >= len(table):
        return -1, 0
    return int(table[j // page_size]), j % page_size


def tree_seen(words, length, new, keys):
    """(new, keys): the cached tokens, and the new ones whose bits are set in each token's words."""
    seen = np.zeros((new, keys), dtype=bool)
    seen[:, :length] = True
    for i in range(new):
        for j in range(min(new, keys - length, 64 * words.shape[1])):
            seen[i, length + j] = int(words[i, j // 64]) >> (j % 64) & 1
    return seen
