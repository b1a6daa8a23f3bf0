"""fp64 oracle of the latent-cache operators and of filtered sampling, from their definitions (numpy; no code shared with the
kernels)."""
import numpy as np


def rotate(x, pos, freqs, interleaved):
    """Rows x [..., rot] turned by pos [...] (broadcast) times freqs [rot / 2]."""
    half = len(freqs)
    i = np.arange(half)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    z = (x[..., ia] + 1j * x[..., ib]) * np.exp(1j * (np.asarray(pos, dtype=np.float64)[..., None] * freqs))
    y = np.array(x, dtype=np.float64)
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def latent_rows(x, weight, eps, pos, freqs, rank, interleaved):
    """One row a token: x [..., rank + rot], positions pos [...]."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    if weight is not None:
        c = x[..., :rank]
        y[..., :rank] = c / np.sqrt((c * c).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    if len(freqs):
        y[..., rank:] = rotate(x[..., rank:], pos, freqs, interleaved)
    return y


def latent_attention(q, prefix, tree, see, scale, rank):
    """q [n][W] of one head, prefix [L][W], tree [n][W], see [n][n]: (output [n][rank], sum of weights times |values|, largest
    sum of |products| of a score) -- the last two for error bounds."""
    keys = np.concatenate([np.asarray(prefix, np.float64), np.asarray(tree, np.float64)])
    q = np.asarray(q, np.float64)
    L = len(prefix)
    z = q @ keys.T * scale
    vis = np.concatenate([np.ones((len(q), L), bool), np.asarray(see, bool)], 1)
    z = np.where(vis, z, -np.inf)
    top = z.max(-1, keepdims=True)
    w = np.where(vis, np.exp(z - np.where(np.isfinite(top), top, 0.0)), 0.0)
    s = w.sum(-1, keepdims=True)
    w = w / np.where(s > 0, s, 1.0)
    return w @ keys[:, :rank], w @ np.abs(keys[:, :rank]), (np.abs(q) @ np.abs(keys).T * abs(scale)).max()


def filtered(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Probabilities of one row after the filters, and the distance of each threshold from the nearest value that would change
    what is kept (relative to the mass it is compared with; inf where a filter is off), and `among`, how many tokens top-p's
    mass is a sum over."""
    x = np.asarray(logits, dtype=np.float64)
    V = len(x)
    live = ~(np.isnan(x) | (x == -np.inf))
    if not live.any():
        return np.zeros(V), dict(top_p=np.inf, min_p=np.inf, among=0)
    key = np.where(live, x, -np.inf)
    order = np.lexsort((np.arange(V), -key))[: live.sum()]
    top = key[order[0]]
    margins = dict(top_p=np.inf, min_p=np.inf, among=1)
    p = np.zeros(V)
    if not temperature > 0:
        p[order[0]] = 1.0
        return p, margins
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.exp(np.where(key[order] == top, 0.0, key[order] - top) / np.float64(temperature))
    kept = len(order) if top_k <= 0 else min(len(order), int(top_k))
    margins["among"] = kept
    if top_p < 1.0:
        c = np.cumsum(w[:kept])
        want = np.float64(max(top_p, 0.0)) * c[-1]
        m = min(kept, int((c < want).sum()) + 1)
        margins["top_p"] = min(abs(c[m - 1] - want), abs(c[m - 2] - want) if m > 1 else np.inf) / c[-1] if top_p > 0 else np.inf
        kept = m
    if min_p > 0:
        margins["min_p"] = np.abs(np.log(np.maximum(w, 1e-300)) - np.log(min(np.float64(min_p), 1.0))).min() if min_p < 1 else np.inf
        kept = max(1, min(kept, int((w >= min(np.float64(min_p), 1.0)).sum())))
    p[order[:kept]] = w[:kept]
    return p / p.sum(), margins


def draws(p, u):
    """Inverse-CDF draws in id order, and the distance of each uniform from the nearest border between two ids."""
    if not p.any():
        return np.full(len(u), -1), np.full(len(u), np.inf)
    c = np.cumsum(p)
    c = c / c[-1]
    last = np.flatnonzero(p)[-1]
    ids = np.minimum(np.searchsorted(c, np.asarray(u, np.float64), side="right"), last)
    edges = np.concatenate([[-1.0], c[:last], [2.0]])      # below 0 and above the last id nothing changes
    at = np.clip(np.searchsorted(edges, np.asarray(u, np.float64)), 1, len(edges) - 1)
    return ids, np.minimum(np.abs(edges[at] - u), np.abs(edges[at - 1] - u))
