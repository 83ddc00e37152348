"""Plain 64-bit sampling of a token: the oracle of sae_sample."""
import numpy as np


def order(logits):
    """Indexes of the tokens that may be taken, by falling logit, the lower index first."""
    l = np.asarray(logits, np.float64)
    ids = np.flatnonzero(l > -np.inf)  # false for NaN
    return ids[np.argsort(-l[ids], kind="stable")].tolist()


def weights(logits, ids, T):
    l = np.asarray(logits, np.float64)[ids]
    with np.errstate(over="ignore", invalid="ignore"):
        w = np.exp((l - l[0]) / float(T))
    return np.where(l == l[0], 1.0, 0.0 if np.isinf(l[0]) else w)  # the infinite ones share the weight at any T


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, share, kept tokens) of one row; the settings as the call takes them."""
    ids = order(logits)
    if not ids:
        return -1, 0.0, 0
    if not temperature > 0:
        return ids[0], 1.0, 1
    w = weights(logits, ids, temperature)
    n = min(top_k, len(ids)) if top_k > 0 else len(ids)
    if top_p < 1:  # the shortest head that holds top_p of the first n
        need, total, m = float(top_p) * w[:n].sum(), 0.0, 0
        while m < n and (m == 0 or total < need):
            total += w[m]
            m += 1
        n = m
    if min_p > 0:
        m = 0
        while m < n and w[m] >= float(min_p):
            m += 1
        n = max(m, 1)
    total = w[:n].sum()
    u = 0.0 if not u > 0 else min(u, 1.0)
    sums = np.cumsum(w[:n])
    at = int(np.searchsorted(sums, u * total, side="right"))
    if at >= n or w[at] == 0:
        at = int(np.nonzero(w[:n])[0][-1])
    return ids[at], w[at] / total, n


def margin(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """How near (in shares of the largest weight) the nearest border of a decision is, for a row that sample() answers:
    a kernel whose sums are off by less decides alike."""
    ids = order(logits)
    if not ids or not temperature > 0:
        return np.inf
    w = weights(logits, ids, temperature)
    n = min(top_k, len(ids)) if top_k > 0 else len(ids)
    near = np.inf
    if top_p < 1:
        need = float(top_p) * w[:n].sum()
        near = min(near, np.abs(np.cumsum(w[:n]) - need).min())
    if min_p > 0:
        near = min(near, np.abs(w - float(min_p)).min())
    n = sample(logits, u, temperature, top_k, top_p, min_p)[2]
    return min(near, np.abs(np.cumsum(w[:n]) - u * w[:n].sum()).min() if 0 < u < 1 else np.inf)
