"""Top-k, top-p and min-p, and a draw among what they keep, a row at a time in float64."""
import numpy as np


def kept_tokens(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The tokens that are kept, the likeliest first (equal logits: the lowest index first); None for a row without a distribution."""
    x = np.asarray(logits, dtype=np.float64)
    t, p, m = np.float64(temperature), np.float64(top_p), np.float64(min_p)
    if np.isnan(x).any() or not (x > -np.inf).any() or x.max() == np.inf or not t >= 0 or np.isnan(p) or np.isnan(m):
        return None
    order = np.argsort(-x, kind="stable")[:int((x > -np.inf).sum())]
    if t == 0 or p <= 0 or m > 1:
        return order[:1]
    w = np.exp((x[order] - x[order[0]]) / t)
    n = len(order) if top_k <= 0 else min(len(order), int(top_k))
    keep = n
    if p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[:n])])
        keep = max(1, int((before[:n] < p * before[n]).sum()))
    if m > 0:
        keep = min(keep, max(1, int((w >= m).sum())))
    return order[:keep]


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, its ln share of the kept weights, tokens kept)"""
    kept = kept_tokens(logits, temperature, top_k, top_p, min_p)
    if kept is None:
        return -1, np.nan, 0
    kept = np.sort(kept)
    x, t = np.asarray(logits, dtype=np.float64)[kept], np.float64(temperature)
    z = (x - x.max()) / t if t > 0 else np.where(x == x.max(), 0.0, -np.inf)
    up = np.cumsum(np.exp(z))
    at = min(int(np.searchsorted(up, np.float64(u) * up[-1], side="right")), len(kept) - 1)
    return int(kept[at]), float(z[at] - np.log(up[-1])), len(kept)


def masked(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(logits where kept, else -infinity; tokens kept); logits that are no distribution as they are, under parameters that are none nothing is kept"""
    kept = kept_tokens(logits, temperature, top_k, top_p, min_p)
    if kept is None:
        good = temperature >= 0 and not np.isnan(top_p) and not np.isnan(min_p)
        return np.array(logits) if good else np.full_like(np.asarray(logits), -np.inf), 0
    out = np.full_like(np.asarray(logits), -np.inf)
    out[kept] = np.asarray(logits)[kept]
    return out, len(kept)
