"""Verification of drafted tokens against the target's probabilities (the paper's subsection "Speculative Decoding"), from given random
numbers, in float64, one sequence at a time."""
import numpy as np


def distribution(logits, temperature):
    """p of a row, or None for a row that has none."""
    x = np.asarray(logits, dtype=np.float64)
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any() or not temperature >= 0:
        return None
    if temperature == 0:
        p = np.zeros(x.shape)
        p[int(np.argmax(x))] = 1.0
        return p
    w = np.exp((x - x.max()) / np.float64(temperature))
    return w / w.sum()


def draw(weights, u):
    """The lowest index up to which the weights sum to more than u times their total; the last one with any weight if none does."""
    c = np.cumsum(weights)
    at = int(np.searchsorted(c, u * c[-1], side="right"))
    return at if at < len(c) else int(np.nonzero(weights)[0][-1])


def accept(logits, drafts, probs, temperature, u):
    """logits [k + 1, vocab], drafts [k], probs [k, vocab] or None, u [k + 1, 2].  Returns (accepted, emitted tokens, their ln p)."""
    vocab, out, logp = len(logits[0]), [], []
    for i in range(len(logits)):
        p = distribution(logits[i], temperature)
        if p is None:
            return i, out + [-1], logp + [float("nan")]
        d = int(drafts[i]) if i < len(drafts) else -1
        weights = p
        if 0 <= d < vocab:
            q = float(probs[i][d]) if probs is not None else 1.0
            if float(u[i][0]) * q < p[d]:
                out.append(d)
                logp.append(float(np.log(p[d])))
                continue
            if probs is None:
                weights = p.copy()
                weights[d] = 0.0
            else:
                weights = np.maximum(p - np.asarray(probs[i], dtype=np.float64), 0.0)
            if not weights.sum() > 0:
                weights = p
        t = draw(weights, float(u[i][1]))
        return i, out + [t], logp + [float(np.log(p[t]))]
