"""Sampling in 64 bits, one row (numpy)."""
import numpy as np


def order(x):
    """Tokens by logit, the lower one first where logits are equal."""
    return np.argsort(-x, kind="stable")


def kept(x, t, k, p, low):
    """Tokens that the cuts keep, in the order of the vocabulary, their weights, and how near the border of p was missed
    (relative to the weight of what k keeps)."""
    top = x.max()
    with np.errstate(all="ignore"):
        w = np.where(x == top, 1.0, np.where(np.isneginf(x), 0.0, np.exp((x - top) / t)))
    o = order(x)
    if 0 < k < len(x):
        o = o[:k]
    near = 1.0
    if p < 1:
        sums = np.cumsum(w[o])
        want = p * sums[-1]
        n = int(np.searchsorted(sums, want)) + 1
        near = np.abs(sums - want).min() / sums[-1]
        o = o[:n]
    if low > 0:
        o = o[:max(1, int((w[o] >= low).sum()))]
    o = np.sort(o)
    return o, w[o], near


def row(x, u, t=1.0, k=0, p=1.0, low=0.0):
    """(token, logprob, margin): margin is how near u fell to a border between two tokens, or p to one, relative to the sum."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    t, p, low, u = (float(a) for a in (t, p, low, u))
    if np.isneginf(x.max()):
        return -1, -np.inf, 1.0
    if t == 0 or k == 1 or p <= 0:
        return int(x.argmax()), 0.0, 1.0
    o, w, near = kept(x, t, k, p, low)
    sums = np.cumsum(w)
    at = min(int(np.searchsorted(sums, u * sums[-1], side="right")), len(o) - 1)
    borders = sums[:-1]
    if len(borders):
        near = min(near, np.abs(borders - u * sums[-1]).min() / sums[-1])
    return int(o[at]), float(np.log(w[at]) - np.log(sums[-1])), near
