"""Plain implementations of a step with drafted tokens: what a tree's tokens see, the
draw from filtered logits in 64 bits, the walk, and the pages behind it."""
import math

import numpy as np
import torch


def random_tree(n, rng, spread=3):
    """Parents of a tree of n tokens: the first one, then each hangs from one before it."""
    return [-1] + [max(0, i - 1 - rng.randrange(spread)) for i in range(1, n)]


def branch(parents, i):
    """Token i and its ancestors, nearest first; a parent that is not before its child counts as none."""
    out = [i]
    while True:
        p = i - 1 if parents is None else parents[i]
        if p < 0 or p >= i:
            return out
        out.append(p)
        i = p


def seen_by(parents, i, base, n, window, sinks):
    """Mask over n positions of what token i of a tree behind `base` positions sees."""
    seen = torch.zeros(n, dtype=torch.bool)
    line = branch(parents, i)
    own = base + len(line) - 1

    def lets(p):
        return window == 0 or p > own - window or p < sinks

    for p in range(base):
        seen[p] = lets(p)
    for back, j in enumerate(line):
        seen[base + j] = lets(own - back)
    return seen


def draw(x, u, scale=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log probability, distance of the draw from the nearest border, relative) of one row of float64 logits.
    The parameters are those that the call takes, in 32 bits."""
    scale, top_p, min_p = (float(np.float32(v)) for v in (scale, top_p, min_p))
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or (x == math.inf).any():
        return -1, math.nan, 1.0
    if not (x > -math.inf).any():
        return -1, -math.inf, 1.0
    z = scale * (x - x.max())
    w = np.where(x > -math.inf, np.exp(z), 0.0)
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -math.inf]
    near = 1.0
    if top_k:
        order = order[:top_k]
    if top_p < 1:
        upto = np.cumsum(w[order])
        enough = top_p * upto[-1]
        near = min(near, float(np.abs(upto - enough).min() / upto[-1]))
        order = order[:int((upto - w[order] < enough).sum())]
    if min_p > 0:
        order = order[z[order] >= math.log(min_p)]
    kept = np.zeros_like(w)
    kept[order] = w[order]
    upto = np.cumsum(kept)
    target = (min(max(u, 0.0), 1 - 2.0 ** -53) if u == u else 0.0) * upto[-1]
    token = int((upto <= target).sum())
    if target > 0:
        near = min(near, float(np.abs(upto - target).min() / upto[-1]))
    return token, float(z[token] - math.log(upto[-1])), near


def walk(parents, drafted, sampled):
    """(the tokens that stay, the one sampled behind them)"""
    n = len(drafted)
    if n == 0:
        return [], -1
    at, path = 0, [0]
    while True:
        below = [j for j in range(at + 1, n) if (j - 1 if parents is None else parents[j]) == at and drafted[j] == sampled[at]]
        if not below:
            return path, sampled[at]
        at = below[0]
        path.append(at)
