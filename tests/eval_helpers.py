"""Plain 64-bit implementations of the evaluation operators, and the bounds the
kernels' arithmetic is held to."""
import math

import numpy as np
import torch

EPS = 2.0 ** -24                # half an ulp of fp32, relative


def visible(n, window=0, sinks=0):
    """Mask of the positions the token at n - 1 sees."""
    j = torch.arange(n)
    return (j < sinks) | (j >= n - window) if window else j >= 0


def attend(q, k, v, seen, scale):
    """One query head over keys [n, D] (float64): (out, lse, bound of out, bound of lse)
    of a kernel that keeps scores, weights' sums and outputs in fp32.

    A score is a sum of D products, each addition rounding the running sum: off
    by at most (D + 4) EPS sum |q k| (twice that, since an instruction may round
    its partial sums its own way).  A weight e^(x - m) then is off by the two
    scores' error, by a rounding of x - m and of its product with log2 e (|x - m|
    2 EPS, relative) and by 2^-21 of the hardware's exponential and, for a bf16
    cache, 2^-17 of the split into two bf16.  The sums over n positions are taken
    16 at a time and then in a tree: n / 16 + 64 roundings."""
    q, k, v = q.double(), k.double(), v.double()
    D, dv = q.numel(), v.shape[1]
    x = (k @ q) * scale
    x = torch.where(seen[:len(x)], x, torch.tensor(-math.inf, dtype=torch.float64))
    if not bool((x > -math.inf).any()):
        zero = torch.zeros(dv, dtype=torch.float64)
        return zero, -math.inf, zero, 0.0
    keep = x > -math.inf
    m = float(x[keep].max())
    p = torch.where(keep, torch.exp(x - m), torch.tensor(0.0, dtype=torch.float64))
    total = float(p.sum())
    vals = torch.where(keep[:, None], v, torch.tensor(0.0, dtype=torch.float64))
    out = (p @ vals) / total
    dx = 2 * (D + 4) * EPS * abs(scale) * float((k[keep].abs() @ q.abs()).max())
    spread = min(100.0, m - float(x[keep].min()))
    e = 2 * dx + 2 * EPS * spread + 2.0 ** -21 + 2.0 ** -16 + (len(x) / 16 + 64) * EPS
    lse = m + math.log(total)
    return out, lse, 2 * e * (p @ vals.abs()) / total, e + 4 * EPS * (abs(m) + abs(lse) + 1)


def rounding(dtype):
    """Half an ulp of the output's type, relative: 8 significant bits in bf16, 24 in fp32."""
    return 2.0 ** -8 if dtype == torch.bfloat16 else EPS


class Pages:
    """Tables, lengths and reference counts as cpes.h defines the page calls."""

    def __init__(self, sequences, width, pages, page_size):
        self.table = np.full((sequences, width), -1, dtype=np.int64)
        self.lengths = np.zeros(sequences, dtype=np.int64)
        self.refs = np.zeros(pages, dtype=np.int64)
        self.page_size = page_size

    def count(self, n):
        return -(-n // self.page_size)

    def free_pages(self):
        return [p for p in range(len(self.refs)) if self.refs[p] <= 0]

    def reserve(self, seqs, new):
        S, W = self.table.shape
        if len(set(seqs)) < len(seqs) or any(s < 0 or s >= S for s in seqs) or any(
                n < 0 or n > W * self.page_size for n in new):
            return 2
        need = [max(0, self.count(n) - self.count(self.lengths[s])) for s, n in zip(seqs, new)]
        free = self.free_pages()
        if sum(need) > len(free):
            return 1
        for s, n, k in zip(seqs, new, need):
            at = self.count(self.lengths[s])
            self.table[s, at:at + k], free = free[:k], free[k:]
            self.refs[self.table[s, at:at + k]] = 1
            self.lengths[s] = max(self.lengths[s], n)
        return 0

    def fork(self, parents, children):
        """(status, pairs of pages copied)"""
        S = len(self.lengths)
        if len(set(children)) < len(children) or any(s < 0 or s >= S for s in list(parents) + list(children)) or any(
                self.lengths[c] != 0 for c in children):
            return 2, []
        lens = [0 if p in children else int(self.lengths[p]) for p in parents]
        free = self.free_pages()
        if sum(n % self.page_size != 0 for n in lens) > len(free):
            return 1, []
        copies = []
        for p, c, n in zip(parents, children, lens):
            full = n // self.page_size
            self.table[c, :full] = self.table[p, :full]
            self.refs[self.table[c, :full]] += 1
            if n % self.page_size:
                self.table[c, full] = free.pop(0)
                self.refs[self.table[c, full]] = 1
                copies.append((int(self.table[p, full]), int(self.table[c, full])))
            self.lengths[c] = n
        return 0, copies

    def free(self, seqs):
        bad = 0
        for s in seqs:
            if s < 0 or s >= len(self.lengths):
                bad = 2
                continue
            n = self.count(self.lengths[s])
            np.subtract.at(self.refs, self.table[s, :n], 1)
            self.table[s, :n], self.lengths[s] = -1, 0
        return bad

    def compact(self):
        """Pairs of pages moved."""
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] <= 0]
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        name = np.arange(len(self.refs))
        name[movers] = holes
        for s, n in enumerate(self.lengths):
            k = self.count(n)
            self.table[s, :k] = name[self.table[s, :k]]
        for a, b in zip(movers, holes):
            self.refs[b], self.refs[a] = self.refs[a], 0
        return list(zip(movers, holes))

    def held(self):
        """Page ids of every sequence's own entries."""
        return [list(self.table[s, :self.count(n)]) for s, n in enumerate(self.lengths)]


def logprobs(x, target, scale, top):
    """Of one row of logits (float64 of the stored values): dict of the numbers."""
    z = scale * x
    V = len(z)
    m = float(z.max())
    if m == -math.inf:
        logp, entropy, lse = np.full(V, -math.inf), 0.0, -math.inf
    else:
        d = z - m
        p = np.exp(d)
        s = float(p.sum())
        lse = m + math.log(s)
        logp = d - math.log(s)
        p = p / s
        entropy = -float((p[p > 0] * logp[p > 0]).sum())
    order = np.lexsort((np.arange(V), -x))[:top]
    ids = np.full(top, -1, dtype=np.int64)
    tops = np.full(top, -math.inf)
    ids[:len(order)] = order
    tops[:len(order)] = logp[order]
    return dict(logp=logp[target] if 0 <= target < V else 0.0, entropy=entropy, lse=lse, ids=ids, tops=tops, every=logp)
