"""Performance cases of a decoding step with drafted tokens: several new tokens of
a sequence at a time go through the paged cache, every one of them gets a next
token from its logits, and the drafted tokens that the samples confirm stay.

A case is one of three kinds of work:

* ``sample``  a token for each row of logits from a given uniform number, with
              temperature, top-k, top-p and min-p;
* ``tree``    attention of a tree of new tokens per sequence (or a chain, which
              is a prompt or a piece of one) over a paged cache, ragged lengths,
              optionally a sliding window with sink tokens;
* ``keep``    the end of the step: room for the drafted tokens is there
              (a reservation), the walk down each tree along the sampled tokens,
              and the kept path's keys and values moved together in every layer,
              the other pages given back.

``listed()`` has the named ones, ``draw()`` spreads over the same ranges.  With
``own`` false a pass computes the operator with elementary torch operations in
32 bits, and in 64 where a sum decides which token it is; with ``own`` true it
makes the calls of ``paper_2608_02391_amd``.  ``exact()`` evaluates a case in 64
bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

VOCAB = 151936                  # vocabulary of the 4 G-parameter configuration; 32 query and 8 key heads of 128
CACHE_BYTES = 2.2e9             # keys and values of the largest attention
ATTEND_FLOPS = 4.5e11           # its operations
LOGIT_BYTES = 1.25e9            # logits of the largest sampling
MOVE_BYTES = 1.2e9              # caches of the largest accepted step


def listed():
    return [
        # the next token of a single rollout, with the usual filters: launches and latency count
        dict(name="sample_token", kind="sample", rows=1, vocab=VOCAB, dtype="bf16", scale=1.25, top_k=20, top_p=0.95,
             min_p=0.0, allowed=1.0),
        # a batch of rollouts sampled from the model's own distribution, as a policy is
        dict(name="sample_plain", kind="sample", rows=256, vocab=VOCAB, dtype="bf16", scale=1.0, top_k=0, top_p=1.0,
             min_p=0.0, allowed=1.0),
        # fp32 logits of an odd vocabulary, half of it forbidden by a grammar, at a high temperature
        dict(name="sample_odd", kind="sample", rows=1000, vocab=50257, dtype="fp32", scale=0.75, top_k=0, top_p=1.0,
             min_p=0.05, allowed=0.5),
        # every node of a batch of drafted trees: the largest logits
        dict(name="sample_nodes", kind="sample", rows=4096, vocab=VOCAB, dtype="bf16", scale=1.0, top_k=0, top_p=0.95,
             min_p=0.0, allowed=1.0),
        # five drafted tokens of a single rollout of a small model
        dict(name="tree_first", kind="tree", rows=1, longest=200, shortest=200, nodes=5, chain=False, lens=1, q_heads=8,
             kv_heads=2, dim=64, page=16, dtype="bf16", order="hnd", window=0, sinks=0),
        # small trees of a batch of rollouts in mid-generation, of very different lengths
        dict(name="tree_ragged", kind="tree", rows=32, longest=8191, shortest=33, nodes=12, chain=False, lens=2, q_heads=32,
             kv_heads=8, dim=128, page=16, dtype="bf16", order="hnd", window=0, sinks=0),
        # wide trees of agents at the 128 K context the method is meant for
        dict(name="tree_long", kind="tree", rows=4, longest=131072, shortest=65000, nodes=64, chain=False, lens=3, q_heads=32,
             kv_heads=8, dim=128, page=64, dtype="bf16", order="hnd", window=0, sinks=0),
        # fp32 weights and cache, token-major pages, a window with sinks over long rollouts
        dict(name="tree_window", kind="tree", rows=24, longest=30000, shortest=900, nodes=7, chain=False, lens=4, q_heads=16,
             kv_heads=8, dim=128, page=32, dtype="fp32", order="nhd", window=4096, sinks=4),
        # the prompts of a batch, ragged, from an empty cache on: the most operations
        dict(name="tree_prompts", kind="tree", rows=8, longest=0, shortest=0, nodes=4095, chain=True, lens=5, q_heads=32,
             kv_heads=8, dim=128, page=16, dtype="bf16", order="hnd", window=0, sinks=0),
        # one rollout of a small model goes on behind its drafted tokens
        dict(name="keep_step", kind="keep", rows=1, longest=150, shortest=150, nodes=8, chain=False, lens=7, layers=2,
             kv_heads=2, dim=64, page=16, dtype="bf16", order="hnd"),
        # a member's whole batch of rollouts, 12 layers
        dict(name="keep_batch", kind="keep", rows=256, longest=400, shortest=20, nodes=24, chain=False, lens=8, layers=12,
             kv_heads=4, dim=64, page=16, dtype="bf16", order="hnd"),
        # drafted chains, fp32, odd pages: little but pages that go back moves
        dict(name="keep_chains", kind="keep", rows=60, longest=900, shortest=30, nodes=10, chain=True, lens=9, layers=8,
             kv_heads=2, dim=128, page=12, dtype="fp32", order="nhd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "tree", "tree", "tree", "keep"])
    dtype, order = rng.choice(["bf16", "bf16", "bf16", "fp32"]), rng.choice(["hnd", "hnd", "nhd"])
    e = 4 if dtype == "fp32" else 2
    if kind == "sample":
        vocab = rng.choice([_log_int(rng, 300, VOCAB), 32768, VOCAB])
        rows = max(1, min(_log_int(rng, 1, 8192), int(LOGIT_BYTES / (vocab * e))))
        return dict(kind=kind, rows=rows, vocab=vocab, dtype=dtype, scale=rng.choice([1.0, 1.0, 1.25, 0.75]),
                    top_k=rng.choice([0, 0, 1, 20, 50, _log_int(rng, 1, 1000)]), top_p=rng.choice([1.0, 1.0, 0.95, 0.9, 0.5]),
                    min_p=rng.choice([0.0, 0.0, 0.05, 0.01]), allowed=rng.choice([1.0, 1.0, 0.5]))
    lens = rng.randint(100, 1 << 30)
    kv, dim, page = rng.choice([1, 2, 4, 8, 8]), rng.choice([64, 128, 128, 128, 80, 256]), rng.choice([8, 16, 16, 32, 64, 48])
    chain = rng.random() < 0.3
    if kind == "keep":
        case = dict(kind=kind, rows=_log_int(rng, 1, 256), longest=_log_int(rng, 1, 1000), nodes=_log_int(rng, 1, 64), chain=chain,
                    lens=lens, layers=rng.randint(1, 12), kv_heads=min(kv, 4), dim=dim, page=page, dtype=dtype, order=order)
        case["shortest"] = max(1, case["longest"] // rng.choice([1, 4, 64]))
        token = 2 * case["layers"] * case["kv_heads"] * dim * e
        while case["rows"] > 1 and case["rows"] * (case["longest"] + case["nodes"] + page) * token > MOVE_BYTES:
            case["rows"] = (case["rows"] + 1) // 2
        return case
    group = rng.choice([1, 2, 4, 4, 8, 16])
    longest, rows = rng.choice([0, _log_int(rng, 1, 131072), _log_int(rng, 1, 131072)]) if chain else _log_int(rng, 1, 131072), _log_int(rng, 1, 64)
    nodes = _log_int(rng, 1, 4096) if chain else _log_int(rng, 1, 64)
    cost = 4 * dim * kv * group * (4 if dtype == "fp32" else 1)
    while rows > 1 and (rows * (longest + nodes) * kv * dim * 2 * e > CACHE_BYTES or rows * nodes * (longest + nodes / 2) * cost > ATTEND_FLOPS):
        rows = (rows + 1) // 2
    while nodes > 1 and rows * nodes * (longest + nodes / 2) * cost > ATTEND_FLOPS:
        nodes = (nodes + 1) // 2
    windowed = rng.random() < 0.3
    return dict(kind=kind, rows=rows, longest=longest, shortest=max(min(longest, 1), longest // rng.choice([1, 4, 64])),
                nodes=nodes, chain=chain, lens=lens, q_heads=kv * group, kv_heads=kv, dim=dim, page=page, dtype=dtype, order=order,
                window=_log_int(rng, 16, 8192) if windowed else 0, sinks=rng.choice([0, 4, 37]) if windowed else 0)


# ------------------------------------------------------------------- inputs --

def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _f32(x):
    """The calls take their parameters in 32 bits."""
    return float(np.float32(x))


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g, std=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for s in range(0, flat.numel(), 1 << 28):
        e = min(flat.numel(), s + (1 << 28))
        flat[s:e] = torch.randn(e - s, generator=g, device="cuda").mul_(std)
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pages(n, page):
    return -(-n // page)


def _spread(rng, count, shortest, longest):
    """Numbers spread over their logarithm, the longest among them."""
    if longest == 0:
        return [0] * count
    out = [longest] + [_log_int(rng, max(1, shortest), longest) for _ in range(count - 1)]
    rng.shuffle(out)
    return out


class _Drafts:
    """Committed lengths and drafted trees of a case, a property of the case alone:
    ``base`` and ``size`` of each row, ``starts``, and for every node its parent
    within the row, its depth, and whether the walk down the tree passes it."""

    def __init__(self, case):
        rng = random.Random(case["lens"])
        self.base = _spread(rng, case["rows"], case["shortest"], case["longest"])
        self.size = _spread(rng, case["rows"], max(1, case["nodes"] // (64 if case["chain"] else 4)), case["nodes"])
        self.starts = [0]
        self.parents, self.depth, self.paths = [], [], []
        for n in self.size:
            # one token is certain, the others hang from the ones before, more often from late ones
            parent = [-1] + [i - 1 if case["chain"] else i - 1 - min(i - 1, int(rng.expovariate(0.5))) for i in range(1, n)]
            depth = [0] * n
            for i in range(1, n):
                depth[i] = depth[parent[i]] + 1
            path, at = [0], 0
            while case["kind"] == "keep" and rng.random() < 0.75:
                below = [i for i in range(at + 1, n) if parent[i] == at]
                if not below:
                    break
                at = rng.choice(below)
                path.append(at)
            self.starts.append(self.starts[-1] + n)
            self.parents += parent
            self.depth += depth
            self.paths.append(path)
        self.tokens = self.starts[-1]
        self.total = [b + n for b, n in zip(self.base, self.size)]


def _cache(case, layers, pages, g):
    """Keys and values [layers, pages, heads, page, dim], token-major in memory for "nhd"."""
    H, P, D = case["kv_heads"], case["page"], case["dim"]
    if case["order"] == "nhd":
        return tuple(_normal((layers, pages, P, H, D), _dtype(case), g).transpose(2, 3) for _ in range(2))
    return tuple(_normal((layers, pages, H, P, D), _dtype(case), g) for _ in range(2))


def _table(pages_of, n_pages, width, seed):
    """A page table whose sequences own pages scattered over the pool."""
    ids = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
    table, at = np.full((len(pages_of), width), -1, dtype=np.int32), 0
    for s, n in enumerate(pages_of):
        table[s, :n] = ids[at:at + n]
        at += n
    return table


def _prepare_sample(case, seed):
    g, N, V = _generator(seed), case["rows"], case["vocab"]
    x = _normal((N, V), _dtype(case), g, 2.5)
    # likely tokens: probabilities fall with a power of their rank, from row to row more or less surely
    ranks = min(200, V // 2)
    ids = torch.randint(0, V, (N, ranks), generator=g, device="cuda")
    top = 16 + 7 * torch.rand(N, 1, generator=g, device="cuda")
    slope = 1 + torch.rand(N, 1, generator=g, device="cuda")
    likely = top - slope * torch.arange(1, ranks + 1, device="cuda").log() + 0.3 * torch.randn(N, ranks, generator=g, device="cuda")
    for i in reversed(range(ranks)):              # an id that comes twice keeps its first value
        x[torch.arange(N, device="cuda"), ids[:, i]] = likely[:, i].to(x.dtype)
    if case["allowed"] < 1.0:
        # a grammar forbids a part of the vocabulary, another part from row to row
        shift = torch.randint(0, V, (N,), generator=g, device="cuda")
        token = torch.arange(V, device="cuda")
        for r in range(0, N, 256):
            x[r:r + 256].masked_fill_((token + shift[r:r + 256, None]) % V >= int(case["allowed"] * V), -math.inf)
    st = dict(case=case, x=x, u=torch.rand(N, generator=g, device="cuda"), token=torch.empty(N, dtype=torch.int64, device="cuda"),
              logp=torch.empty(N, device="cuda"))
    if own:
        import paper_2608_02391_amd as cp

        st["ws"] = torch.empty(cp.cpes_sample_workspace_bytes(N, V), dtype=torch.uint8, device="cuda")
    return st


def _prepare_tree(case, seed):
    g, D, d = _generator(seed), case["dim"], _Drafts(case)
    counts = [_pages(n, case["page"]) for n in d.total]
    n_pages = sum(counts) + 3
    k, v = _cache(case, 1, n_pages, g)
    table = torch.from_numpy(_table(counts, n_pages, max(counts), seed)).cuda()
    # the queries come out of one projection together with the keys and values of the new tokens
    qkv = _normal((d.tokens, case["q_heads"] + 2 * case["kv_heads"], D), _dtype(case), g, 2.0)
    st = dict(case=case, k=k, v=v, table=table, drafts=d, q=qkv[:, :case["q_heads"]], starts=_ints(d.starts),
              parents=None if case["chain"] else _ints(d.parents), out=torch.empty(d.tokens, case["q_heads"], D, dtype=_dtype(case), device="cuda"),
              lse=torch.empty(d.tokens, case["q_heads"], device="cuda"))
    if own:
        import paper_2608_02391_amd as cp

        st["cache"], st["pool"] = cp.paged_cache(k, v), cp.page_pool(table, _ints(d.total), case["page"])
        nbytes = cp.cpes_attend_tree_workspace_bytes(case["rows"], d.tokens, case["nodes"], case["q_heads"], case["kv_heads"], D)
        st["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return st


def _prepare_keep(case, seed):
    g, d, P, N = _generator(seed), _Drafts(case), case["page"], case["rows"]
    counts = [_pages(n, P) for n in d.base]
    need = sum(_pages(n, P) for n in d.total)
    n_pages, width = need + need // 8 + 2, max(_pages(n, P) for n in d.total)
    k, v = _cache(case, case["layers"], n_pages, g)
    table = _table(counts, n_pages, width, seed)
    refs = np.zeros(n_pages, dtype=np.int32)
    refs[table[table >= 0]] = 1
    # drafted tokens, and what the model says behind each of them: on the path the next one, elsewhere anything
    rng = np.random.default_rng(seed)
    drafted = np.concatenate([(rng.integers(0, VOCAB) + 7919 * np.arange(n)) % VOCAB for n in d.size])     # apart in a row
    sampled = VOCAB + rng.integers(0, VOCAB, d.tokens)        # no drafted token
    for r, path in enumerate(d.paths):
        at = d.starts[r]
        for a, b in zip(path, path[1:]):
            sampled[at + a] = drafted[at + b]
        # a node off the path may agree with one of its children: the walk does not get there
        for i in range(1, d.size[r]):
            if i not in path and d.parents[at + i] not in path and rng.random() < 0.5:
                sampled[at + d.parents[at + i]] = drafted[at + i]
    longest = max(d.size)
    st = dict(case=case, k=k, v=v, drafts=d, table=torch.from_numpy(table).cuda(), refs=torch.from_numpy(refs).cuda(),
              lengths=_ints(d.base), seqs=_ints(list(range(N))), new=_ints(d.total), starts=_ints(d.starts),
              parents=None if case["chain"] else _ints(d.parents), drafted=torch.from_numpy(drafted).cuda(),
              sampled=torch.from_numpy(sampled).cuda(), kept=_ints([0] * N), path=_ints([[0] * longest] * N),
              next=torch.zeros(N, dtype=torch.int64, device="cuda"), status=torch.zeros(2, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2608_02391_amd as cp

        st["cache"], st["codes"] = cp.paged_cache(k, v), st["status"].split(1)
        st["pool"] = cp.page_pool(st["table"], st["lengths"], P, st["refs"])
        nbytes = max(cp.cpes_pages_workspace_bytes(n_pages), cp.cpes_pages_keep_workspace_bytes(N, longest))
        st["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return st


def prepare(case, seed):
    return {"sample": _prepare_sample, "tree": _prepare_tree, "keep": _prepare_keep}[case["kind"]](case, seed)


# ---------------------------------------------- one pass, elementary operations --

def _plain_sample(st):
    case = st["case"]
    scale, top_p, min_p = _f32(case["scale"]), _f32(case["top_p"]), _f32(case["min_p"])
    step = max(1, (1 << 26) // case["vocab"])
    for a in range(0, case["rows"], step):
        x = st["x"][a:a + step].double()
        z = (x - x.amax(-1, keepdim=True)) * scale
        w = z.exp()
        if case["top_k"] or top_p < 1 or min_p > 0:
            _, ids = st["x"][a:a + step].sort(dim=-1, descending=True, stable=True)
            k = min(case["top_k"] or case["vocab"], case["vocab"])
            ids = ids[:, :k]
            ranked = w.gather(1, ids)
            upto = ranked.cumsum(-1)
            keep = z.gather(1, ids) >= (math.log(min_p) if min_p > 0 else -math.inf)
            if top_p < 1:
                keep &= upto - ranked < top_p * upto[:, -1:]
            w = torch.zeros_like(w).scatter_(1, ids, torch.where(keep, ranked, 0.0))
        upto = w.cumsum(-1)
        total = upto[:, -1:]
        token = (upto <= st["u"][a:a + step, None] * total).sum(-1)
        st["token"][a:a + step] = token
        st["logp"][a:a + step] = (z.gather(1, token[:, None]) - total.log())[:, 0]
    return {"token": st["token"], "logp": st["logp"]}


def _ancestors(st, r):
    """Truth values [nodes, nodes]: the nodes of row r that each of them descends from, or is."""
    d, at = st["drafts"], st["drafts"].starts[r]
    parent = st["parents"][at:at + d.size[r]].long()
    node = torch.arange(d.size[r], device="cuda")
    seen, above = node[:, None] == node, parent
    for _ in range(max(d.depth[at:at + d.size[r]])):
        seen |= above[:, None] == node
        above = torch.where(above >= 0, parent[above.clamp(min=0)], -1)
    return seen


def _seen_rows(st, r, lo, hi, family):
    """Truth values [hi - lo, positions] of what nodes lo .. hi - 1 of row r see."""
    case, d = st["case"], st["drafts"]
    b, n, at = d.base[r], d.size[r], d.starts[r]
    if case["chain"]:
        depth = torch.arange(n, device="cuda")
        new = torch.arange(n, device="cuda") <= torch.arange(lo, hi, device="cuda")[:, None]
    else:
        depth = torch.tensor(d.depth[at:at + n], device="cuda")
        new = family[lo:hi]
    seen = torch.cat([torch.ones(hi - lo, b, dtype=torch.bool, device="cuda"), new], 1)
    if case["window"]:
        place = torch.cat([torch.arange(b, device="cuda"), b + depth])
        seen &= (place > (b + depth[lo:hi])[:, None] - case["window"]) | (place < case["sinks"])
    return seen


def _plain_tree(st):
    case, d, P, H, D = st["case"], st["drafts"], st["case"]["page"], st["case"]["kv_heads"], st["case"]["dim"]
    for r, n in enumerate(d.total):
        family = None if case["chain"] else _ancestors(st, r)
        at = torch.arange(n, device="cuda")
        page, slot = st["table"][r].long()[at // P], at % P
        k = st["k"][0][page, :, slot].float().transpose(0, 1)
        v = st["v"][0][page, :, slot].float().transpose(0, 1)
        step = max(1, (1 << 29) // (n * case["q_heads"]))
        for lo in range(0, d.size[r], step):
            hi = min(d.size[r], lo + step)
            rows = slice(d.starts[r] + lo, d.starts[r] + hi)
            q = st["q"][rows].float().view(hi - lo, H, -1, D).permute(1, 2, 0, 3).reshape(H, -1, D)
            s = ((q @ k.transpose(1, 2)) * D ** -0.5).view(H, -1, hi - lo, n)
            s = s.masked_fill(~_seen_rows(st, r, lo, hi, family), -math.inf)
            m = s.amax(-1, keepdim=True)
            p = (s - m).exp()
            total = p.sum(-1, keepdim=True)
            out = (p.view(H, -1, n) @ v).view(H, -1, hi - lo, D) / total
            st["out"][rows] = out.permute(2, 0, 1, 3).reshape(hi - lo, -1, D)
            st["lse"][rows] = (m + total.log()).view(-1, hi - lo).t()
    return {"out": st["out"], "lse": st["lse"]}


def _plain_keep(st):
    case, d, P, N = st["case"], st["drafts"], st["case"]["page"], st["case"]["rows"]
    table, refs, lengths = st["table"], st["refs"], st["lengths"]
    longest, width = st["path"].shape[1], table.shape[1]
    slot = torch.arange(width, device="cuda")
    row = torch.arange(N, device="cuda")
    # reserve: the lowest free pages, in the order of the sequences
    old, want = (lengths + P - 1) // P, (st["new"] + P - 1) // P
    lacks = (slot >= old[:, None]) & (slot < want[:, None])
    free = (refs == 0).nonzero().view(-1)[:int(lacks.sum())]
    table[lacks] = free.int()
    refs[free] = 1
    torch.maximum(lengths, st["new"], out=lengths)
    # the walk: nodes in a row's columns
    starts = st["starts"].long()
    size = starts[1:] - starts[:-1]
    node = torch.arange(longest, device="cuda")
    there = node < size[:, None]
    flat = (starts[:-1, None] + node).clamp(max=d.tokens - 1)
    parent = (node - 1).expand(N, -1) if case["chain"] else st["parents"].long()[flat]
    drafted, sampled = st["drafted"][flat], st["sampled"][flat]
    at, live = torch.zeros(N, dtype=torch.int64, device="cuda"), size > 0
    st["path"].fill_(-1)
    st["kept"].zero_()
    st["next"].fill_(-1)
    for i in range(longest):
        st["path"][:, i] = torch.where(live, at, -1)
        st["kept"] += live
        st["next"].copy_(torch.where(live, sampled[row, at], st["next"]))
        below = there & (parent == at[:, None]) & (node > at[:, None]) & (drafted == sampled[row, at][:, None]) & live[:, None]
        live = below.any(-1)
        at = torch.where(live, below.int().argmax(-1), at)
    # keys and values of the path, to where the drafted tokens begin
    base = lengths.long() - size
    moves = (node < st["kept"][:, None]) & (st["path"] != node)
    who, i = moves.nonzero(as_tuple=True)
    to, source = base[who] + i, base[who] + st["path"][who, i]
    to_page, from_page = table[who, to // P].long(), table[who, source // P].long()
    for cache in (st["k"], st["v"]):
        cache[:, to_page, :, to % P] = cache[:, from_page, :, source % P]
    lengths.copy_(base + st["kept"])
    behind = (slot >= ((lengths + P - 1) // P)[:, None]) & (slot < want[:, None])
    refs.index_add_(0, table[behind].long(), torch.full((), -1, dtype=torch.int32, device="cuda").expand(int(behind.sum())))
    table[behind] = -1
    return {"kept": st["kept"], "path": st["path"], "next": st["next"], "table": table, "lengths": lengths, "refs": refs,
            "status": st["status"], "k": st["k"], "v": st["v"]}


# -------------------------------------------------- one pass, the framework's --

def _own(st):
    import paper_2608_02391_amd as cp

    case, kind = st["case"], st["case"]["kind"]
    if kind == "sample":
        cp.cpes_sample(st["x"], st["u"], st["token"], logp=st["logp"], scale=case["scale"], top_k=case["top_k"],
                       top_p=case["top_p"], min_p=case["min_p"], workspace=st["ws"])
        return {"token": st["token"], "logp": st["logp"]}
    if kind == "tree":
        cp.cpes_attend_tree(st["cache"], 0, st["pool"], st["q"], st["out"], st["starts"], case["nodes"], parents=st["parents"],
                            lse=st["lse"], window=case["window"], sinks=case["sinks"], workspace=st["ws"])
        return {"out": st["out"], "lse": st["lse"]}
    code = st["codes"]
    cp.cpes_pages_reserve(st["pool"], st["seqs"], st["new"], st["ws"], status=code[0])
    cp.cpes_tree_accept(st["starts"], st["drafted"], st["sampled"], st["kept"], st["path"], st["next"], parents=st["parents"])
    cp.cpes_pages_keep(st["cache"], st["pool"], st["starts"], st["kept"], st["path"], st["ws"], seqs=st["seqs"], status=code[1])
    return {"kept": st["kept"], "path": st["path"], "next": st["next"], "table": st["table"], "lengths": st["lengths"],
            "refs": st["refs"], "status": st["status"], "k": st["k"], "v": st["v"]}


def run(st):
    if own:
        return _own(st)
    return {"sample": _plain_sample, "tree": _plain_tree, "keep": _plain_keep}[st["case"]["kind"]](st)


# -------------------------------------------------------------------- costs --

def work(case):
    """Each input read once and each output written once; the operations of the formulas."""
    kind, e = case["kind"], 4 if case["dtype"] == "fp32" else 2
    if kind == "sample":
        N, V = case["rows"], case["vocab"]
        return {"bytes": N * (V * e + 4 + 12), "flops": 4 * N * V}
    d = _Drafts(case)
    token = 2 * case["kv_heads"] * case["dim"] * e                 # key and value of one token in one layer
    if kind == "tree":
        w, s, read, pairs = case["window"], case["sinks"], 0, 0
        for r, (b, n) in enumerate(zip(d.base, d.size)):
            depth = d.depth[d.starts[r]:d.starts[r + 1]]
            read += min(b, max(0, w - 1) + s) + n if w else b + n
            pairs += sum(min(b + x + 1, w + s) if w else b + x + 1 for x in depth)
        return {"bytes": read * token + 4 * -(-read // case["page"]) + d.tokens * (case["q_heads"] * (2 * case["dim"] * e + 4) + 4),
                "flops": 4 * pairs * case["q_heads"] * case["dim"]}
    moved = sum(i != node for path in d.paths for i, node in enumerate(path))
    kept = sum(len(path) for path in d.paths)
    pages = sum(_pages(n, case["page"]) - _pages(b + len(p), case["page"]) for n, b, p in zip(d.total, d.base, d.paths))
    return {"bytes": 2 * moved * token * case["layers"] + 20 * d.tokens + 4 * kept + 16 * pages + 40 * case["rows"], "flops": 0}


# ------------------------------------------------------------------- 64 bits --

def _exact_sample(case, seed):
    st = _prepare_sample(case, seed)
    N, V = case["rows"], case["vocab"]
    tokens, logps = [], []
    for a in range(0, N, 256):
        x = st["x"][a:a + 256].double()
        p = torch.softmax(_f32(case["scale"]) * x, -1)
        order = torch.argsort(x, dim=-1, descending=True, stable=True)
        rank = torch.empty_like(order).scatter_(1, order, torch.arange(V, device="cuda").expand_as(order))
        if case["top_k"]:
            p = torch.where(rank < case["top_k"], p, 0.0)
        largest = p.amax(-1, keepdim=True)
        if case["top_p"] < 1:
            falling = p.gather(1, order)
            enough = _f32(case["top_p"]) * p.sum(-1, keepdim=True)
            # as many tokens as it takes for their sum to get there
            needed = torch.searchsorted(falling.cumsum(-1), enough) + 1
            p = torch.where(rank < needed, p, 0.0)
        p = torch.where(p >= _f32(case["min_p"]) * largest, p, 0.0)
        p /= p.sum(-1, keepdim=True)
        below = p.cumsum(-1)
        t = torch.searchsorted(below, st["u"][a:a + 256, None].double() * below[:, -1:], right=True)
        tokens.append(t[:, 0])
        logps.append(p.gather(1, t)[:, 0].log())
    return {"token": torch.cat(tokens), "logp": torch.cat(logps)}


def _exact_tree(case, seed):
    st = _prepare_tree(case, seed)
    d, D, P, group = st["drafts"], case["dim"], case["page"], case["q_heads"] // case["kv_heads"]
    if 4.0 * case["q_heads"] * D * sum(n * t for n, t in zip(d.total, d.size)) > 3e12:
        return None
    out = torch.empty(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    for r, n in enumerate(d.total):
        b, at = d.base[r], d.starts[r]
        # the text along each node's branch: node i continues what its parent has seen
        own_place, behind = [b + x for x in d.depth[at:at + d.size[r]]], []
        for i in range(d.size[r]):
            if case["chain"]:
                break
            behind.append([i] + (behind[d.parents[at + i]] if d.parents[at + i] >= 0 else []))
        pages = st["table"][r, :_pages(n, P)].long()
        j = torch.arange(n, device="cuda")
        place = torch.where(j < b, j, torch.tensor([0] * b + own_place, device="cuda"))
        step = max(1, (1 << 27) // n)
        for lo in range(0, d.size[r], step):
            hi = min(d.size[r], lo + step)
            hidden = torch.ones(hi - lo, n, dtype=torch.bool, device="cuda")
            hidden[:, :b] = False
            for i in range(lo, hi):
                if case["chain"]:
                    hidden[i - lo, b:b + i + 1] = False
                else:
                    hidden[i - lo, torch.tensor(behind[i], device="cuda") + b] = False
            if case["window"]:
                mine = torch.tensor(own_place[lo:hi], device="cuda")[:, None]
                hidden |= (mine - place >= case["window"]) & (place >= case["sinks"])
            for h in range(case["q_heads"]):
                keys, values = (x[0, pages, h // group].reshape(-1, D)[:n].double() for x in (st["k"], st["v"]))
                logits = st["q"][at + lo:at + hi, h].double() @ keys.t() / math.sqrt(D)
                logits[hidden] = -math.inf
                z = torch.logsumexp(logits, -1)
                lse[at + lo:at + hi, h] = z
                out[at + lo:at + hi, h] = torch.exp(logits - z[:, None]) @ values
    return {"out": out, "lse": lse}


def _exact_keep(case, seed):
    st = _prepare_keep(case, seed)
    d, P = st["drafts"], case["page"]
    table, refs, sampled = st["table"].tolist(), st["refs"].tolist(), st["sampled"].tolist()
    free = [p for p, n in enumerate(refs) if n == 0]
    for r, n in enumerate(d.total):
        for j in range(_pages(d.base[r], P), _pages(n, P)):
            table[r][j] = free.pop(0)
            refs[table[r][j]] = 1
    longest = st["path"].shape[1]
    moves = []
    for r, path in enumerate(d.paths):
        place = lambda i: (table[r][(d.base[r] + i) // P], (d.base[r] + i) % P)
        moves += [place(node) + place(i) for i, node in enumerate(path) if node != i]
    for r, path in enumerate(d.paths):
        for j in range(_pages(d.base[r] + len(path), P), _pages(d.total[r], P)):
            refs[table[r][j]] -= 1
            table[r][j] = -1
    if moves:
        a, b, c, e = torch.tensor(moves, device="cuda").t()
        for cache in (st["k"], st["v"]):
            flat = cache.permute(1, 3, 0, 2, 4)              # pages, tokens first
            flat[c, e] = flat[a, b]
    return {"kept": _ints([len(p) for p in d.paths]), "path": _ints([p + [-1] * (longest - len(p)) for p in d.paths]),
            "next": torch.tensor([sampled[d.starts[r] + p[-1]] for r, p in enumerate(d.paths)], device="cuda"),
            "table": _ints(table), "lengths": _ints([b + len(p) for b, p in zip(d.base, d.paths)]), "refs": _ints(refs),
            "status": _ints([0, 0]), "k": st["k"], "v": st["v"]}


def exact(case, seed):
    return {"sample": _exact_sample, "tree": _exact_tree, "keep": _exact_keep}[case["kind"]](case, seed)
