"""Performance cases of the operators that evaluate a member of the evolution
strategy: the pages of its rollouts' key-value cache, the attention that reads
them, and the scores of the tokens.

A case is one of six kinds of work:

* ``attend``    one new token per sequence over a paged cache, ragged lengths,
                optionally a sliding window with sink tokens;
* ``append``    the keys and values of new tokens enter their pages;
* ``rollouts``  the next member's rollouts start: every sequence of the last
                member is freed, the prompts' pages are reserved and each
                prompt is forked into its rollouts;
* ``compact``   the live pages of a fragmented pool move to its front;
* ``score``     log probabilities of given tokens, entropies and the most
                likely alternatives;
* ``train``     log probabilities and entropies with the gradient of both.

``listed()`` has the named ones, ``draw()`` spreads over the same ranges.  With
``own`` false a pass computes the operator with elementary torch operations in
32 bits; with ``own`` true it makes the calls of ``paper_2608_02391_amd``.
``exact()`` evaluates a case in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

VOCAB = 151936                  # vocabulary of the 4 G-parameter configuration; 32 query and 8 key heads of 128
ATTEND_BYTES = 3.3e9            # keys and values of the largest attention
LOGIT_BYTES = 1.25e9            # logits of the largest scoring


def listed():
    return [
        # the first tokens of a single rollout of a small model: launches and latency count
        dict(name="attend_first", kind="attend", rows=1, longest=200, shortest=200, lens=1, q_heads=8, kv_heads=2, dim=64,
             page=16, dtype="bf16", order="hnd", window=0, sinks=0),
        # a batch of rollouts in mid-generation, of very different lengths
        dict(name="attend_ragged", kind="attend", rows=40, longest=8191, shortest=33, lens=2, q_heads=32, kv_heads=8,
             dim=128, page=16, dtype="bf16", order="hnd", window=0, sinks=0),
        # agents at the 128 K context the method is meant for: the largest call
        dict(name="attend_long", kind="attend", rows=8, longest=131072, shortest=65000, lens=3, q_heads=32, kv_heads=8,
             dim=128, page=64, dtype="bf16", order="hnd", window=0, sinks=0),
        # fp32 weights and cache, token-major pages, a window with sinks over long rollouts
        dict(name="attend_window", kind="attend", rows=24, longest=30000, shortest=900, lens=4, q_heads=16, kv_heads=8,
             dim=128, page=32, dtype="fp32", order="nhd", window=4096, sinks=4),
        # one decoding step of 48 rollouts
        dict(name="append_step", kind="append", rows=48, tokens=1, lens=5, kv_heads=8, dim=128, page=16, dtype="bf16",
             order="hnd"),
        # the prompts of a batch, ragged
        dict(name="append_prompts", kind="append", rows=24, tokens=2047, lens=6, kv_heads=8, dim=128, page=16,
             dtype="bf16", order="hnd"),
        # four rollouts of one short prompt
        dict(name="rollouts_small", kind="rollouts", prompts=1, each=4, longest=100, lens=7, layers=2, kv_heads=2,
             dim=64, page=16, dtype="bf16", order="hnd"),
        # a member's whole batch: 32 prompts of up to 2,000 tokens, 8 rollouts each, 12 layers
        dict(name="rollouts_batch", kind="rollouts", prompts=32, each=8, longest=2000, lens=8, layers=12, kv_heads=4,
             dim=64, page=16, dtype="bf16", order="hnd"),
        # a pool of 6,000 pages a third full after most rollouts have ended
        dict(name="compact_pool", kind="compact", pages=6000, seqs=64, live=0.33, lens=9, layers=12, kv_heads=4, dim=64,
             page=16, dtype="bf16", order="hnd"),
        # the alternatives of one sampled token
        dict(name="score_token", kind="score", rows=1, vocab=VOCAB, top=20, dtype="bf16", scale=1.0, allowed=1.0),
        # the tokens of a batch of rollouts: the largest logits
        dict(name="score_rollouts", kind="score", rows=4096, vocab=VOCAB, top=5, dtype="bf16", scale=1.0, allowed=1.0),
        # the gradient of a scored batch over an odd vocabulary, sampled at a temperature
        dict(name="train_rollouts", kind="train", rows=2000, vocab=50257, dtype="bf16", scale=1.25, allowed=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "rollouts", "compact", "score", "score", "train"])
    dtype, order = rng.choice(["bf16", "bf16", "bf16", "fp32"]), rng.choice(["hnd", "hnd", "nhd"])
    lens = rng.randint(100, 1 << 30)
    kv, dim, page = rng.choice([1, 2, 4, 8, 8]), rng.choice([64, 128, 128, 128, 80, 256]), rng.choice([8, 16, 16, 32, 64, 48])
    e = 4 if dtype == "fp32" else 2
    if kind == "attend":
        group, rows, longest = rng.choice([1, 2, 4, 4, 8, 16]), _log_int(rng, 1, 128), _log_int(rng, 1, 131072)
        while rows > 1 and rows * longest * kv * dim * 2 * e > ATTEND_BYTES:
            rows = (rows + 1) // 2
        windowed = rng.random() < 0.3
        return dict(kind=kind, rows=rows, longest=longest, shortest=max(1, longest // rng.choice([1, 4, 64])), lens=lens,
                    q_heads=kv * group, kv_heads=kv, dim=dim, page=page, dtype=dtype, order=order,
                    window=_log_int(rng, 16, 8192) if windowed else 0, sinks=rng.choice([0, 4, 37]) if windowed else 0)
    if kind == "append":
        return dict(kind=kind, rows=_log_int(rng, 1, 64), tokens=rng.choice([1, _log_int(rng, 2, 1000)]), lens=lens,
                    kv_heads=kv, dim=dim, page=page, dtype=dtype, order=order)
    if kind == "rollouts":
        return dict(kind=kind, prompts=_log_int(rng, 1, 32), each=rng.randint(1, 8), longest=_log_int(rng, 4, 2000), lens=lens,
                    layers=rng.randint(1, 12), kv_heads=min(kv, 4), dim=64, page=rng.choice([8, 16, 16]), dtype="bf16",
                    order=order)
    if kind == "compact":
        return dict(kind=kind, pages=_log_int(rng, 50, 6000), seqs=_log_int(rng, 1, 64), live=rng.uniform(0.1, 0.9), lens=lens,
                    layers=rng.randint(1, 12), kv_heads=min(kv, 4), dim=64, page=rng.choice([8, 16, 16]), dtype="bf16",
                    order=order)
    vocab = rng.choice([_log_int(rng, 300, VOCAB), 32768, VOCAB])
    most = LOGIT_BYTES / (vocab * e) / (2 if kind == "train" else 1)
    case = dict(kind=kind, rows=max(1, min(_log_int(rng, 1, 8192), int(most))), vocab=vocab, dtype=dtype,
                scale=rng.choice([1.0, 1.0, 1.25, 0.7]), allowed=rng.choice([1.0, 1.0, 0.5]))
    return dict(case, top=rng.choice([1, 5, 20, 32])) if kind == "score" else case


# ------------------------------------------------------------------- inputs --

def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


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


def _lengths(case, count, shortest, longest):
    """Lengths spread over their logarithm, the longest among them: a property of the case."""
    rng = random.Random(case["lens"])
    out = [longest] + [_log_int(rng, shortest, longest) for _ in range(count - 1)]
    rng.shuffle(out)
    return out


def _pages(n, page):
    return -(-n // page)


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


def _prepare_attend(case, seed):
    g, B, D = _generator(seed), case["rows"], case["dim"]
    lens = _lengths(case, B, case["shortest"], case["longest"])
    counts = [_pages(n, case["page"]) for n in lens]
    n_pages = sum(counts) + 3
    k, v = _cache(case, 1, n_pages, g)
    table = torch.from_numpy(_table(counts, n_pages, max(counts), seed)).cuda()
    # the queries come out of one projection together with the keys and values of the new token
    qkv = _normal((B, case["q_heads"] + 2 * case["kv_heads"], D), _dtype(case), g, 2.0)
    out = torch.empty(B, case["q_heads"], D, dtype=_dtype(case), device="cuda")
    lse = torch.empty(B, case["q_heads"], dtype=torch.float32, device="cuda")
    st = dict(case=case, k=k, v=v, table=table, lens=lens, q=qkv[:, :case["q_heads"]], out=out, lse=lse)
    if own:
        import paper_2608_02391_amd as cp

        st["cache"], st["pool"] = cp.paged_cache(k, v), cp.page_pool(table, _ints(lens), case["page"])
        nbytes = cp.cpes_attend_workspace_bytes(B, case["q_heads"], case["kv_heads"], D)
        st["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return st


def _append_tokens(case):
    """(tokens of each sequence, its length after them)."""
    if case["tokens"] == 1:
        return [1] * case["rows"], _lengths(case, case["rows"], 1, 500)
    n = _lengths(case, case["rows"], 1, case["tokens"])
    return n, n


def _prepare_append(case, seed):
    g = _generator(seed)
    new, lens = _append_tokens(case)
    counts = [_pages(n, case["page"]) for n in lens]
    n_pages = sum(counts) + 3
    k, v = _cache(case, 1, n_pages, g)
    table = torch.from_numpy(_table(counts, n_pages, max(counts), seed)).cuda()
    H = case["kv_heads"]
    qkv = _normal((sum(new), 3 * H, case["dim"]), _dtype(case), g)
    seqs = _ints([s for s, n in enumerate(new) for _ in range(n)])
    pos = _ints([lens[s] - n + t for s, n in enumerate(new) for t in range(n)])
    st = dict(case=case, k=k, v=v, table=table, seqs=seqs, pos=pos, k_new=qkv[:, H:2 * H], v_new=qkv[:, 2 * H:])
    if own:
        import paper_2608_02391_amd as cp

        st["cache"], st["pool"] = cp.paged_cache(k, v), cp.page_pool(table, _ints(lens), case["page"])
    return st


def _rollout_shape(case):
    """(prompt lengths, pages in the pool, width of the table)."""
    lens = _lengths(case, case["prompts"], min(3, case["longest"]), case["longest"])
    need = sum(_pages(n, case["page"]) + case["each"] for n in lens)
    return lens, need + need // 4 + 2, _pages(case["longest"], case["page"]) + 4


def _prepare_rollouts(case, seed):
    g, P, R = _generator(seed), case["prompts"], case["each"]
    lens, n_pages, width = _rollout_shape(case)
    k, v = _cache(case, case["layers"], n_pages, g)
    # the last member's rollouts as they ended: the same prompts in another order, on scattered pages
    last = [int(n) for n in np.random.default_rng(seed + 1).permutation(lens)]
    counts = [_pages(n, case["page"]) for n in last] + [1] * (P * R)
    table = _table(counts, n_pages, width, seed)
    refs = np.zeros(n_pages, dtype=np.int32)
    for p in range(P):
        full = last[p] // case["page"]
        refs[table[p, :counts[p]]] += 1
        for c in range(P + p * R, P + (p + 1) * R):
            tail, table[c, 0] = table[c, 0], -1
            table[c, :full] = table[p, :full]
            refs[table[c, :full]] += 1
            if last[p] % case["page"]:
                table[c, full] = tail
                refs[tail] += 1
    lengths = last + [n for n in last for _ in range(R)]
    st = dict(case=case, k=k, v=v, table=torch.from_numpy(table).cuda(), refs=torch.from_numpy(refs).cuda(),
              lengths=_ints(lengths), everyone=_ints(list(range(P + P * R))), prompts=_ints(list(range(P))),
              new=_ints(lens), parents=_ints([p for p in range(P) for _ in range(R)]),
              children=_ints(list(range(P, P + P * R))), status=torch.zeros(3, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2608_02391_amd as cp

        st["cache"], st["codes"] = cp.paged_cache(k, v), st["status"].split(1)
        st["pool"] = cp.page_pool(st["table"], st["lengths"], case["page"], st["refs"])
        st["ws"] = torch.empty(cp.cpes_pages_workspace_bytes(n_pages), dtype=torch.uint8, device="cuda")
    return st


def _compact_counts(case):
    """Pages of each sequence: about live x pages in all."""
    rng, left = random.Random(case["lens"]), int(case["live"] * case["pages"])
    cuts = sorted(rng.randint(0, left) for _ in range(case["seqs"] - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [left])]


def _prepare_compact(case, seed):
    g, n = _generator(seed), case["pages"]
    counts = _compact_counts(case)
    k, v = _cache(case, case["layers"], n, g)
    table = _table(counts, n, max(1, max(counts)), seed)
    refs = np.zeros(n, dtype=np.int32)
    refs[table[table >= 0]] = 1
    lengths = [c * case["page"] - (s % case["page"] if c else 0) for s, c in enumerate(counts)]
    st = dict(case=case, k=k, v=v, table=torch.from_numpy(table).cuda(), refs=torch.from_numpy(refs).cuda(),
              lengths=_ints(lengths))
    st.update(table2=torch.empty_like(st["table"]), refs2=torch.empty_like(st["refs"]),
              lengths2=torch.empty_like(st["lengths"]), moved=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2608_02391_amd as cp

        st["cache"] = cp.paged_cache(k, v)
        st["pool"] = cp.page_pool(st["table"], st["lengths"], case["page"], st["refs"])
        st["packed"] = cp.page_pool(st["table2"], st["lengths2"], case["page"], st["refs2"])
        st["ws"] = torch.empty(cp.cpes_pages_workspace_bytes(n), dtype=torch.uint8, device="cuda")
    return st


def _prepare_logits(case, seed):
    g, N, V = _generator(seed), case["rows"], case["vocab"]
    x = _normal((N, V), _dtype(case), g, 2.5)
    target = torch.randint(0, V, (N,), generator=g, device="cuda")
    # a sampled token is a likely one more often than not
    boost = torch.randn(N, generator=g, device="cuda") * 4 + 12
    if case["allowed"] < 1.0:
        # a grammar forbids a part of the vocabulary, another part from row to row
        shift = torch.randint(0, V, (N,), generator=g, device="cuda")
        token = torch.arange(V, device="cuda")
        for r in range(0, N, 256):
            x[r:r + 256].masked_fill_((token + shift[r:r + 256, None]) % V >= int(case["allowed"] * V), -math.inf)
    x[torch.arange(N, device="cuda"), target] = boost.to(x.dtype)
    st = dict(case=case, x=x, target=target, logp=torch.empty(N, device="cuda"), entropy=torch.empty(N, device="cuda"),
              lse=torch.empty(N, device="cuda"), stats=torch.empty(N, 2, device="cuda"))
    if case["kind"] == "train":
        st.update(d_logp=torch.randn(N, generator=g, device="cuda") / N, d_entropy=torch.full((N,), 0.01 / N, device="cuda"),
                  dx=torch.empty_like(x))
    else:
        st.update(top_logp=torch.empty(N, case["top"], device="cuda"),
                  top_ids=torch.empty(N, case["top"], dtype=torch.int64, device="cuda"))
    if own:
        import paper_2608_02391_amd as cp

        nbytes = cp.cpes_logprobs_workspace_bytes(N, V, case.get("top", 0))
        st["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return st


def prepare(case, seed):
    return {"attend": _prepare_attend, "append": _prepare_append, "rollouts": _prepare_rollouts,
            "compact": _prepare_compact, "score": _prepare_logits, "train": _prepare_logits}[case["kind"]](case, seed)


# ---------------------------------------------- one pass, elementary operations --

def _visible(case, n):
    """Positions the token at n - 1 sees."""
    w, s = case["window"], case["sinks"]
    if w == 0 or s + w >= n:
        return torch.arange(n, device="cuda")
    return torch.cat([torch.arange(s, device="cuda"), torch.arange(n - w, n, device="cuda")])


def _plain_attend(st):
    case, P, H = st["case"], st["case"]["page"], st["case"]["kv_heads"]
    for r, n in enumerate(st["lens"]):
        at = _visible(case, n)
        page, slot = st["table"][r].long()[at // P], at % P
        k = st["k"][0][page, :, slot].float().transpose(0, 1)
        v = st["v"][0][page, :, slot].float().transpose(0, 1)
        q = st["q"][r].float().view(H, -1, case["dim"])
        s = (q @ k.transpose(1, 2)) * case["dim"] ** -0.5
        m = s.amax(-1, keepdim=True)
        p = (s - m).exp()
        total = p.sum(-1, keepdim=True)
        st["out"][r] = ((p @ v) / total).reshape(-1, case["dim"])
        st["lse"][r] = (m + total.log()).reshape(-1)
    return {"out": st["out"], "lse": st["lse"]}


def _plain_append(st):
    P, pos = st["case"]["page"], st["pos"].long()
    page = st["table"][st["seqs"].long(), pos // P].long()
    st["k"][0][page, :, pos % P] = st["k_new"]
    st["v"][0][page, :, pos % P] = st["v_new"]
    return {"k": st["k"], "v": st["v"]}


def _plain_rollouts(st):
    case, table, refs, lengths = st["case"], st["table"], st["refs"], st["lengths"]
    P, width = case["page"], table.shape[1]
    slot = torch.arange(width, device="cuda")
    everyone, prompts, parents, children = (st[n].long() for n in ("everyone", "prompts", "parents", "children"))
    # free: every page loses one reference for each sequence that held it
    held = slot < ((lengths[everyone] + P - 1) // P)[:, None]
    refs.index_add_(0, table[everyone][held].long(), torch.full((), -1, dtype=torch.int32, device="cuda").expand(int(held.sum())))
    table[everyone], lengths[everyone] = -1, 0
    # reserve: the lowest free pages, in the order of the prompts
    new = st["new"]
    used = slot < ((new + P - 1) // P)[:, None]
    free = (refs == 0).nonzero().view(-1)[:int(used.sum())]
    rows = table[prompts]
    rows[used] = free.int()
    table[prompts], lengths[prompts], refs[free] = rows, new, 1
    # fork: full pages are shared, the last partial one is copied
    n = lengths[parents]
    shared = slot < (n // P)[:, None]
    rows = torch.where(shared, table[parents], table[children])
    refs.index_add_(0, rows[shared].long(), torch.ones((), dtype=torch.int32, device="cuda").expand(int(shared.sum())))
    ragged = ((n % P) > 0).nonzero().view(-1)
    tail = (refs == 0).nonzero().view(-1)[:ragged.numel()]
    last = (n[ragged] // P).long()
    source = table[parents[ragged], last].long()
    rows[ragged, last] = tail.int()
    refs[tail] = 1
    for cache in (st["k"], st["v"]):
        cache[:, tail] = cache[:, source]
    table[children], lengths[children] = rows, n
    return {"table": table, "lengths": lengths, "refs": refs, "status": st["status"], "k": st["k"], "v": st["v"]}


def _plain_compact(st):
    case, table, refs = st["case"], st["table"], st["refs"]
    live = refs > 0
    n = int(live.sum())
    holes, movers = (~live[:n]).nonzero().view(-1), live[n:].nonzero().view(-1) + n
    for cache in (st["k"], st["v"]):
        cache[:, holes] = cache[:, movers]
    name = torch.arange(refs.numel(), device="cuda")
    name[movers] = holes
    held = torch.arange(table.shape[1], device="cuda") < ((st["lengths"] + case["page"] - 1) // case["page"])[:, None]
    st["table2"].copy_(torch.where(held, name[table.long().clamp(min=0)].int(), table))
    st["refs2"].copy_(refs)
    st["refs2"][holes] = refs[movers]
    st["refs2"][movers] = 0
    st["lengths2"].copy_(st["lengths"])
    st["moved"].fill_(movers.numel())
    return {"table": st["table2"], "refs": st["refs2"], "lengths": st["lengths2"], "moved": st["moved"],
            "k": st["k"], "v": st["v"]}


def _plain_statistics(st, x):
    """Of scaled logits x in 32 bits: log probabilities of every token, entropies."""
    m = x.amax(-1, keepdim=True)
    p = (x - m).exp()
    total = p.sum(-1, keepdim=True)
    st["lse"].copy_((m + total.log()).view(-1))
    every = x - m - total.log()
    p /= total
    entropy = -torch.where(p > 0, p * every, 0.0).sum(-1)
    st["logp"].copy_(every[torch.arange(x.shape[0], device="cuda"), st["target"]])
    st["entropy"].copy_(entropy)
    return every, p


def _plain_score(st):
    case = st["case"]
    raw = st["x"].float()
    every, _ = _plain_statistics(st, raw * case["scale"])
    row = torch.arange(case["rows"], device="cuda")
    raw = raw.clone() if raw.data_ptr() == st["x"].data_ptr() else raw
    for j in range(case["top"]):                      # the first of the largest, again and again
        at = raw.argmax(-1)
        st["top_ids"][:, j], st["top_logp"][:, j] = at, every[row, at]
        raw[row, at] = -math.inf
    return {"logp": st["logp"], "entropy": st["entropy"], "lse": st["lse"], "top_logp": st["top_logp"], "top_ids": st["top_ids"]}


def _plain_train(st):
    case = st["case"]
    every, p = _plain_statistics(st, st["x"].float() * case["scale"])
    g, h = st["d_logp"][:, None], st["d_entropy"][:, None]
    every += st["entropy"][:, None]
    d = torch.where(p > 0, p * (-g - h * every), 0.0)
    d[torch.arange(case["rows"], device="cuda"), st["target"]] += st["d_logp"]
    st["dx"].copy_(d * case["scale"])
    return {"logp": st["logp"], "entropy": st["entropy"], "lse": st["lse"], "dx": st["dx"]}


# -------------------------------------------------- one pass, the framework's --

def _own(st):
    import paper_2608_02391_amd as cp

    case, kind = st["case"], st["case"]["kind"]
    if kind == "attend":
        cp.cpes_attend(st["cache"], 0, st["pool"], st["q"], st["out"], lse=st["lse"], window=case["window"],
                       sinks=case["sinks"], workspace=st["ws"])
        return {"out": st["out"], "lse": st["lse"]}
    if kind == "append":
        cp.cpes_cache_append(st["cache"], 0, st["pool"], st["k_new"], st["v_new"], st["pos"], seqs=st["seqs"])
        return {"k": st["k"], "v": st["v"]}
    if kind == "rollouts":
        code = st["codes"]
        cp.cpes_pages_free(st["pool"], st["everyone"], status=code[0])
        cp.cpes_pages_reserve(st["pool"], st["prompts"], st["new"], st["ws"], status=code[1])
        cp.cpes_pages_fork(st["cache"], st["pool"], st["parents"], st["children"], st["ws"], status=code[2])
        return {"table": st["table"], "lengths": st["lengths"], "refs": st["refs"], "status": st["status"],
                "k": st["k"], "v": st["v"]}
    if kind == "compact":
        cp.cpes_pages_compact(st["cache"], st["pool"], st["packed"], st["ws"], moved=st["moved"])
        return {"table": st["table2"], "refs": st["refs2"], "lengths": st["lengths2"], "moved": st["moved"],
                "k": st["k"], "v": st["v"]}
    cp.cpes_logprobs(st["x"], st["target"], st["logp"], entropy=st["entropy"], lse=st["lse"], stats=st["stats"],
                     top_logp=st.get("top_logp"), top_ids=st.get("top_ids"), scale=case["scale"], workspace=st["ws"])
    out = {"logp": st["logp"], "entropy": st["entropy"], "lse": st["lse"]}
    if kind == "score":
        return dict(out, top_logp=st["top_logp"], top_ids=st["top_ids"])
    cp.cpes_logprobs_backward(st["x"], st["target"], st["stats"], st["entropy"], st["d_logp"], st["d_entropy"], st["dx"],
                              scale=case["scale"])
    return dict(out, dx=st["dx"])


def run(st):
    if own:
        return _own(st)
    return {"attend": _plain_attend, "append": _plain_append, "rollouts": _plain_rollouts, "compact": _plain_compact,
            "score": _plain_score, "train": _plain_train}[st["case"]["kind"]](st)


# -------------------------------------------------------------------- costs --

def work(case):
    """Each input read once and each output written once; the operations of the formulas."""
    kind, e = case["kind"], 4 if case["dtype"] == "fp32" else 2
    if kind in ("score", "train"):
        N, V = case["rows"], case["vocab"]
        if kind == "score":
            return {"bytes": N * (V * e + 8 + 12 + 12 * case["top"]), "flops": 5 * N * V}
        return {"bytes": N * (2 * V * e + 8 + 12 + 8), "flops": 11 * N * V}
    token = 2 * case["kv_heads"] * case["dim"] * e                 # key and value of one token in one layer
    if kind == "attend":
        n, B = _lengths(case, case["rows"], case["shortest"], case["longest"]), case["rows"]
        seen = sum(min(x, case["window"] + case["sinks"]) if case["window"] else x for x in n)
        rows = B * case["q_heads"]
        return {"bytes": seen * token + 4 * -(-seen // case["page"]) + rows * (2 * case["dim"] * e + 4),
                "flops": 4 * seen * case["q_heads"] * case["dim"]}
    if kind == "append":
        n = sum(_append_tokens(case)[0])
        return {"bytes": n * (2 * token + 12), "flops": 0}
    page = token * case["page"] * case["layers"]
    if kind == "rollouts":
        lens, n_pages, _ = _rollout_shape(case)
        tails = sum(case["each"] for n in lens if n % case["page"])
        entries = sum(_pages(n, case["page"]) * (1 + case["each"]) for n in lens)
        return {"bytes": 2 * page * tails + 16 * entries + 12 * n_pages, "flops": 0}
    # the expected number of live pages behind the front of their count
    live = sum(_compact_counts(case))
    moved = live - live * live // case["pages"]
    return {"bytes": 2 * page * moved + 8 * live + 8 * case["pages"], "flops": 0}


# ------------------------------------------------------------------- 64 bits --

def _exact_attend(case, seed):
    st = _prepare_attend(case, seed)
    D, P, group = case["dim"], case["page"], case["q_heads"] // case["kv_heads"]
    out = torch.empty(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    for r, n in enumerate(st["lens"]):
        pages = st["table"][r, :_pages(n, P)].long()
        j = torch.arange(n, device="cuda")
        seen = (j < case["sinks"]) | (j >= n - case["window"]) if case["window"] else j >= 0
        for h in range(case["kv_heads"]):
            keys, values = (x[0, pages, h].reshape(-1, D)[:n].double()[seen] for x in (st["k"], st["v"]))
            for i in range(h * group, (h + 1) * group):
                logits = (keys * st["q"][r, i].double()).sum(-1) / math.sqrt(D)
                lse[r, i] = torch.logsumexp(logits, 0)
                out[r, i] = (torch.exp(logits - lse[r, i])[:, None] * values).sum(0)
    return {"out": out, "lse": lse}


def _exact_append(case, seed):
    st = _prepare_append(case, seed)
    table, pos, seqs, P = (st[n].cpu().numpy() if n != "page" else case["page"] for n in ("table", "pos", "seqs", "page"))
    for t in range(len(pos)):
        page, slot = int(table[seqs[t]][pos[t] // P]), int(pos[t] % P)
        for cache, new in ((st["k"], st["k_new"]), (st["v"], st["v_new"])):
            cache[0, page, :, slot].copy_(new[t])
    return {"k": st["k"], "v": st["v"]}


def _exact_rollouts(case, seed):
    st = _prepare_rollouts(case, seed)
    P, R, page = case["prompts"], case["each"], case["page"]
    lens, n_pages, width = _rollout_shape(case)
    free, refs = list(range(n_pages)), [0] * n_pages
    rows = []
    for n in lens:
        rows.append([free.pop(0) for _ in range(_pages(n, page))])
        for i in rows[-1]:
            refs[i] += 1
    copies = []
    for p, n in enumerate(lens):
        for _ in range(R):
            row = rows[p][:n // page]
            if n % page:
                copies.append((rows[p][-1], free.pop(0)))
                row = row + [copies[-1][1]]
            for i in row:
                refs[i] += 1
            rows.append(row)
    for cache in (st["k"], st["v"]):
        for a, b in copies:
            cache[:, b] = cache[:, a]
    return {"table": _ints([row + [-1] * (width - len(row)) for row in rows]),
            "lengths": _ints(lens + [n for n in lens for _ in range(R)]), "refs": _ints(refs), "status": _ints([0, 0, 0]),
            "k": st["k"], "v": st["v"]}


def _exact_compact(case, seed):
    st = _prepare_compact(case, seed)
    refs, table, n = st["refs"].tolist(), st["table"].tolist(), case["pages"]
    live = [i for i in range(n) if refs[i] > 0]
    name = dict(zip(live, live))
    empty = [i for i in range(len(live)) if refs[i] == 0]
    late = [i for i in live if i >= len(live)]
    for a, b in zip(late, empty):
        name[a], refs[b], refs[a] = b, refs[a], 0
        for cache in (st["k"], st["v"]):
            cache[:, b] = cache[:, a]
    return {"table": _ints([[name.get(i, -1) for i in row] for row in table]), "refs": _ints(refs),
            "lengths": st["lengths"], "moved": _ints([len(late)]), "k": st["k"], "v": st["v"]}


def _exact_logits(case, seed):
    st = _prepare_logits(case, seed)
    N = case["rows"]
    out = {n: torch.empty(N, dtype=torch.float64, device="cuda") for n in ("logp", "entropy", "lse")}
    if case["kind"] == "train":
        out["dx"] = torch.empty(N, case["vocab"], dtype=torch.float64, device="cuda")
    else:
        out["top_logp"] = torch.empty(N, case["top"], dtype=torch.float64, device="cuda")
        out["top_ids"] = torch.empty(N, case["top"], dtype=torch.int64, device="cuda")
    for a in range(0, N, 256):
        b = min(N, a + 256)
        x, t = st["x"][a:b].double(), st["target"][a:b, None]
        lse = torch.logsumexp(case["scale"] * x, -1, keepdim=True)
        logp = case["scale"] * x - lse
        p = logp.exp()
        entropy = -(p * logp.clamp(min=-1e6)).sum(-1, keepdim=True)
        out["lse"][a:b], out["entropy"][a:b] = lse[:, 0], entropy[:, 0]
        out["logp"][a:b] = logp.gather(1, t)[:, 0]
        if case["kind"] == "train":
            # the softmax's Jacobian applied to the gradients of log p and of the entropy
            onehot = torch.zeros_like(p).scatter_(1, t, 1.0)
            g, h = st["d_logp"][a:b, None].double(), st["d_entropy"][a:b, None].double()
            out["dx"][a:b] = case["scale"] * (g * (onehot - p) - h * p * (logp.clamp(min=-1e6) + entropy))
        else:
            ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :case["top"]]
            out["top_ids"][a:b], out["top_logp"][a:b] = ids, logp.gather(1, ids)
    return out


def exact(case, seed):
    return {"attend": _exact_attend, "append": _exact_append, "rollouts": _exact_rollouts, "compact": _exact_compact,
            "score": _exact_logits, "train": _exact_logits}[case["kind"]](case, seed)
