"""The end of a step with drafted tokens: the walk along the sampled ones, and what stays
moving together in the cache, against host models; and a whole step as a program runs it."""
import math
import random

import pytest
import torch

import draft_helpers as D
import eval_helpers as H
import paper_2608_02391_amd as cp

pytestmark = pytest.mark.gpu
BF16, F32, INT32 = torch.bfloat16, torch.float32, torch.int32


def ints(x):
    return torch.tensor(x, dtype=INT32, device="cuda")


def accept(starts, drafted, sampled, longest, parents=None, stream=None):
    rows = len(starts) - 1
    kept, path = torch.full((rows,), -9, dtype=INT32, device="cuda"), torch.full((rows, longest), -9, dtype=INT32, device="cuda")
    behind = torch.full((rows,), -9, dtype=torch.int64, device="cuda")
    cp.cpes_tree_accept(ints(starts), torch.tensor(drafted, device="cuda", dtype=torch.int64),
                        torch.tensor(sampled, device="cuda", dtype=torch.int64), kept, path, behind,
                        parents=None if parents is None else ints(parents), stream=stream)
    return kept.tolist(), path.tolist(), behind.tolist()


@pytest.mark.parametrize("sizes", [[1], [0, 3, 1], [5, 64, 65, 2, 0, 128, 129, 256], [7] * 300])
@pytest.mark.parametrize("chain", [False, True], ids=["tree", "chain"])
def test_walks(sizes, chain):
    """Few different tokens, so that siblings agree and walks go far."""
    print(f"accept {sizes[:4]} chain={chain}", flush=True)
    rng = random.Random(len(sizes))
    for alike in (1, 2, 5):
        starts, trees, drafted, sampled = [0], [], [], []
        for n in sizes:
            trees.append(None if chain else D.random_tree(n, rng, 4) if n else [])
            starts.append(starts[-1] + n)
            drafted += [rng.randrange(alike) + (1 << 40) for _ in range(n)]
            sampled += [rng.randrange(alike) + (1 << 40) for _ in range(n)]
        longest = max(sizes)
        kept, path, behind = accept(starts, drafted, sampled, longest, None if chain else [p for t in trees for p in t])
        for r, n in enumerate(sizes):
            part = slice(starts[r], starts[r + 1])
            ref, last = D.walk(trees[r], drafted[part], sampled[part])
            assert kept[r] == len(ref) and path[r] == ref + [-1] * (longest - len(ref)) and behind[r] == last, r


def test_walks_of_odd_trees():
    """Parents that are no parents, starts that lie."""
    parents = [-1, 5, 1, 0, 2 ** 31 - 1, -2 ** 31, 3, 6]
    drafted, sampled = [1] * 8, [1] * 8
    assert accept([0, 8], drafted, sampled, 8, parents) == ([4], [[0, 3, 6, 7, -1, -1, -1, -1]], [1])
    for starts in ([0, 9], [-1, 8], [5, 3], [0, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1]):
        assert accept(starts, drafted, sampled, 8, parents) == ([0], [[-1] * 8], [-1]), starts
    assert accept([0, 8], drafted, sampled, 7, parents) == ([0], [[-1] * 7], [-1])
    assert accept([0, 0], [], [], 3) == ([0], [[-1] * 3], [-1])


class Batch:
    """Sequences with drafted tokens in a pool, and the host's model of it."""

    def __init__(self, bases, sizes, page, layers=3, heads=2, dim=16, dtype=BF16, order="hnd", seed=0, spare=5, width=None):
        g = torch.Generator().manual_seed(seed)
        self.rng = random.Random(seed)
        self.bases, self.sizes, self.page = bases, sizes, page
        lens = [b + t for b, t in zip(bases, sizes)]
        S, W = len(bases), width or max(1, max(-(-n // page) for n in lens) + 2)
        need = sum(-(-n // page) for n in lens)
        self.model = H.Pages(S, W, need + spare, page)
        self.model.refs[:] = 0
        ids, at = torch.randperm(need + spare, generator=g).tolist(), 0
        for s, n in enumerate(lens):
            c = -(-n // page)
            self.model.table[s, :c] = ids[at:at + c]
            self.model.refs[ids[at:at + c]] = 1
            at += c
            self.model.lengths[s] = n
        shape = (layers, need + spare, heads, page, dim)
        self.k, self.v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
        self.dk, self.dv = (t.cuda() if order == "hnd" else t.transpose(2, 3).contiguous().cuda().transpose(2, 3) for t in (self.k, self.v))
        self.load()

    def load(self):
        self.table, self.lengths, self.refs = (ints(t.tolist()) for t in (self.model.table, self.model.lengths, self.model.refs))
        self.cache, self.pool = cp.paged_cache(self.dk, self.dv), cp.page_pool(self.table, self.lengths, self.page, self.refs)

    def keep(self, paths, seqs=None, starts=None, longest=None, kept=None):
        n = len(paths)
        longest = longest or max(1, max(self.sizes))
        starts = [sum(self.sizes[:i]) for i in range(n + 1)] if starts is None else starts
        status = torch.full((1,), -9, dtype=INT32, device="cuda")
        ws = torch.full((cp.cpes_pages_keep_workspace_bytes(n, longest),), 0xFF, dtype=torch.uint8, device="cuda")
        path = [(p + [-1] * longest)[:longest] for p in paths]
        cp.cpes_pages_keep(self.cache, self.pool, ints(starts), ints([len(p) for p in paths] if kept is None else kept),
                           ints(path).view(n, longest), ws, seqs=None if seqs is None else ints(seqs), status=status)
        return int(status)

    def expect(self, paths, seqs=None, sizes=None):
        m, P = self.model, self.page
        for i, path in enumerate(paths):
            s, T = i if seqs is None else seqs[i], (sizes or self.sizes)[i]
            base = int(m.lengths[s]) - T
            old = -(-int(m.lengths[s]) // P)
            for j, node in enumerate(path):
                a, b = base + node, base + j
                for t in (self.k, self.v):
                    t[:, m.table[s, b // P], :, b % P] = t[:, m.table[s, a // P], :, a % P].clone()
            m.lengths[s] = base + len(path)
            for e in range(-(-int(m.lengths[s]) // P), old):
                m.refs[m.table[s, e]] -= 1
                m.table[s, e] = -1

    def same(self):
        m = self.model
        assert self.lengths.tolist() == m.lengths.tolist() and self.table.tolist() == m.table.tolist() and self.refs.tolist() == m.refs.tolist()
        assert torch.equal(self.dk.cpu(), self.k) and torch.equal(self.dv.cpu(), self.v)


def some_path(rng, n):
    return sorted(rng.sample(range(n), rng.randrange(n + 1))) if n else []


@pytest.mark.parametrize("page", [1, 2, 7, 16, 48])
@pytest.mark.parametrize("order,dtype,dim", [("hnd", BF16, 16), ("nhd", F32, 40), ("hnd", BF16, 128)])
def test_kept_paths(page, order, dtype, dim):
    print(f"keep page={page} {order} {dtype} dim={dim}", flush=True)
    bases, sizes = [0, 1, 15, 16, 33, 47, 5, 100, 64], [1, 9, 16, 40, 3, 17, 0, 64, 5]
    b = Batch(bases, sizes, page, dim=dim, dtype=dtype, order=order, seed=page)
    paths = [some_path(b.rng, n) for n in sizes]
    assert b.keep(paths) == cp.PAGES_OK
    b.expect(paths)
    b.same()
    for paths in ([list(range(n)) for n in sizes], [[] for _ in sizes], [[n - 1] if n else [] for n in sizes]):
        b = Batch(bases, sizes, page, dim=dim, dtype=dtype, order=order, seed=page + 1)
        assert b.keep(paths) == cp.PAGES_OK
        b.expect(paths)
        b.same()


@pytest.mark.parametrize("n", [1, 255, 256, 257, 1030, 2100])
def test_many_sequences(n):
    """On either side of what the plan's threads see at once."""
    rng = random.Random(n)
    bases, sizes = [rng.randrange(20) for _ in range(n)], [rng.randrange(1, 7) for _ in range(n)]
    b = Batch(bases, sizes, 4, layers=2, heads=1, dim=8, seed=n)
    paths = [some_path(b.rng, t) for t in sizes]
    assert b.keep(paths) == cp.PAGES_OK
    b.expect(paths)
    b.same()
    # listed twice, far behind: nothing changes
    if n > 1:
        seqs = list(range(n))
        seqs[-1] = 0
        assert b.keep([[] for _ in range(n)], seqs=seqs, starts=[0] * (n + 1)) == cp.PAGES_BAD_SEQUENCE
        b.same()
        b.lengths[n // 2] = -3
        b.model.lengths[n // 2] = -3
        assert b.keep([[] for _ in range(n)], starts=[0] * (n + 1)) == cp.PAGES_BAD_SEQUENCE
        b.same()


def test_longest_trees():
    b = Batch([3, 60], [256, 200], 16, layers=1, seed=2)
    paths = [sorted(b.rng.sample(range(256), 130)), [199]]
    assert b.keep(paths) == cp.PAGES_OK
    b.expect(paths)
    b.same()


def test_listed_sequences():
    b = Batch([10, 20, 30, 40], [4, 5, 6, 7], 8, seed=3)
    paths, seqs = [[1, 3], [0], [2, 4, 6]], [2, 0, 3]
    sizes = [6, 4, 7]
    assert b.keep(paths, seqs=seqs, starts=[100, 106, 110, 117]) == cp.PAGES_OK
    b.expect(paths, seqs=seqs, sizes=sizes)
    b.same()
    assert b.keep([], starts=[0]) == cp.PAGES_OK          # nobody
    b.same()


def test_refused_steps_change_nothing():
    b = Batch([10, 20, 30], [4, 5, 6], 8, seed=4)
    good = [[0, 2], [1], [0, 1, 5]]
    starts = [0, 4, 9, 15]
    for kw in (dict(seqs=[0, 1, 3]), dict(seqs=[0, -1, 2]), dict(seqs=[0, 1, 1]), dict(starts=[0, 4, 3, 9]), dict(starts=[0, 4, 9, 16]),
               dict(starts=[-2 ** 31, 4, 9, 2 ** 31 - 1]), dict(kept=[2, 1, 7]), dict(kept=[2, -1, 3]), dict(kept=[2, 2 ** 31 - 1, 3]),
               dict(kept=[3, 1, 3]), dict(longest=5)):
        assert b.keep(good, **{"starts": starts, **kw}) == cp.PAGES_BAD_SEQUENCE, kw
        b.same()
    for bad in ([0, 0], [2, 1], [0, 4], [-1, 2], [1, 2 ** 31 - 1]):
        assert b.keep([bad, [1], [0]], starts=starts) == cp.PAGES_BAD_SEQUENCE, bad
        b.same()
    # a sequence shorter than its drafted tokens, and ones beyond their tables
    for length in (3, 0, -4, 8 * b.model.table.shape[1] + 1, 2 ** 31 - 1):
        b.lengths[1] = length
        b.model.lengths[1] = length
        assert b.keep(good, starts=starts) == cp.PAGES_BAD_SEQUENCE, length
        b.same()


def test_entries_without_a_page():
    """Tokens whose entry names no page move nowhere, and no page is given back twice."""
    b = Batch([6, 30], [12, 3], 4, seed=5)
    m = b.model
    for entry, bad in ((2, -1), (4, len(m.refs)), (3, 2 ** 31 - 1)):
        m.refs[m.table[0, entry]] -= 1
        m.table[0, entry] = bad
    b.load()
    path = [[1, 3, 6, 11], [2]]
    status = b.keep(path)
    assert status == cp.PAGES_OK
    refs = b.refs.tolist()
    assert min(refs) >= 0 and b.lengths.tolist() == [10, 31]
    # sequence 0 keeps pages 0 .. 2; of the others one has a page
    assert b.table[0, 3:5].tolist() == [-1, -1]


def test_shared_pages_lose_one_reference():
    """A rollout forked in front of its drafted tokens shares its prompt's pages."""
    b = Batch([16, 16], [5, 6], 8, seed=6)
    b.model.refs[b.model.table[0, 0]] += 1
    b.model.refs[b.model.table[1, 0]] -= 1
    b.model.table[1, 0] = b.model.table[0, 0]
    b.load()
    paths = [[0, 4], []]
    assert b.keep(paths) == cp.PAGES_OK
    b.expect(paths)
    b.same()


def test_captured_walk_and_keep():
    """Both calls in a graph, replayed on other samples and lengths."""
    page, sizes, bases = 8, [9, 12, 1], [20, 3, 50]
    b = Batch(bases, sizes, page, seed=7)
    rng = random.Random(7)
    trees = [D.random_tree(n, rng, 3) for n in sizes]
    starts, longest = [0, 9, 21, 22], 12
    dstarts, parents = ints(starts), ints([p for t in trees for p in t])
    drafted, sampled = (torch.zeros(22, dtype=torch.int64, device="cuda") for _ in range(2))
    kept, path, behind = ints([0] * 3), ints([[0] * longest] * 3), torch.zeros(3, dtype=torch.int64, device="cuda")
    status = ints([0])
    ws = torch.empty(cp.cpes_pages_keep_workspace_bytes(3, longest), dtype=torch.uint8, device="cuda")

    def step():
        cp.cpes_tree_accept(dstarts, drafted, sampled, kept, path, behind, parents=parents)
        cp.cpes_pages_keep(b.cache, b.pool, dstarts, kept, path, ws, status=status)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    b.same()
    before = (b.table.clone(), b.lengths.clone(), b.refs.clone(), b.dk.clone(), b.dv.clone())
    fresh = b
    for turn in range(3):
        for t, x in zip((fresh.table, fresh.lengths, fresh.refs, fresh.dk, fresh.dv), before):
            t.copy_(x)
        model = Batch(bases, sizes, page, seed=7)
        a, c = ([rng.randrange(2) for _ in range(22)] for _ in range(2))
        drafted.copy_(torch.tensor(a))
        sampled.copy_(torch.tensor(c))
        graph.replay()
        torch.cuda.synchronize()
        paths = [D.walk(trees[r], a[starts[r]:starts[r + 1]], c[starts[r]:starts[r + 1]])[0] for r in range(3)]
        assert kept.tolist() == [len(p) for p in paths] and int(status) == 0
        model.expect(paths)
        fresh.model, fresh.k, fresh.v = model.model, model.k, model.v
        fresh.same()


@pytest.mark.parametrize("dtype,window,sinks", [(BF16, 0, 0), (F32, 0, 0), (BF16, 20, 3)])
def test_steps_with_drafts_write_what_single_tokens_write(dtype, window, sinks):
    """Greedy text of a small model (attention, an embedding, a table of logits) by one token a step, and by trees of
    drafted tokens, right and wrong ones: the same tokens, and the same cache."""
    g = torch.Generator().manual_seed(21)
    V, Hq, Hk, dim, L, page, S = 50, 4, 2, 16, 2, 4, 3
    embed = (torch.randn(V, L, Hq + 2 * Hk, dim, generator=g)).to(dtype).cuda()
    head = torch.randn(L * Hq * dim, V, generator=g).cuda()
    prompts = [[3, 1, 4], [1] * 11, [7]]
    steps, longest, rng = 9, 6, random.Random(3)

    class Text:
        def __init__(self):
            pages, width = 80, 12
            self.k, self.v = (torch.zeros(L, pages, Hk, page, dim, dtype=dtype, device="cuda") for _ in range(2))
            self.table = torch.full((S, width), -1, dtype=INT32, device="cuda")
            self.lengths, self.refs = ints([0] * S), ints([0] * pages)
            self.cache, self.pool = cp.paged_cache(self.k, self.v), cp.page_pool(self.table, self.lengths, page, self.refs)
            self.ws = torch.empty(max(cp.cpes_pages_workspace_bytes(pages), cp.cpes_pages_keep_workspace_bytes(S, 64)), dtype=torch.uint8, device="cuda")
            self.status = ints([0])

        def logits(self, trees, tokens):
            """Logits behind each token of each sequence's tree (None: a chain)."""
            sizes = [len(t) for t in tokens]
            starts = [sum(sizes[:i]) for i in range(S + 1)]
            n, most = starts[-1], max(sizes)
            base = self.lengths.tolist()
            cp.cpes_pages_reserve(self.pool, ints(list(range(S))), ints([b + t for b, t in zip(base, sizes)]), self.ws, status=self.status)
            assert int(self.status) == 0
            x = embed[torch.tensor([t for row in tokens for t in row], device="cuda")]
            pos = ints([b + i for b, t in zip(base, sizes) for i in range(t)])
            seqs = ints([s for s, t in enumerate(sizes) for _ in range(t)])
            parents = None if trees is None else ints([p for t in trees for p in t])
            dstarts = ints(starts)
            aws = torch.empty(cp.cpes_attend_tree_workspace_bytes(S, n, most, Hq, Hk, dim), dtype=torch.uint8, device="cuda")
            outs = []
            for layer in range(L):
                out = torch.empty(n, Hq, dim, dtype=dtype, device="cuda")
                cp.cpes_cache_append(self.cache, layer, self.pool, x[:, layer, Hq:Hq + Hk], x[:, layer, Hq + Hk:], pos, seqs=seqs)
                cp.cpes_attend_tree(self.cache, layer, self.pool, x[:, layer, :Hq], out, dstarts, most, parents=parents,
                                    window=window, sinks=sinks, workspace=aws)
                outs.append(out)
            return torch.cat(outs, 1).reshape(n, -1).float() @ head, dstarts, parents

        def sample(self, logits):
            n = len(logits)
            token = torch.empty(n, dtype=torch.int64, device="cuda")
            ws = torch.empty(cp.cpes_sample_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
            cp.cpes_sample(logits, torch.zeros(n, device="cuda"), token, top_k=1, workspace=ws)
            return token

    one = Text()
    logits, starts, _ = one.logits(None, prompts)
    last = one.sample(logits)[starts[1:].long() - 1].tolist()
    written = [[t] for t in last]
    for _ in range(steps - 1):
        logits, _, _ = one.logits(None, [[w[-1]] for w in written])
        for s, t in enumerate(one.sample(logits).tolist()):
            written[s].append(t)
    tree = Text()
    logits, starts, _ = tree.logits(None, prompts)
    last = tree.sample(logits)[starts[1:].long() - 1].tolist()
    text, calls = [[t] for t in last], 0
    while min(len(t) for t in text) < steps:
        trees, drafts = [], []
        for s in range(S):
            # node 0 is the last token; then right guesses, wrong ones, and the right one a second time
            at = len(text[s])
            right = written[s][at:at + 2]
            parents, tokens = [-1], [text[s][-1]]
            for i, t in enumerate(right):
                parents += [len(tokens) - 1 if i == 0 else right_at, len(tokens) - 1 if i == 0 else right_at]
                tokens += [(t + 1) % V, t]
                right_at = len(tokens) - 1
            trees.append(parents[:longest])
            drafts.append(tokens[:longest])
        logits, starts, parents = tree.logits(trees, drafts)
        sampled = tree.sample(logits)
        most = max(len(t) for t in drafts)
        kept, path, behind = ints([0] * S), ints([[0] * most] * S), torch.zeros(S, dtype=torch.int64, device="cuda")
        cp.cpes_tree_accept(starts, torch.tensor([t for d in drafts for t in d], device="cuda"), sampled, kept, path, behind, parents=parents)
        cp.cpes_pages_keep(tree.cache, tree.pool, starts, kept, path, tree.ws, status=tree.status)
        assert int(tree.status) == 0
        for s in range(S):
            text[s] += [drafts[s][i] for i in path[s, 1:int(kept[s])].tolist()] + [int(behind[s])]
        calls += 1
    assert calls <= 5
    for s in range(S):
        assert text[s][:steps] == written[s], s
        # keys and values of the text that both have
        n = min(int(one.lengths[s]), int(tree.lengths[s]))
        for a, b in ((one.k, tree.k), (one.v, tree.v)):
            for j in range(n):
                assert torch.equal(a[:, one.table[s, j // page].long(), :, j % page], b[:, tree.table[s, j // page].long(), :, j % page])
    assert int((tree.refs > 0).sum()) == sum(-(-int(n) // page) for n in tree.lengths)
