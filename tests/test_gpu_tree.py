"""Attention of trees and chains of new tokens over the paged cache against a plain
implementation in 64 bits.  What no token sees -- other slots of pages, positions
outside every window, pages nobody holds -- holds NaN or infinities."""
import math
import random

import pytest
import torch

import draft_helpers as D
import eval_helpers as H
import paper_2608_02391_amd as cp

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


class Trees:
    """Rows of `base` committed tokens and a tree of `sizes` new ones (chain: parents None), in scattered pages."""

    def __init__(self, bases, sizes, kv_heads=2, dim=64, page=16, dtype=BF16, order="hnd", window=0, sinks=0, seed=0,
                 chain=False, width=None, layers=2, layer=1, spread=3):
        g = torch.Generator().manual_seed(seed)
        rng = random.Random(seed)
        self.bases, self.sizes, self.kv, self.dim, self.page, self.dtype, self.layer = bases, sizes, kv_heads, dim, page, dtype, layer
        self.window, self.sinks = window, sinks
        self.lens = [b + t for b, t in zip(bases, sizes)]
        self.trees = [None if chain else D.random_tree(t, rng, spread) if t else [] for t in sizes]
        self.starts = [0]
        for t in sizes:
            self.starts.append(self.starts[-1] + t)
        self.tokens, self.longest = self.starts[-1], max(1, max(sizes))
        counts = [-(-n // page) for n in self.lens]
        self.pages = sum(counts) + 3
        self.width = width or max(1, max(counts) + 1)
        ids = torch.randperm(self.pages, generator=g)
        shape = (layers, self.pages, kv_heads, page, dim)
        poison = torch.tensor([math.nan, math.inf, -math.inf, 3e38])
        host = []
        for _ in range(2):
            t = torch.empty(shape, dtype=dtype) if order == "hnd" else torch.empty(layers, self.pages, page, kv_heads, dim, dtype=dtype).transpose(2, 3)
            t.copy_(poison[torch.randint(0, 4, shape, generator=g)].to(dtype))
            host.append(t)
        self.table = torch.full((len(bases), self.width), -1, dtype=torch.int32)
        self.keys, self.values, self.seen, at = [], [], [], 0
        for s, n in enumerate(self.lens):
            own = ids[at:at + counts[s]]
            at += counts[s]
            self.table[s, :counts[s]] = own.int()
            k, v = (torch.randn(n, kv_heads, dim, generator=g).to(dtype) for _ in range(2))
            seen = [D.seen_by(self.trees[s], i, bases[s], n, window, sinks) for i in range(sizes[s])]
            j = torch.arange(n)[torch.stack(seen).any(0)] if seen else torch.arange(0)
            for t, x in zip(host, (k, v)):
                t[layer][own[j // page], :, j % page] = x[j]
            self.keys.append(k)
            self.values.append(v)
            self.seen.append(seen)
        self.k, self.v = (t.cuda() if order == "hnd" else t.transpose(2, 3).contiguous().cuda().transpose(2, 3) for t in host)
        self.lengths = torch.tensor(self.lens, dtype=torch.int32)
        self.parents = None if chain else torch.tensor([p for t in self.trees for p in t], dtype=torch.int32)
        self.bind()

    def bind(self):
        self.cache = cp.paged_cache(self.k, self.v)
        self.dtable, self.dlengths = self.table.cuda(), self.lengths.cuda()
        self.pool = cp.page_pool(self.dtable, self.dlengths, self.page)

    def queries(self, q_heads, seed=1):
        g = torch.Generator().manual_seed(seed)
        return (torch.randn(self.tokens, q_heads, self.dim, generator=g) * 2).to(self.dtype)

    def run(self, q, out=None, starts=None, parents="own", seqs=None, longest=None, stream=None, lse=True, scale=None):
        heads, tokens = q.shape[1], q.shape[0]
        starts = torch.tensor(self.starts if starts is None else starts, dtype=torch.int32, device="cuda")
        parents = self.parents if isinstance(parents, str) else parents
        longest = longest or self.longest
        nbytes = cp.cpes_attend_tree_workspace_bytes(starts.numel() - 1, tokens, longest, heads, self.kv, self.dim)
        ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda")
        out = torch.full(q.shape, math.nan, dtype=self.dtype, device="cuda") if out is None else out
        dl = torch.full((tokens, heads), math.nan, device="cuda") if lse else None
        cp.cpes_attend_tree(self.cache, self.layer, self.pool, q if q.is_cuda else q.cuda(), out, starts, longest,
                            parents=None if parents is None else parents.cuda(), lse=dl, seqs=None if seqs is None else seqs.cuda(),
                            scale=scale, window=self.window, sinks=self.sinks, workspace=ws, stream=stream)
        return out, dl

    def check(self, q, out, lse, rows=None, skip=()):
        """rows: those looked at; skip: (row, token) pairs that are not."""
        out, lse, group = out.float().cpu(), lse.cpu(), q.shape[1] // self.kv
        for r in range(len(self.bases)) if rows is None else rows:
            for i in range(self.sizes[r]):
                if (r, i) in skip:
                    continue
                at = self.starts[r] + i
                for h in range(q.shape[1]):
                    k, v = self.keys[r][:, h // group], self.values[r][:, h // group]
                    ref, ref_lse, tol, tol_lse = H.attend(q[at, h].cpu(), k, v, self.seen[r][i], self.dim ** -0.5)
                    got = out[at, h].double()
                    assert torch.isfinite(got).all(), (r, i, h)
                    off = (got - ref).abs() - (tol + H.rounding(self.dtype) * (ref.abs() + tol) + 1e-38)
                    assert float(off.max()) <= 0, (r, i, h, float(off.max()), float((got - ref).abs().max()))
                    assert abs(float(lse[at, h]) - ref_lse) <= tol_lse, (r, i, h, float(lse[at, h]), ref_lse)


BASES = [0, 1, 15, 16, 31, 33, 64, 257, 600]
SIZES = [1, 3, 7, 2, 16, 5, 12, 9, 4]


@pytest.mark.parametrize("chain", [False, True], ids=["tree", "chain"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dim,page", [(8, 16), (40, 7), (64, 16), (80, 16), (128, 16), (128, 7), (136, 16), (256, 24), (256, 32)])
def test_head_dims(dtype, dim, page, chain):
    print(f"tree dim={dim} page={page} {dtype} chain={chain}", flush=True)
    c = Trees(BASES, SIZES, dim=dim, page=page, dtype=dtype, seed=dim, chain=chain)
    q = c.queries(4)
    c.check(q, *c.run(q))


@pytest.mark.parametrize("page", [1, 2, 8, 16, 48, 100])
@pytest.mark.parametrize("order", ["hnd", "nhd"])
def test_page_sizes(page, order):
    print(f"tree page={page} {order}", flush=True)
    c = Trees(BASES, SIZES, page=page, order=order, seed=page)
    q = c.queries(8)
    c.check(q, *c.run(q))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("page", [96, 128, 1000])
def test_large_pages(page, dtype):
    """Pages of several tiles, and of more tokens than any row has."""
    print(f"tree page={page} {dtype}", flush=True)
    c = Trees(BASES, SIZES, page=page, dtype=dtype, seed=page)
    q = c.queries(8)
    c.check(q, *c.run(q))


@pytest.mark.parametrize("kv,group", [(1, 1), (3, 1), (2, 5), (1, 16), (2, 17), (1, 33), (1, 70), (1, 300)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_head_groups(kv, group, dtype):
    """From one query a row to several blocks of a key-value head's query heads."""
    print(f"tree kv={kv} group={group} {dtype}", flush=True)
    c = Trees([1, 33, 0, 95], [3, 1, 6, 2], kv_heads=kv, dim=128, dtype=dtype, seed=group)
    q = c.queries(kv * group)
    c.check(q, *c.run(q))


@pytest.mark.parametrize("nodes", [1, 2, 4, 5, 8, 9, 16, 17, 31, 32, 33, 40, 63, 64, 65, 130, 256])
@pytest.mark.parametrize("dtype,dim,page", [(BF16, 64, 16), (F32, 64, 5), (BF16, 136, 16)])
def test_tree_sizes(nodes, dtype, dim, page):
    """On either side of what a wave, a workgroup and a word of ancestors hold; bushy and deep."""
    print(f"tree nodes={nodes} {dtype} dim={dim}", flush=True)
    c = Trees([0, 45, 130], [nodes, max(1, nodes // 2), 1], kv_heads=1, dim=dim, page=page, dtype=dtype, seed=nodes, spread=nodes if nodes % 2 else 2)
    q = c.queries(4)
    c.check(q, *c.run(q))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (4, 0), (16, 4), (33, 0), (100, 37), (64, 200), (5000, 4), (300, 31)])
@pytest.mark.parametrize("dtype,page,chain", [(BF16, 16, False), (F32, 24, False), (BF16, 5, True), (F32, 16, True)])
def test_windows_and_sinks(window, sinks, dtype, page, chain):
    print(f"tree window={window} sinks={sinks} {dtype} page={page} chain={chain}", flush=True)
    c = Trees([0, 1, 2, 17, 36, 101, 333, 900], [20, 3, 40, 9, 1, 33, 12, 64], kv_heads=1, page=page, dtype=dtype, window=window,
              sinks=sinks, seed=window, chain=chain)
    q = c.queries(4)
    c.check(q, *c.run(q))


@pytest.mark.parametrize("bases,sizes", [([20000], [6]), ([3] * 200, [2] * 200), ([9000, 1, 0, 5000], [30, 1, 64, 2]),
                                         ([6000] * 3 + [100] * 50, [8] * 53), ([7000], [200])],
                         ids=["one_long", "many_short", "mixed", "few_long", "wide"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_splits(bases, sizes, dtype):
    """Long rows over many workgroups, many rows in one, and mixtures."""
    print(f"tree bases={bases[:4]} sizes={sizes[:4]} {dtype}", flush=True)
    c = Trees(bases, sizes, kv_heads=1, dtype=dtype, layers=1, layer=0, seed=len(bases))
    q = c.queries(2)
    c.check(q, *c.run(q))


@pytest.mark.parametrize("dtype,dim,group", [(BF16, 128, 4), (BF16, 64, 1), (F32, 64, 4), (BF16, 256, 2)])
def test_prompts(dtype, dim, group):
    """Chains of many pieces from an empty cache, and behind one: a query in every few tokens is looked at."""
    print(f"prompts {dtype} dim={dim} group={group}", flush=True)
    c = Trees([0, 100, 0, 30], [1500, 700, 1, 333], kv_heads=2, dim=dim, dtype=dtype, chain=True, seed=dim)
    q = c.queries(2 * group)
    out, lse = c.run(q)
    c.check(q, out, lse, skip={(r, i) for r in range(4) for i in range(c.sizes[r]) if i % 61 and i != c.sizes[r] - 1})


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes", [10, 25, 50, 75])
@pytest.mark.parametrize("chain", [False, True], ids=["tree", "chain"])
def test_many_queries_over_long_contexts(dim, nodes, chain):
    """40 to 300 queries a KV head, on contexts that several workgroups share; rows with fewer, and a window."""
    print(f"tree shares dim={dim} nodes={nodes} chain={chain}", flush=True)
    for window, sinks in ((0, 0), (2500, 70)):
        c = Trees([5000, 40, 2911], [nodes, nodes // 3, 1 + nodes // 2], dim=dim, chain=chain, window=window, sinks=sinks, seed=nodes)
        q = c.queries(8)
        out, lse = c.run(q)
        skip = {(r, i) for r in range(3) for i in range(c.sizes[r]) if i % 7 and i != c.sizes[r] - 1}
        c.check(q, out, lse, skip=skip)
        again, again_lse = c.run(q)
        assert torch.equal(again, out) and torch.equal(again_lse, lse)


def check_scaled(c, q, scale, step=1):
    scale = float(torch.tensor(scale, dtype=torch.float32))
    out, lse = c.run(q, scale=scale)
    out, lse, group = out.double().cpu(), lse.cpu(), q.shape[1] // c.kv
    for r in range(len(c.bases)):
        for i in range(0, c.sizes[r], step):
            at = c.starts[r] + i
            for h in range(q.shape[1]):
                ref, ref_lse, tol, tol_lse = H.attend(q[at, h].cpu(), c.keys[r][:, h // group], c.values[r][:, h // group], c.seen[r][i], scale)
                off = (out[at, h] - ref).abs() - (tol + H.rounding(c.dtype) * (ref.abs() + tol) + 1e-38)
                assert float(off.max()) <= 0, (r, i, h, scale, float(off.max()))
                assert abs(float(lse[at, h]) - ref_lse) <= tol_lse, (r, i, h, scale, float(lse[at, h]), ref_lse)


@pytest.mark.parametrize("scale", [-0.125, 0.0, -0.0, 1e-40, 1e-6, 1.0, -3.0])
@pytest.mark.parametrize("dtype,dim,heads", [(BF16, 64, 1), (BF16, 64, 8), (BF16, 128, 32), (F32, 64, 4)])
def test_scales(dtype, dim, heads, scale):
    """Of either sign, none at all, and so small or large that all or one of the positions count."""
    print(f"tree scale={scale} {dtype} dim={dim} heads={heads}", flush=True)
    for bases, sizes, chain in (([0, 77, 3000], [5, 12, 1], False), ([4500], [9], False), ([20], [60], True)):
        c = Trees(bases, sizes, kv_heads=1, dim=dim, dtype=dtype, seed=dim + heads, chain=chain)
        check_scaled(c, c.queries(heads), scale, 1 if heads < 32 and max(sizes) < 60 else 5)


@pytest.mark.parametrize("dtype,heads", [(BF16, 1), (BF16, 8), (F32, 4)])
@pytest.mark.parametrize("scale", [2.0 ** 60, -(2.0 ** 101), 2.0 ** 127, 3e38, -3e38])
def test_scales_near_the_largest_number(scale, dtype, heads):
    """Scores that are ordinary numbers behind a scale whose product with log2 e may not be one."""
    print(f"tree scale={scale} {dtype} heads={heads}", flush=True)
    for bases, sizes in (([0, 77, 1000], [5, 12, 1]), ([2500], [9])):
        c = Trees(bases, sizes, kv_heads=1, dtype=dtype, seed=heads)
        q = c.queries(heads).float()
        # one product a score, of numbers that have all their bits
        q[..., 1:] = 0.0
        q[..., 0] = (1.0 + q[..., 0].abs()) * 2.0 ** -math.floor(math.log2(abs(scale))) * q[..., 0].sign()
        check_scaled(c, q.to(dtype), scale)


def test_one_new_token_is_the_decode_attention():
    """Trees of one token: the same positions as cpes_attend, the same bounds; and a chain in two calls is one call's."""
    c = Trees([0, 40, 333, 2000], [1, 1, 1, 1], dim=128, seed=3)
    q = c.queries(8)
    out, lse = c.run(q)
    c.check(q, out, lse)
    ws = torch.empty(cp.cpes_attend_workspace_bytes(4, 8, 2, 128), dtype=torch.uint8, device="cuda")
    one, one_lse = torch.empty_like(out), torch.empty_like(lse)
    cp.cpes_attend(c.cache, 1, c.pool, q.cuda(), one, lse=one_lse, workspace=ws)
    c.check(q, one, one_lse)
    # two roundings of nearly the same number
    assert float((one.float() - out.float()).abs().max()) <= 2 * 2.0 ** -8 * float(one.float().abs().max())


def test_no_parents_is_a_chain():
    c = Trees([50, 7], [20, 33], chain=True, seed=8)
    q = c.queries(4)
    out, lse = c.run(q)
    c.check(q, out, lse)
    line = torch.tensor(list(range(-1, 19)) + list(range(-1, 32)), dtype=torch.int32)
    again, again_lse = c.run(q, parents=line)
    c.check(q, again, again_lse)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("base", [0, 13, 3000])
def test_a_broken_branch_stays_its_own(dtype, bad, base):
    """Keys and values of some tokens are NaN or infinite: whoever does not descend from them is not touched."""
    print(f"broken branch {dtype} {bad} base={base}", flush=True)
    for where in ("k", "v", "kv"):
        c = Trees([base, 5], [40, 9], dtype=dtype, seed=11, kv_heads=1)
        hurt = {(0, 7), (0, 8), (0, 23), (0, 39), (1, 4)}
        for r, i in hurt:
            pos = c.bases[r] + i
            page, slot = int(c.table[r, pos // 16]), pos % 16
            for t, name in ((c.k, "k"), (c.v, "v")):
                if name in where:
                    t[1, page, 0, slot, 3] = bad
        q = c.queries(4)
        out, lse = c.run(q)
        sees = {(r, i) for r in range(2) for i in range(c.sizes[r]) if any((r, j) in hurt for j in D.branch(c.trees[r], i))}
        assert len(sees) < 30
        c.check(q, out, lse, skip=sees)
    c = Trees([base], [12], dtype=dtype, seed=12, kv_heads=1, chain=True)
    pos = base + 6
    c.v[1, int(c.table[0, pos // 16]), 0, pos % 16] = bad
    q = c.queries(4)
    out, lse = c.run(q)
    c.check(q, out, lse, skip={(0, i) for i in range(6, 12)})
    assert not bool(torch.isfinite(out[6:].float()).all(-1).any())


def expect_infinities(c, q, out, lse, rows, step=1):
    """What is promised where values that are seen are not finite: a dim that sees an infinity is that or, of a bf16 cache,
    NaN; one that sees a NaN or both signs is NaN; the others and the lse are as ever."""
    out, lse, group, hit = out.float().cpu(), lse.cpu(), q.shape[1] // c.kv, [0, 0]
    for r in rows:
        for i in range(0, c.sizes[r], step):
            at = c.starts[r] + i
            for h in range(q.shape[1]):
                k, v, seen = c.keys[r][:, h // group], c.values[r][:, h // group].double(), c.seen[r][i]
                finite = torch.where(torch.isfinite(v), v, 0.0)
                ref, ref_lse, tol, tol_lse = H.attend(q[at, h].cpu(), k, finite, seen, c.dim ** -0.5)
                lost = torch.where(torch.isfinite(v) | ~seen[:len(v), None], 0.0, v).sum(0)
                got = out[at, h].double()
                odd = lost != 0
                infinite = odd & ~lost.isnan()
                as_promised = got[infinite] == lost[infinite]
                if c.dtype == BF16:
                    as_promised |= got[infinite].isnan()
                assert bool(as_promised.all()), (r, i, h)
                assert bool(got[lost.isnan()].isnan().all()), (r, i, h)
                off = (got - ref).abs() - (tol + H.rounding(c.dtype) * (ref.abs() + tol) + 1e-38)
                assert not bool((off[~odd] > 0).any()) and bool(torch.isfinite(got[~odd]).all()), (r, i, h)
                assert abs(float(lse[at, h]) - ref_lse) <= tol_lse, (r, i, h)
                hit[0] += int(odd.sum())
                hit[1] += int(lost.isnan().sum())
    return hit


@pytest.mark.parametrize("dtype,dim,page", [(BF16, 64, 16), (BF16, 128, 16), (BF16, 128, 5), (BF16, 200, 16), (F32, 64, 16)])
@pytest.mark.parametrize("heads", [1, 3, 8])
def test_values_that_are_not_finite_and_seen(heads, dtype, dim, page):
    """Infinities and NaN in the context and among the new tokens, in tiles that all see and in others, with one query a wave
    or hundreds a workgroup, in one share or several: they stay in their dims."""
    print(f"tree infinities {dtype} dim={dim} page={page} heads={heads}", flush=True)
    for bases, sizes, chain in (([0, 40, 700, 5000], [9, 24, 2, 1], False), ([6000, 130], [70, 3], False), ([300, 0], [90, 33], True)):
        c = Trees(bases, sizes, dim=dim, page=page, dtype=dtype, seed=dim + heads, chain=chain)
        g = random.Random(heads)
        for r, n in enumerate(c.lens):
            for bad, d in ((math.inf, 3), (-math.inf, 17), (math.inf, 40), (-math.inf, 40), (math.nan, dim - 1)):
                pos = g.randrange(n) if d != 3 else max(0, c.bases[r] - 1)
                for kv in range(2):
                    c.values[r][pos, kv, d] = bad
                    c.v[1, int(c.table[r, pos // page]), kv, pos % page, d] = bad
        q = c.queries(2 * heads) / 4
        out, lse = c.run(q)
        hit = expect_infinities(c, q, out, lse, range(len(bases)), 1 if max(sizes) < 60 else 9)
        assert hit[0] > hit[1] > 0
        again, again_lse = c.run(q)
        assert torch.equal(again.isnan(), out.isnan()) and torch.equal(again.nan_to_num(), out.nan_to_num()) and torch.equal(again_lse, lse)


def test_rows_that_do_not_fit():
    """Sequences without their tokens, unknown ids, starts that lie: zeros or nothing, and the others as ever."""
    c = Trees([60, 0, 100, 20], [5, 6, 7, 8], seed=13)
    q = c.queries(4)
    c.lengths = torch.tensor([65, 5, 107, 28], dtype=torch.int32)          # the second lacks one
    c.bind()
    out, lse = c.run(q)
    c.check(q, out, lse, rows=[0, 2, 3])
    assert not bool(out[5:11].any()) and bool((lse[5:11] == -math.inf).all())
    for bad in (-1, 4, 2 ** 31 - 1):
        out, lse = c.run(q, seqs=torch.tensor([0, bad, 2, 3], dtype=torch.int32))
        c.check(q, out, lse, rows=[0, 2, 3])
        assert not bool(out[5:11].any()) and bool((lse[5:11] == -math.inf).all())
    # a row longer than allowed is left out, and what no row covers is left alone
    c = Trees([60, 3, 100], [5, 6, 7], seed=13)
    q = c.queries(4)
    out, lse = c.run(q, longest=6)
    c.check(q, out, lse, rows=[0, 1])
    assert bool(torch.isnan(out[11:]).all()) and bool(torch.isnan(lse[11:]).all())
    # the other rows stay where they are
    out, lse = c.run(q, starts=[0, 5, 11, 11])
    c.check(q, out, lse, rows=[0, 1])
    assert bool(torch.isnan(out[11:]).all())
    for starts in ([0, 5, 11, 19], [0, 5, 11, 2 ** 31 - 1], [0, 5, 11, 10]):
        out, lse = c.run(q, starts=starts)
        c.check(q, out, lse, rows=[0, 1])
        assert bool(torch.isnan(out[11:]).all())
    out, lse = c.run(q, starts=[-5, 5, 11, 18])
    c.check(q, out, lse, rows=[1, 2])
    assert bool(torch.isnan(out[:5]).all())


def test_rows_without_tokens_and_odd_parents():
    c = Trees([0, 60, 7, 9, 30], [0, 5, 0, 12, 0], seed=14)
    q = c.queries(4)
    c.check(q, *c.run(q))
    # parents that are not before their child count as none
    lies = c.parents.clone()
    c.trees[3][4] = c.trees[3][9] = c.trees[3][11] = -1
    lies[5 + 4], lies[5 + 9], lies[5 + 11] = 4, 2 ** 31 - 1, -2 ** 31
    c.seen[3] = [D.seen_by(c.trees[3], i, 9, 21, 0, 0) for i in range(12)]
    c.check(q, *c.run(q, parents=lies))


def test_positions_without_a_page_are_not_seen():
    c = Trees([200, 90], [12, 5], seed=15)
    for r, entry, bad in ((0, 2, -1), (0, 12, c.pages), (1, 0, 2 ** 31 - 1)):
        c.table[r, entry] = bad
        for s in c.seen[r]:
            s[16 * entry:16 * entry + 16] = False
    c.bind()
    q = c.queries(4)
    out, lse = c.run(q)
    # tokens whose own page is missing may see nothing of the tree, but the context
    c.check(q, out, lse)
    c.table[1, :] = -1
    c.bind()
    out, lse = c.run(q)
    c.check(q, out, lse, rows=[0])
    assert not bool(out[12:].any()) and bool((lse[12:] == -math.inf).all())


def test_strides_alignment_and_order():
    """Queries and outputs inside wider tensors at odd elements; sequences in any order, twice."""
    c = Trees([50, 700, 3], [7, 20, 1], seed=16)
    starts, order = [0, 20, 27, 28, 48], [1, 0, 2, 1]
    parents = torch.tensor(c.trees[1] + c.trees[0] + c.trees[2] + c.trees[1], dtype=torch.int32)
    g = torch.Generator().manual_seed(2)
    fused = torch.randn(48 * 8 * 66 + 1, generator=g).to(BF16).cuda()[1:].view(48, 8, 66)
    wide = torch.full((48 * 9 * 71 + 3,), math.nan, dtype=BF16, device="cuda")[3:].view(48, 9, 71)
    q, out = fused[:, 1:5, 1:65], wide[:, 2:6, 3:67]
    _, lse = c.run(q, out=out, starts=starts, parents=parents, seqs=torch.tensor(order, dtype=torch.int32))
    plain = Trees([50, 700, 3], [7, 20, 1], seed=16)
    for r, s in enumerate(order):
        part = slice(starts[r], starts[r + 1])
        plain.starts = [0, 0, 0]
        plain.check(q[part], out[part], lse[part], rows=[s])
    rest = wide.clone()
    rest[:, 2:6, 3:67] = math.nan
    assert bool(torch.isnan(rest).all())
    again = torch.empty(48, 4, 64, dtype=BF16, device="cuda")
    c.run(q, out=again, starts=starts, parents=parents, seqs=torch.tensor(order, dtype=torch.int32), lse=False)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dim,extra,first", [(64, 1, 1), (128, 4, 0), (128, 8, 4), (72, 0, 8)])
def test_caches_at_any_alignment(dim, extra, first):
    """Keys and values whose rows, or whose first element, do not lie at multiples of 16 bytes."""
    print(f"tree cache dim={dim} rows {extra} apart, first at {first}", flush=True)
    for sizes in ([5, 8], [20, 13], [60, 33]):
        c = Trees([50, 300], sizes, dim=dim, seed=dim + extra)
        q = c.queries(8)
        for name in ("k", "v"):
            t = getattr(c, name)
            room = torch.full((t.numel() // dim * (dim + extra) + first + dim,), math.nan, dtype=BF16, device="cuda")
            moved = room[first:first + t.numel() // dim * (dim + extra)].view(*t.shape[:-1], dim + extra)[..., :dim]
            moved.copy_(t)
            setattr(c, name, moved)
        c.bind()
        c.check(q, *c.run(q))


def test_captured_step_follows_lengths_and_trees():
    """A captured call reads lengths, starts and parents when it is replayed."""
    c = Trees([30, 2500], [9, 24], seed=17)
    q = c.queries(4).cuda()
    starts = torch.tensor(c.starts, dtype=torch.int32, device="cuda")
    parents = c.parents.cuda()
    ws = torch.empty(cp.cpes_attend_tree_workspace_bytes(2, 33, 24, 4, 2, 64), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(33, 4, device="cuda")

    def call(o, l):
        cp.cpes_attend_tree(c.cache, 1, c.pool, q, o, starts, 24, parents=parents, lse=l, workspace=ws)

    call(out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse)
    for turn in range(4):
        if turn == 1:
            parents.copy_(torch.tensor([-1] + [0] * 8 + [-1] + [0] * 23, dtype=torch.int32))
        if turn == 2:
            starts.copy_(torch.tensor([0, 4, 20], dtype=torch.int32))
        if turn == 3:
            c.dlengths.copy_(torch.tensor([20, 1000], dtype=torch.int32))
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager, eager_lse = torch.zeros_like(out), torch.zeros_like(lse)
        call(eager, eager_lse)
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse), turn


def test_runs_agree_and_streams_are_respected():
    c = Trees([5000, 12, 700], [24, 3, 60], seed=18, kv_heads=1)
    q = c.queries(4).cuda()
    first, first_lse = c.run(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            out, lse = c.run(q, stream=side)
            side.synchronize()
            assert torch.equal(out, first) and torch.equal(lse, first_lse)


def test_large_caches():
    """Offsets beyond 2^32 bytes and 2^31 elements."""
    pages = 40000                          # of 16 tokens x 2 heads x 128 in 1 layer: 2.6 G elements of keys
    k = torch.zeros(1, pages, 2, 16, 2048 // 1, dtype=BF16, device="cuda")[..., :128]
    v = torch.zeros(1, pages, 2, 16, 2048, dtype=BF16, device="cuda")[..., :128]
    g = torch.Generator().manual_seed(19)
    far = [pages - 1, pages - 7, 3, pages - 100]
    own = torch.randn(2, 4, 2, 16, 128, generator=g).to(BF16)
    for i, p in enumerate(far):
        k[0, p], v[0, p] = own[0, i].cuda(), own[1, i].cuda()
    table = torch.tensor([far], dtype=torch.int32, device="cuda")
    cache, pool = cp.paged_cache(k, v), cp.page_pool(table, torch.tensor([60], dtype=torch.int32, device="cuda"), 16)
    q = torch.randn(5, 4, 128, generator=g).to(BF16)
    out, lse = torch.empty(5, 4, 128, dtype=BF16, device="cuda"), torch.empty(5, 4, device="cuda")
    ws = torch.empty(cp.cpes_attend_tree_workspace_bytes(1, 5, 5, 4, 2, 128), dtype=torch.uint8, device="cuda")
    tree = [-1, 0, 0, 1, 1]
    cp.cpes_attend_tree(cache, 0, pool, q.cuda(), out, torch.tensor([0, 5], dtype=torch.int32, device="cuda"), 5,
                        parents=torch.tensor(tree, dtype=torch.int32, device="cuda"), lse=lse, workspace=ws)
    keys, values = (own[x].permute(1, 0, 2, 3).reshape(2, 64, 128)[:, :60] for x in range(2))
    for i in range(5):
        seen = D.seen_by(tree, i, 55, 60, 0, 0)
        for h in range(4):
            ref, ref_lse, tol, tol_lse = H.attend(q[i, h], keys[h // 2], values[h // 2], seen, 128 ** -0.5)
            off = (out[i, h].double().cpu() - ref).abs() - (tol + 2.0 ** -8 * (ref.abs() + tol))
            assert float(off.max()) <= 0 and abs(float(lse[i, h]) - ref_lse) <= tol_lse
