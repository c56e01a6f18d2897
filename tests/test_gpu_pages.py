"""Pages of the key-value cache -- reserving, forking, freeing, copying and
compacting -- against a plain model on the host: tables, lengths and reference
counts exactly, page contents bit for bit."""
import numpy as np
import pytest
import torch

import eval_helpers as H
import paper_2608_02391_amd as cp

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Rig:
    def __init__(self, sequences, width, pages, page_size, layers=2, heads=2, dim=8, dtype=torch.bfloat16, order="hnd", seed=0):
        self.m = H.Pages(sequences, width, pages, page_size)
        g = torch.Generator(device="cuda").manual_seed(seed)
        shape = (layers, pages, page_size, heads, dim) if order == "nhd" else (layers, pages, heads, page_size, dim)
        self.k, self.v = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
        if order == "nhd":
            self.k, self.v = self.k.transpose(2, 3), self.v.transpose(2, 3)
        if order == "apart":       # heads, tokens and layers with gaps, keys beside values
            both = torch.randn(pages, layers, heads + 1, page_size + 2, 2, dim, generator=g, device="cuda").to(dtype)
            self.k, self.v = (both[:, :, :heads, :page_size, i].transpose(0, 1) for i in range(2))
        self.k0, self.v0 = self.k.clone(), self.v.clone()
        self.table = torch.full((sequences, width), -1, dtype=torch.int32, device="cuda")
        self.lengths, self.refs = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (sequences, pages))
        self.cache = cp.paged_cache(self.k, self.v)
        self.pool = cp.page_pool(self.table, self.lengths, page_size, self.refs)
        self.ws = torch.full((cp.cpes_pages_workspace_bytes(pages),), 0xAA, dtype=torch.uint8, device="cuda")
        self.status = ints([9])

    def same(self, status=0):
        assert int(self.status) == status
        assert np.array_equal(self.lengths.cpu().numpy(), self.m.lengths)
        assert np.array_equal(self.refs.cpu().numpy(), self.m.refs)
        t = self.table.cpu().numpy()
        for s, row in enumerate(self.m.held()):
            assert list(t[s, :len(row)]) == row, s
        for a, b in ((self.k, self.k0), (self.v, self.v0)):
            assert torch.equal(a, b)

    def reserve(self, seqs, new):
        cp.cpes_pages_reserve(self.pool, ints(seqs), ints(new), self.ws, status=self.status)
        self.same(self.m.reserve(seqs, new))

    def fork(self, parents, children):
        cp.cpes_pages_fork(self.cache, self.pool, ints(parents), ints(children), self.ws, status=self.status)
        status, copies = self.m.fork(parents, children)
        for a, b in copies:
            self.k0[:, b], self.v0[:, b] = self.k0[:, a], self.v0[:, a]
        self.same(status)

    def free(self, seqs):
        cp.cpes_pages_free(self.pool, ints(seqs), status=self.status)
        self.same(self.m.free(seqs))

    def compact(self):
        moved = ints([-1])
        cp.cpes_pages_compact(self.cache, self.pool, self.pool, self.ws, moved=moved)
        pairs = self.m.compact()
        for a, b in pairs:
            self.k0[:, b], self.v0[:, b] = self.k0[:, a], self.v0[:, a]
        assert int(moved) == len(pairs)
        self.status.fill_(0)
        self.same()


@pytest.mark.parametrize("order", ["hnd", "nhd", "apart"])
@pytest.mark.parametrize("page_size,dim,dtype", [(16, 64, torch.bfloat16), (1, 8, torch.bfloat16), (5, 40, torch.float32)])
def test_life_of_a_batch(order, page_size, dim, dtype):
    """Prompts reserved and forked, rollouts that grow one token at a time, some
    freed, compaction, more rollouts."""
    print(f"batch {order} page={page_size} dim={dim} {dtype}", flush=True)
    r = Rig(12, 40, 160, page_size, dim=dim, dtype=dtype, order=order)
    P = page_size
    r.reserve([0, 5], [3 * P + (P > 1), 2 * P])
    r.fork([0, 0, 5, 0, 5], [1, 2, 6, 3, 7])
    for t in range(1, 2 * P + 2):
        live = [1, 2, 3, 6, 7]
        r.reserve(live, [int(r.m.lengths[s]) + 1 for s in live])
    r.free([0, 2, 6])
    r.compact()
    r.fork([7, 1], [0, 2])
    r.free([1, 7, 3])
    r.compact()
    r.reserve([9, 8], [10 * P, 7])
    r.free(list(range(12)))
    assert int(r.refs.abs().sum()) == 0
    r.compact()


def test_random_life():
    rng = np.random.default_rng(4)
    r = Rig(40, 30, 300, 4, layers=1, heads=1, dim=8)
    for step in range(120):
        op = rng.integers(0, 5)
        empty = [s for s in range(40) if r.m.lengths[s] == 0]
        full = [s for s in range(40) if r.m.lengths[s] > 0]
        if op <= 1:
            n = int(rng.integers(0, 8))
            seqs = [int(s) for s in rng.permutation(40)[:n]]
            r.reserve(seqs, [int(rng.integers(0, 121)) for _ in seqs])
        elif op == 2 and empty and full:
            kids = [int(s) for s in rng.permutation(empty)[:int(rng.integers(1, 6))]]
            r.fork([int(rng.choice(full)) for _ in kids], kids)
        elif op == 3:
            r.free([int(s) for s in rng.permutation(40)[:int(rng.integers(0, 6))]])
        else:
            r.compact()


def test_all_or_nothing():
    r = Rig(6, 10, 20, 4)
    r.reserve([0, 1], [40, 17])                       # 10 + 5 pages of 20
    r.reserve([2, 3], [12, 12])                       # 6 more: too few, nothing changes
    assert int(r.status) == cp.PAGES_SHORT
    r.reserve([2, 3], [12, 8])                        # exactly what is left
    r.fork([1], [4])                                  # a partial page, and none left
    assert int(r.status) == cp.PAGES_SHORT
    r.fork([0], [4])                                  # full pages only: nothing to copy
    assert int(r.status) == cp.PAGES_OK
    for seqs, new in (([1, 1], [18, 18]), ([6], [1]), ([-1], [1]), ([1, 5], [18, 41]), ([1], [-1])):
        r.reserve(seqs, new)
        assert int(r.status) == cp.PAGES_BAD_SEQUENCE
    for parents, children in (([0], [1]), ([0, 0], [5, 5]), ([6], [5]), ([0], [6]), ([0, 1], [5, -1])):
        r.fork(parents, children)
        assert int(r.status) == cp.PAGES_BAD_SEQUENCE
    r.fork([5], [5])                                  # an empty sequence from itself
    assert int(r.status) == cp.PAGES_OK
    r.reserve([1, 0], [3, 40])                        # not above the present lengths
    assert int(r.status) == cp.PAGES_OK
    r.free([2, 2, 7])                                 # twice is once; 7 does not exist
    assert int(r.status) == cp.PAGES_BAD_SEQUENCE
    for call in (lambda: r.reserve([], []), lambda: r.fork([], []), lambda: r.free([])):
        call()
        assert int(r.status) == cp.PAGES_OK


def test_many_pages_and_sequences():
    """More pages and sequences than one step of the bookkeeping takes."""
    r = Rig(2600, 40, 40000, 2, layers=1, heads=1, dim=8)
    everyone = list(range(2500))
    r.reserve(everyone, [1 + (s * 7) % 20 for s in everyone])
    r.reserve([2599, 2598], [80, 79])
    rng = np.random.default_rng(1)
    r.free([int(s) for s in rng.permutation(2500)[:1400]])
    live = [s for s in everyone if r.m.lengths[s] > 0]
    empty = [s for s in everyone if r.m.lengths[s] == 0]
    r.fork([live[i % len(live)] for i in range(1200)], empty[:1200])
    r.free(live[::2])
    r.compact()
    r.reserve(everyone, [40] * 2500)


def test_compact_into_another_pool():
    r = Rig(5, 6, 50, 4)
    r.reserve([0, 1, 2, 3], [24, 9, 13, 20])
    r.fork([1], [4])
    r.free([0, 2])
    table, lengths, refs = r.table.clone(), r.lengths.clone(), r.refs.clone()
    wide = torch.full((5, 9), -3, dtype=torch.int32, device="cuda")
    out = [wide[:, :6], torch.full_like(lengths, 77), torch.full_like(refs, 77)]
    packed = cp.page_pool(out[0], out[1], 4, out[2])
    moved = ints([-1])
    for _ in range(3):                                # the source is untouched, so the same again
        cp.cpes_pages_compact(r.cache, r.pool, packed, r.ws, moved=moved)
    assert torch.equal(r.table, table) and torch.equal(r.lengths, lengths) and torch.equal(r.refs, refs)
    pairs = r.m.compact()
    assert int(moved) == len(pairs) > 0
    assert np.array_equal(out[2].cpu().numpy(), r.m.refs) and np.array_equal(out[1].cpu().numpy(), r.m.lengths)
    for s, row in enumerate(r.m.held()):
        assert out[0][s, :len(row)].tolist() == row
    assert bool((wide[:, 6:] == -3).all())
    for a, b in pairs:
        assert torch.equal(r.k[:, b], r.k0[:, a]) and torch.equal(r.v[:, b], r.v0[:, a])


@pytest.mark.parametrize("order", ["hnd", "nhd", "apart"])
def test_copy(order):
    r = Rig(1, 1, 30, 6, layers=3, heads=3, dim=24, order=order)
    src, dst = [4, 29, 0, 5, 31, 6, -1], [7, 2, 28, 30, 3, -2, 1]
    cp.cpes_pages_copy(r.cache, ints(src), ints(dst))
    for a, b in zip(src, dst):
        if 0 <= a < 30 and 0 <= b < 30:
            r.k0[:, b], r.v0[:, b] = r.k0[:, a], r.v0[:, a]
    assert torch.equal(r.k, r.k0) and torch.equal(r.v, r.v0)
    cp.cpes_pages_copy(r.cache, ints([]), ints([]))


def test_captured_cycle():
    """Free, reserve and fork in a graph, replayed with other lengths."""
    r = Rig(6, 8, 60, 4)
    new, status = ints([10, 7]), ints([9])
    r.reserve([0, 1], [3, 4])
    r.fork([0, 1], [2, 3])
    lists = [ints(x) for x in ([0, 1, 2, 3, 4, 5], [0, 1], [0, 0, 1, 1], [2, 3, 4, 5])]

    def cycle():
        cp.cpes_pages_free(r.pool, lists[0])
        cp.cpes_pages_reserve(r.pool, lists[1], new, r.ws)
        cp.cpes_pages_fork(r.cache, r.pool, lists[2], lists[3], r.ws, status=r.status)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        cycle()
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in ((10, 7), (1, 32), (16, 3)):
        new.copy_(torch.tensor([a, b], dtype=torch.int32))
        graph.replay()
        r.m.free(range(6))
        assert r.m.reserve([0, 1], [a, b]) == 0
        code, copies = r.m.fork([0, 0, 1, 1], [2, 3, 4, 5])
        for x, y in copies:
            r.k0[:, y], r.v0[:, y] = r.k0[:, x], r.v0[:, x]
        r.same(code)


def test_random_life_of_a_larger_pool():
    """More pages than the smaller plan takes, in a few steps of each kind."""
    rng = np.random.default_rng(9)
    r = Rig(300, 60, 5000, 3, layers=1, heads=1, dim=8)
    for step in range(24):
        empty = [s for s in range(300) if r.m.lengths[s] == 0]
        full = [s for s in range(300) if r.m.lengths[s] > 0]
        if step % 4 == 0:
            seqs = [int(s) for s in rng.permutation(300)[:int(rng.integers(1, 290))]]
            r.reserve(seqs, [int(rng.integers(0, 100)) for _ in seqs])
        elif step % 4 == 1 and empty and full:
            kids = [int(s) for s in rng.permutation(empty)[:int(rng.integers(1, 200))]]
            r.fork([int(rng.choice(full)) for _ in kids], kids)
        elif step % 4 == 2:
            r.free([int(s) for s in rng.permutation(300)[:int(rng.integers(0, 150))]])
        else:
            r.compact()


@pytest.mark.parametrize("n", [1, 5, 300, 1500])
@pytest.mark.parametrize("length", [-1, -5, -2 ** 31])
def test_negative_lengths_are_left_alone(n, length):
    """A sequence whose length is negative is refused, and the call changes nothing."""
    print(f"negative lengths n={n} {length}", flush=True)
    r = Rig(2 * n, 4, 64, 16)
    r.lengths[n // 2] = length
    before = [x.clone() for x in (r.lengths, r.refs, r.table)]
    for call in ("reserve", "fork"):
        r.status.fill_(9)
        if call == "reserve":
            cp.cpes_pages_reserve(r.pool, ints(range(n)), ints([1] * n), r.ws, status=r.status)
        else:
            cp.cpes_pages_fork(r.cache, r.pool, ints(range(n, 2 * n)), ints(range(n)), r.ws, status=r.status)
        assert int(r.status) == 2
        for a, b in zip((r.lengths, r.refs, r.table), before):
            assert torch.equal(a, b), call
