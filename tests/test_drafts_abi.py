"""Sampling, attention of trees, the walk and the kept path reject bad arguments on the
host, with a status code and a message; the binding rejects tensors that do not fit;
workspaces serve smaller calls.  Nothing is launched here."""
import math
import random

import pytest
import torch

import draft_helpers as D
import paper_2608_02391_amd as cp
from test_eval_abi import (BAD, BAD_CACHES, BAD_POOLS, FAKE, MISFITS, NO_REFS, REF, UNSUPPORTED, WORKSPACE, FakeGpu, cache, lib,  # noqa: F401
                           pool, refused)


def sample(lib, x=FAKE, dtype=cp.BF16, rows=1000, vocab=100, stride=100, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, u=FAKE,
           tokens=FAKE, ws=None, size=0):
    return lib.cpes_sample(x, dtype, rows, vocab, stride, scale, top_k, top_p, min_p, u, tokens, None, ws, size, None)


def tree(lib, c=None, layer=0, p=None, rows=2, starts=FAKE, tokens=10, longest=6, parents=FAKE, q=FAKE, strides=(256, 64),
         heads=4, scale=0.1, window=0, sinks=0, out=FAKE, out_strides=(256, 64), ws=FAKE, size=1 << 30):
    return lib.cpes_attend_tree(REF(c or cache()), layer, REF(p or pool()), rows, None, starts, tokens, longest, parents, q, *strides,
                                heads, scale, window, sinks, out, *out_strides, None, ws, size, None)


def accept(lib, rows=2, starts=FAKE, tokens=10, longest=6, drafted=FAKE, sampled=FAKE, kept=FAKE, path=FAKE, behind=FAKE):
    return lib.cpes_tree_accept(rows, starts, tokens, longest, None, drafted, sampled, kept, path, behind, None)


def keep(lib, c=None, p=None, n=2, starts=FAKE, longest=6, kept=FAKE, path=FAKE, ws=FAKE, size=1 << 20):
    return lib.cpes_pages_keep(REF(c or cache()), REF(p or pool()), n, None, starts, longest, kept, path, ws, size, None, None)


def test_sample(lib):
    for null in ("x", "u", "tokens"):
        refused(lib, BAD, sample(lib, **{null: None}))
    refused(lib, BAD, sample(lib, dtype=2))
    refused(lib, BAD, sample(lib, rows=-1))
    refused(lib, BAD, sample(lib, vocab=0))
    refused(lib, BAD, sample(lib, stride=99))
    for scale in (0.0, -1.0, math.nan, math.inf, 3e38):
        refused(lib, BAD, sample(lib, scale=scale), "scale")
    refused(lib, BAD, sample(lib, top_k=-1), "top_k")
    for top_p in (0.0, -0.5, 1.01, math.nan, math.inf):
        refused(lib, BAD, sample(lib, top_p=top_p), "top_p")
    for min_p in (-0.1, 1.01, math.nan):
        refused(lib, BAD, sample(lib, min_p=min_p), "min_p")
    assert sample(lib, rows=0, x=None, u=None, tokens=None) == cp.OK
    need = cp.cpes_sample_workspace_bytes(2, 100000)
    few = dict(rows=2, vocab=100000, stride=100000)
    assert need > 0
    refused(lib, WORKSPACE, sample(lib, **few))
    refused(lib, WORKSPACE, sample(lib, **few, ws=FAKE, size=100))
    refused(lib, WORKSPACE, sample(lib, **few, ws=FAKE + 4, size=need))
    assert cp.cpes_sample_workspace_bytes(-1, 100) == 0 and cp.cpes_sample_workspace_bytes(1, 0) == 0


def test_attend_tree(lib):
    for bad in BAD_CACHES:
        refused(lib, BAD, tree(lib, c=cache(**bad)))
    for bad in BAD_POOLS:
        refused(lib, BAD, tree(lib, p=pool(**bad)))
    for bad in MISFITS:
        refused(lib, BAD, tree(lib, p=pool(**bad)))
    for layer in (-1, 2):
        refused(lib, BAD, tree(lib, layer=layer), "layer")
    for null in ("starts", "q", "out"):
        refused(lib, BAD, tree(lib, **{null: None}))
    refused(lib, BAD, tree(lib, rows=-1))
    refused(lib, UNSUPPORTED, tree(lib, rows=(1 << 20) + 1))
    refused(lib, BAD, tree(lib, tokens=-1))
    for longest in (0, -1, 11):
        refused(lib, BAD, tree(lib, longest=longest), "longest")
    refused(lib, UNSUPPORTED, tree(lib, tokens=1000, longest=257), "CPES_MAX_TREE")
    for heads in (0, -2, 3):
        refused(lib, BAD, tree(lib, heads=heads), "heads")
    refused(lib, UNSUPPORTED, tree(lib, heads=2 * 65536), "heads")
    for scale in (math.nan, math.inf):
        refused(lib, BAD, tree(lib, scale=scale), "scale")
    refused(lib, BAD, tree(lib, window=-1))
    refused(lib, BAD, tree(lib, sinks=-1))
    refused(lib, BAD, tree(lib, strides=(-1, 64)))
    refused(lib, BAD, tree(lib, out_strides=(256, -1)))
    need = cp.cpes_attend_tree_workspace_bytes(2, 10, 6, 4, 2, 64)
    refused(lib, WORKSPACE, tree(lib, ws=None))
    refused(lib, WORKSPACE, tree(lib, size=need - 1))
    refused(lib, WORKSPACE, tree(lib, ws=FAKE + 8))
    assert tree(lib, rows=0, starts=None) == cp.OK
    assert tree(lib, tokens=0, longest=0, q=None, out=None) == cp.OK
    for args in ((-1, 10, 6, 4, 2, 64), (2, -1, 6, 4, 2, 64), (2, 10, 0, 4, 2, 64), (2, 10, 11, 4, 2, 64), (2, 10, 6, 4, 0, 64),
                 (2, 10, 6, 5, 2, 64), (2, 10, 6, 4, 2, 60), (2, 10, 6, 4, 2, 512), ((1 << 20) + 1, 10, 6, 4, 2, 64),
                 (2, 10, 6, 2 * 65536, 2, 64)):
        assert cp.cpes_attend_tree_workspace_bytes(*args) == 0, args


def test_accept_and_keep(lib):
    for null in ("starts", "drafted", "sampled", "kept", "path", "behind"):
        refused(lib, BAD, accept(lib, **{null: None}))
    refused(lib, BAD, accept(lib, rows=-1))
    refused(lib, UNSUPPORTED, accept(lib, rows=(1 << 20) + 1))
    refused(lib, BAD, accept(lib, tokens=-1))
    for call in (accept, keep):
        for longest in (0, -1):
            refused(lib, BAD, call(lib, longest=longest), "longest")
        refused(lib, UNSUPPORTED, call(lib, longest=257), "CPES_MAX_TREE")
    assert accept(lib, rows=0, starts=None, kept=None, path=None, behind=None) == cp.OK
    for bad in BAD_CACHES:
        refused(lib, BAD, keep(lib, c=cache(**bad)))
    for bad in BAD_POOLS + NO_REFS:
        refused(lib, BAD, keep(lib, p=pool(**bad)))
    for bad in MISFITS:
        refused(lib, BAD, keep(lib, p=pool(**bad)))
    for null in ("starts", "kept", "path"):
        refused(lib, BAD, keep(lib, **{null: None}))
    refused(lib, BAD, keep(lib, n=-1))
    refused(lib, BAD, keep(lib, n=4), "listed")
    refused(lib, UNSUPPORTED, keep(lib, p=pool(sequences=1 << 21), n=(1 << 20) + 1))
    refused(lib, WORKSPACE, keep(lib, ws=None))
    refused(lib, WORKSPACE, keep(lib, size=cp.cpes_pages_keep_workspace_bytes(2, 6) - 1))
    refused(lib, WORKSPACE, keep(lib, ws=FAKE + 4))
    big = dict(layers=1 << 14, heads=1 << 10, page_size=16, head_dim=256)
    refused(lib, UNSUPPORTED, keep(lib, c=cache(**dict(big, page_size=1 << 10)), p=pool(page_size=1 << 10)), "32 GB")
    for args in ((-1, 6), (2, 0), (2, 257)):
        assert cp.cpes_pages_keep_workspace_bytes(*args) == 0


def test_workspaces_serve_smaller_calls():
    for vocab in (100, 8192, 50257, 151936, 1 << 20):
        sizes = [cp.cpes_sample_workspace_bytes(rows, vocab) for rows in range(600)]
        assert sizes == sorted(sizes)
        assert sizes[-1] <= cp.cpes_sample_workspace_bytes(8192, vocab) == cp.cpes_sample_workspace_bytes(2 ** 31 - 1, vocab) < 1 << 27
    for heads in ((8, 2, 64), (32, 8, 128), (33, 1, 256), (3, 1, 64), (300, 1, 128), (7, 7, 256), (20, 1, 40)):
        for longest in (1, 7, 60, 200):
            sizes = [cp.cpes_attend_tree_workspace_bytes(rows, 10000, longest, *heads) for rows in range(200)]
            assert sizes == sorted(sizes) and sizes[0] > 0
        for rows in (1, 8, 300):
            sizes = [cp.cpes_attend_tree_workspace_bytes(rows, 10000, longest, *heads) for longest in range(1, 600)]
            assert sizes == sorted(sizes), heads
    for n in (0, 1, 50):
        sizes = [cp.cpes_pages_keep_workspace_bytes(n, longest) for longest in range(1, 257)]
        assert sizes == sorted(sizes) and sizes[0] > 0


def test_binding_rejects_tensors_that_do_not_fit():
    c, p = cache(), pool()
    c._dtype = torch.bfloat16
    gpu = lambda t: FakeGpu(t)
    bf = lambda *s: gpu(torch.zeros(*s, dtype=torch.bfloat16))
    ints = lambda *s: gpu(torch.zeros(*s, dtype=torch.int32))
    longs = lambda *s: gpu(torch.zeros(*s, dtype=torch.int64))
    floats = lambda *s: gpu(torch.zeros(*s))
    with pytest.raises(ValueError, match="logits must be"):
        cp.cpes_sample(bf(4), floats(4), longs(4))
    with pytest.raises(TypeError, match="uniforms"):
        cp.cpes_sample(bf(4, 9), gpu(torch.zeros(4, dtype=torch.float64)), longs(4))
    with pytest.raises(ValueError, match="uniforms holds 3"):
        cp.cpes_sample(bf(4, 9), floats(3), longs(4))
    with pytest.raises(TypeError, match="tokens"):
        cp.cpes_sample(bf(4, 9), floats(4), ints(4))
    with pytest.raises(ValueError, match="tokens holds 3"):
        cp.cpes_sample(bf(4, 9), floats(4), longs(3))
    with pytest.raises(ValueError, match="q must be"):
        cp.cpes_attend_tree(c, 0, p, bf(3, 4, 32), bf(3, 4, 32), ints(2), 3)
    with pytest.raises(ValueError, match="out has shape"):
        cp.cpes_attend_tree(c, 0, p, bf(3, 4, 64), bf(3, 3, 64), ints(2), 3)
    with pytest.raises(ValueError, match="rows \\+ 1"):
        cp.cpes_attend_tree(c, 0, p, bf(3, 4, 64), bf(3, 4, 64), ints(0), 3)
    with pytest.raises(ValueError, match="parents holds 2"):
        cp.cpes_attend_tree(c, 0, p, bf(3, 4, 64), bf(3, 4, 64), ints(2), 3, parents=ints(2))
    with pytest.raises(ValueError, match="seqs holds 1"):
        cp.cpes_attend_tree(c, 0, p, bf(3, 4, 64), bf(3, 4, 64), ints(3), 3, seqs=ints(1))
    with pytest.raises(ValueError, match="lse holds"):
        cp.cpes_attend_tree(c, 0, p, bf(3, 4, 64), bf(3, 4, 64), ints(2), 3, lse=floats(3, 3))
    with pytest.raises(ValueError, match="path must be"):
        cp.cpes_tree_accept(ints(3), longs(5), longs(5), ints(2), ints(3, 4), longs(2))
    with pytest.raises(ValueError, match="sampled holds 4"):
        cp.cpes_tree_accept(ints(3), longs(5), longs(4), ints(2), ints(2, 4), longs(2))
    with pytest.raises(TypeError, match="next_tokens"):
        cp.cpes_tree_accept(ints(3), longs(5), longs(5), ints(2), ints(2, 4), ints(2))
    with pytest.raises(ValueError, match="path must be"):
        cp.cpes_pages_keep(c, p, ints(3), ints(2), ints(2), None)
    with pytest.raises(ValueError, match="kept holds 1"):
        cp.cpes_pages_keep(c, p, ints(3), ints(1), ints(2, 4), None)


def test_plain_implementations():
    """The tests' own oracles on cases that are known."""
    assert D.branch([-1, 0, 0, 2, 9, 3], 5) == [5, 3, 2, 0] and D.branch([-1, 0, 0, 2, 9, 3], 4) == [4] and D.branch(None, 2) == [2, 1, 0]
    seen = D.seen_by([-1, 0, 0, 1], 3, 4, 8, 0, 0)
    assert seen.tolist() == [True] * 6 + [False, True]
    # window of 3 at position 6 of its text: 4, 5, 6; one sink
    assert D.seen_by([-1, 0, 0, 1], 3, 4, 8, 3, 1).tolist() == [True, False, False, False, True, True, False, True]
    x = [1.0, 2.0, 2.0, -math.inf, 0.0]
    p = [math.exp(v) if v > -math.inf else 0.0 for v in x]
    for u, token in ((0.0, 0), (0.99, 4), (p[0] / sum(p) + 1e-6, 1), ((p[0] + p[1]) / sum(p) + 1e-6, 2)):
        assert D.draw(x, u)[0] == token
    assert D.draw(x, 0.9, top_k=1)[:2] == (1, 0.0) and D.draw(x, 0.9, top_p=0.5)[0] == 2 and D.draw(x, 0.9, min_p=0.5)[0] == 2
    assert D.draw([-math.inf] * 3, 0.5)[:2] == (-1, -math.inf) and math.isnan(D.draw([0.0, math.nan], 0.5)[1])
    assert D.walk([-1, 0, 0, 2], [9, 5, 5, 7], [5, 8, 7, 3]) == ([0, 1], 8) and D.walk(None, [9, 5, 7], [5, 7, 3]) == ([0, 1, 2], 3)
    rng = random.Random(0)
    for n in (1, 2, 50):
        t = D.random_tree(n, rng)
        assert t[0] == -1 and all(0 <= a < i for i, a in enumerate(t) if i)


def test_tree_workspace_holds_every_share():
    """Where shares are of 256 queries of a KV head, 256 of them are resident, each with two partial results."""
    for dim in (64, 128):
        assert cp.cpes_attend_tree_workspace_bytes(1, 64, 64, 4, 1, dim) >= 2 * 256 * 256 * (2 + dim) * 4
        assert cp.cpes_attend_tree_workspace_bytes(1, 4096, 4096, 8, 8, dim) >= 2 * 256 * 256 * (2 + dim) * 4
