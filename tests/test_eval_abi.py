"""The evaluation operators reject bad arguments on the host, with a status code
and a message, before any HIP call; the binding rejects tensors that do not fit.
No compute is launched here."""
import ctypes
import math
import os

import pytest
import torch

import paper_2608_02391_amd as cp

FAKE = 0x10000  # a non-null, 16-byte aligned address that is never dereferenced on these paths
BAD, UNSUPPORTED, WORKSPACE = cp.ERR_INVALID_ARGUMENT, cp.ERR_UNSUPPORTED, cp.ERR_WORKSPACE
REF = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cp.LIB_PATH):
        pytest.fail("libcpes.so is not built (run __graft_entry__.build())")
    return cp.load()


def cache(**kw):
    f = dict(k=FAKE, v=FAKE, layer_stride=4096, page_stride=2048, head_stride=1024, token_stride=64, layers=2, pages=8,
             heads=2, page_size=16, head_dim=64, dtype=cp.BF16)
    f.update(kw)
    return cp.Cache(*(f[n] for n, _ in cp.Cache._fields_))


def pool(**kw):
    f = dict(table=FAKE, lengths=FAKE, refs=FAKE, table_stride=4, sequences=3, width=4, pages=8, page_size=16)
    f.update(kw)
    return cp.Pool(*(f[n] for n, _ in cp.Pool._fields_))


def refused(lib, code, rc, word=""):
    msg = lib.cpes_last_error().decode()
    assert rc == code and msg and word in msg, (rc, msg)


BAD_CACHES = [dict(k=None), dict(v=None), dict(dtype=2), dict(layers=0), dict(pages=0), dict(heads=0), dict(page_size=0),
              dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(layer_stride=-1), dict(page_stride=-1),
              dict(head_stride=-1), dict(token_stride=-1)]
BAD_POOLS = [dict(table=None), dict(lengths=None), dict(sequences=0), dict(width=0), dict(page_size=0), dict(table_stride=3)]
NO_REFS = [dict(refs=None), dict(pages=0)]
MISFITS = [dict(page_size=32), dict(pages=7)]


def fork(lib, c=None, p=None, n=1, a=FAKE, b=FAKE, ws=FAKE, size=1 << 20):
    return lib.cpes_pages_fork(REF(c or cache()), REF(p or pool()), n, a, b, ws, size, None, None)


def reserve(lib, p=None, n=1, a=FAKE, b=FAKE, ws=FAKE, size=1 << 20):
    return lib.cpes_pages_reserve(REF(p or pool()), n, a, b, ws, size, None, None)


def compact(lib, c=None, p=None, q=None, ws=FAKE, size=1 << 20):
    return lib.cpes_pages_compact(REF(c or cache()), REF(p or pool()), REF(q or pool()), ws, size, None, None)


def append(lib, c=None, layer=0, p=None, n=1, pos=FAKE, k=FAKE, v=FAKE, stride=128, head=64):
    return lib.cpes_cache_append(REF(c or cache()), layer, REF(p or pool()), n, None, pos, k, v, stride, head, None)


def attend(lib, c=None, layer=0, p=None, rows=1, q=FAKE, strides=(256, 64), heads=4, scale=0.1, window=0, sinks=0,
           out=FAKE, out_strides=(256, 64), ws=FAKE, size=1 << 30):
    return lib.cpes_attend(REF(c or cache()), layer, REF(p or pool()), rows, None, q, *strides, heads, scale, window, sinks,
                           out, *out_strides, None, ws, size, None)


def test_caches_and_pools(lib):
    for bad in BAD_CACHES:
        for call in (fork, compact, append, attend):
            refused(lib, BAD, call(lib, c=cache(**bad)))
        refused(lib, BAD, lib.cpes_pages_copy(REF(cache(**bad)), 1, FAKE, FAKE, None))
    for bad in BAD_POOLS:
        for call in (fork, compact, append, attend, reserve):
            refused(lib, BAD, call(lib, p=pool(**bad)))
        refused(lib, BAD, lib.cpes_pages_free(REF(pool(**bad)), 1, FAKE, None, None))
    for bad in NO_REFS:
        for call in (fork, compact, reserve):
            refused(lib, BAD, call(lib, p=pool(**bad)), "reference")
        refused(lib, BAD, lib.cpes_pages_free(REF(pool(**bad)), 1, FAKE, None, None))
    for bad in MISFITS:
        for call in (fork, compact, append, attend):
            refused(lib, BAD, call(lib, p=pool(**bad)))
    assert lib.cpes_attend(None, 0, REF(pool()), 1, None, FAKE, 1, 1, 2, 0.1, 0, 0, FAKE, 1, 1, None, FAKE, 1 << 30, None) == BAD
    assert lib.cpes_attend(REF(cache()), 0, None, 1, None, FAKE, 1, 1, 2, 0.1, 0, 0, FAKE, 1, 1, None, FAKE, 1 << 30, None) == BAD
    assert lib.cpes_pages_reserve(None, 1, FAKE, FAKE, FAKE, 1 << 20, None, None) == BAD
    assert lib.cpes_pages_free(None, 1, FAKE, None, None) == BAD
    assert lib.cpes_pages_copy(None, 1, FAKE, FAKE, None) == BAD


def test_pages(lib):
    for call in (reserve, fork):
        refused(lib, BAD, call(lib, n=-1))
        refused(lib, BAD, call(lib, n=4), "listed")                       # more than there are sequences
        refused(lib, BAD, call(lib, a=None))
        refused(lib, BAD, call(lib, b=None))
        refused(lib, UNSUPPORTED, call(lib, p=pool(sequences=1 << 21), n=(1 << 20) + 1))
        refused(lib, WORKSPACE, call(lib, ws=None))
        refused(lib, WORKSPACE, call(lib, size=cp.cpes_pages_workspace_bytes(8) - 1))
        refused(lib, WORKSPACE, call(lib, ws=FAKE + 4))
    refused(lib, WORKSPACE, compact(lib, ws=None))
    for other in (dict(sequences=2), dict(width=3), dict(pages=9), dict(page_size=8), dict(table_stride=5), dict(refs=None)):
        refused(lib, BAD, compact(lib, q=pool(**other)))
    refused(lib, BAD, lib.cpes_pages_free(REF(pool()), -1, FAKE, None, None))
    refused(lib, BAD, lib.cpes_pages_free(REF(pool()), 1, None, None, None))
    refused(lib, UNSUPPORTED, lib.cpes_pages_free(REF(pool()), (1 << 20) + 1, FAKE, None, None))
    for n, a, b in ((-1, FAKE, FAKE), (1, None, FAKE), (1, FAKE, None)):
        refused(lib, BAD, lib.cpes_pages_copy(REF(cache()), n, a, b, None))
    assert lib.cpes_pages_copy(REF(cache()), 0, None, None, None) == cp.OK
    big = dict(layers=1 << 14, heads=1 << 10, page_size=1 << 10, head_dim=256)
    refused(lib, UNSUPPORTED, lib.cpes_pages_copy(REF(cache(**big)), 1, FAKE, FAKE, None), "32 GB")
    assert cp.cpes_pages_workspace_bytes(0) == 0 and cp.cpes_pages_workspace_bytes(-3) == 0
    assert cp.cpes_pages_workspace_bytes(1000) >= 8000


def test_append(lib):
    refused(lib, BAD, append(lib, layer=2), "layer")
    refused(lib, BAD, append(lib, layer=-1), "layer")
    refused(lib, BAD, append(lib, n=-1))
    for null in ("pos", "k", "v"):
        refused(lib, BAD, append(lib, **{null: None}))
    refused(lib, BAD, append(lib, stride=-1))
    refused(lib, BAD, append(lib, head=-1))
    assert append(lib, n=0, pos=None, k=None, v=None) == cp.OK


def test_attend(lib):
    refused(lib, BAD, attend(lib, layer=2), "layer")
    refused(lib, BAD, attend(lib, rows=-1))
    refused(lib, UNSUPPORTED, attend(lib, rows=(1 << 20) + 1))
    refused(lib, BAD, attend(lib, q=None))
    refused(lib, BAD, attend(lib, out=None))
    for heads in (0, -2, 3):
        refused(lib, BAD, attend(lib, heads=heads), "heads")
    for scale in (math.nan, math.inf):
        refused(lib, BAD, attend(lib, scale=scale), "scale")
    refused(lib, BAD, attend(lib, window=-1))
    refused(lib, BAD, attend(lib, sinks=-1))
    refused(lib, BAD, attend(lib, strides=(-1, 64)))
    refused(lib, BAD, attend(lib, out_strides=(256, -1)))
    need = cp.cpes_attend_workspace_bytes(1, 4, 2, 64)
    refused(lib, WORKSPACE, attend(lib, ws=None))
    refused(lib, WORKSPACE, attend(lib, size=need - 1))
    refused(lib, WORKSPACE, attend(lib, ws=FAKE + 8))
    assert attend(lib, rows=0) == cp.OK
    for args in ((-1, 4, 2, 64), (1, 4, 0, 64), (1, 0, 2, 64), (1, 5, 2, 64), (1, 4, 2, 60), (1, 4, 2, 512), ((1 << 20) + 1, 4, 2, 64)):
        assert cp.cpes_attend_workspace_bytes(*args) == 0


def score(lib, x=FAKE, dtype=cp.BF16, rows=1000, vocab=100, stride=100, scale=1.0, targets=FAKE, logp=FAKE, top=0,
          top_logp=None, top_ids=None, ws=None, size=0):
    return lib.cpes_logprobs(x, dtype, rows, vocab, stride, scale, targets, logp, None, None, None, top, top_logp, top_ids,
                             ws, size, None)


def grad(lib, x=FAKE, dtype=cp.BF16, rows=2, vocab=100, stride=100, scale=1.0, targets=FAKE, stats=FAKE, entropy=FAKE,
         d_logp=FAKE, d_entropy=FAKE, dx=FAKE + 4096, dx_stride=100):
    return lib.cpes_logprobs_backward(x, dtype, rows, vocab, stride, scale, targets, stats, entropy, d_logp, d_entropy, dx,
                                      dx_stride, None)


def test_logprobs(lib):
    for call in (score, grad):
        refused(lib, BAD, call(lib, x=None))
        refused(lib, BAD, call(lib, dtype=2))
        refused(lib, BAD, call(lib, rows=-1))
        refused(lib, BAD, call(lib, vocab=0))
        refused(lib, BAD, call(lib, stride=99))
        for scale in (0.0, -1.0, math.nan, math.inf):
            refused(lib, BAD, call(lib, scale=scale), "scale")
        assert call(lib, rows=0) == cp.OK
    refused(lib, BAD, score(lib, targets=None), "targets")
    refused(lib, BAD, score(lib, top=-1, top_logp=FAKE, top_ids=FAKE))
    refused(lib, BAD, score(lib, top=65, top_logp=FAKE, top_ids=FAKE))
    refused(lib, BAD, score(lib, top=3, top_logp=FAKE))
    refused(lib, BAD, score(lib, top=3, top_ids=FAKE))
    need = cp.cpes_logprobs_workspace_bytes(2, 100000, 3)
    few = dict(rows=2, vocab=100000, stride=100000, top=3, top_logp=FAKE, top_ids=FAKE)
    assert need > 0
    refused(lib, WORKSPACE, score(lib, **few))
    refused(lib, WORKSPACE, score(lib, **few, ws=FAKE, size=100))
    refused(lib, WORKSPACE, score(lib, **few, ws=FAKE + 4, size=need))
    for args in ((-1, 100, 0), (1, 0, 0), (1, 100, -1), (1, 100, 65)):
        assert cp.cpes_logprobs_workspace_bytes(*args) == 0
    refused(lib, BAD, grad(lib, stats=None))
    refused(lib, BAD, grad(lib, dx=None))
    refused(lib, BAD, grad(lib, targets=None))
    refused(lib, BAD, grad(lib, entropy=None))
    refused(lib, BAD, grad(lib, dx_stride=99))
    refused(lib, BAD, grad(lib, dx=FAKE, dx_stride=101), "in place")


def test_binding_rejects_tensors_that_do_not_fit():
    """Sizes, dtypes and shapes the C ABI cannot see (host tensors: refused before any launch)."""
    c, p = cache(), pool()
    c._dtype = torch.bfloat16
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    ints = lambda n: torch.zeros(n, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU tensors"):
        cp.paged_cache(bf(1, 2, 2, 4, 8), bf(1, 2, 2, 4, 8))
    for k, v in ((bf(2, 2, 4, 8), bf(2, 2, 4, 8)), (bf(1, 2, 2, 4, 8), bf(1, 2, 2, 4, 16)),
                 (bf(1, 2, 2, 4, 8), torch.zeros(1, 2, 2, 4, 8)), (bf(1, 2, 2, 4, 8), bf(1, 2, 4, 2, 8).transpose(2, 3))):
        with pytest.raises(ValueError, match="one shape"):
            cp.paged_cache(k, v)
    with pytest.raises(ValueError, match="page table"):
        cp.page_pool(ints(4), ints(4), 16)
    with pytest.raises(ValueError, match="GPU tensor"):
        cp.page_pool(ints(4).view(2, 2), ints(2), 16)
    with pytest.raises(TypeError, match="new_lengths"):
        cp.cpes_pages_reserve(p, FakeGpu(ints(0)), torch.zeros(0, dtype=torch.int64), None)
    with pytest.raises(ValueError, match="k_new has shape"):
        cp.cpes_cache_append(c, 0, p, FakeGpu(bf(3, 2, 32)), bf(3, 2, 32), ints(3))
    with pytest.raises(TypeError, match="k_new must have dtype"):
        cp.cpes_cache_append(c, 0, p, torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), ints(3))
    with pytest.raises(ValueError, match="q must be"):
        cp.cpes_attend(c, 0, p, bf(3, 4, 32), bf(3, 4, 32))
    with pytest.raises(ValueError, match="out has shape"):
        cp.cpes_attend(c, 0, p, FakeGpu(bf(3, 4, 64)), FakeGpu(bf(3, 3, 64)))
    with pytest.raises(ValueError, match="logits must be"):
        cp.cpes_logprobs(bf(4), None, None)
    with pytest.raises(ValueError, match="GPU tensor"):
        cp.cpes_logprobs(bf(4, 9), None, None)
    with pytest.raises(TypeError, match="targets"):
        cp.cpes_logprobs(FakeGpu(bf(4, 9)), ints(4), None)
    with pytest.raises(ValueError, match="both be"):
        cp.cpes_logprobs(FakeGpu(bf(4, 9)), None, None, top_ids=torch.zeros(4, 2, dtype=torch.int64))
    with pytest.raises(ValueError, match="shape and dtype"):
        cp.cpes_logprobs_backward(FakeGpu(bf(4, 9)), None, None, None, None, None, FakeGpu(bf(4, 8)))


class FakeGpu:
    """A host tensor that says it is on the GPU, to reach the checks behind that one."""

    def __init__(self, t):
        self.t = t

    is_cuda = True

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_sizes_beyond_any_memory(lib):
    """Strides and counts whose products would overflow 64 bits, and more heads than the kernels count."""
    for huge in (dict(layer_stride=1 << 62), dict(page_stride=1 << 60), dict(head_stride=1 << 61), dict(token_stride=1 << 62),
                 dict(layer_stride=1 << 40, layers=1 << 30)):
        for call in (fork, compact, append, attend):
            refused(lib, BAD, call(lib, c=cache(**huge)), "stride")
    for call in (fork, compact, append, attend):
        refused(lib, UNSUPPORTED, call(lib, c=cache(heads=65537)), "heads")
    refused(lib, UNSUPPORTED, attend(lib, heads=2 * 65536), "heads")
    assert cp.cpes_attend_workspace_bytes(1, 2 * 65536, 2, 64) == 0
    most = dict(layers=2 ** 31 - 1, heads=65536, page_size=2 ** 31 - 1, head_dim=256, layer_stride=0, page_stride=0, head_stride=0,
                token_stride=0)
    refused(lib, UNSUPPORTED, lib.cpes_pages_copy(REF(cache(**most)), 1, FAKE, FAKE, None), "32 GB")
