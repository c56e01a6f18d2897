"""Keys and values whose strides differ only in dimensions of one entry, which address nothing: one layer, one page,
one head, one token."""
import pytest
import torch

import paper_2608_02391_amd as cp

pytestmark = pytest.mark.gpu


def odd(t, dim, stride):
    """t again, `dim`, of one entry, with another stride."""
    strides = list(t.stride())
    strides[dim] = stride
    return t.as_strided(t.shape, strides)


@pytest.mark.parametrize("shape", [(1, 6, 2, 4, 8), (3, 1, 2, 4, 8), (3, 6, 1, 4, 8), (3, 6, 2, 1, 8), (1, 1, 1, 1, 8)])
def test_caches(shape):
    """Entry, copy and attention through a descriptor whose values' strides are odd where they do not count."""
    layers, pages, heads, size, dim = shape
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    k, v = (torch.randn(shape, generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    n = pages * size
    lengths = torch.full((1,), n, dtype=torch.int32, device="cuda")
    new = torch.randn(n, 2 * heads, dim, generator=g, device="cuda").bfloat16()
    q = torch.randn(1, 2 * heads, dim, generator=g, device="cuda").bfloat16()
    pos, seqs = torch.arange(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    ids = torch.tensor([0, pages - 1], dtype=torch.int32, device="cuda")
    ws = torch.empty(cp.cpes_attend_workspace_bytes(1, 2 * heads, heads, dim), dtype=torch.uint8, device="cuda")
    results = []
    for differ in (False, True):
        kk, vv = k.clone(), v.clone()
        if differ:
            for d in range(4):
                if shape[d] == 1:
                    vv = odd(vv, d, 40 + 8 * d)
        cache, pool = cp.paged_cache(kk, vv), cp.page_pool(table, lengths, size)
        cp.cpes_cache_append(cache, layers - 1, pool, new[:, :heads], new[:, heads:], pos, seqs=seqs)
        out, lse = torch.empty_like(q), torch.empty(1, 2 * heads, device="cuda")
        cp.cpes_attend(cache, layers - 1, pool, q, out, lse=lse, workspace=ws)
        cp.cpes_pages_copy(cache, ids[:1], ids[1:])
        results.append([x.clone() for x in (kk, vv, out, lse)])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_one_token_from_a_fused_projection():
    """A single new token whose keys are a tensor of their own and whose values are part of a wider one."""
    k, v = (torch.zeros(1, 3, 2, 4, 8, dtype=torch.float32, device="cuda") for _ in range(2))
    pool = cp.page_pool(torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3),
                        torch.full((1,), 6, dtype=torch.int32, device="cuda"), 4)
    k_new = torch.randn(1, 2, 8, device="cuda")
    v_new = torch.randn(1, 6, 8, device="cuda")[:, 2:4]
    assert k_new.stride() != v_new.stride()
    cp.cpes_cache_append(cp.paged_cache(k, v), 0, pool, k_new, v_new, torch.tensor([5], dtype=torch.int32, device="cuda"))
    assert torch.equal(k[0, 1, :, 1], k_new[0]) and torch.equal(v[0, 1, :, 1], v_new[0])
    assert int((k != 0).sum()) == 16 and int((v != 0).sum()) == 16


def test_strides_that_count_must_agree():
    k = torch.zeros(2, 3, 2, 4, 8, device="cuda")
    with pytest.raises(ValueError, match="strides"):
        cp.paged_cache(k, torch.zeros(2, 3, 4, 2, 8, device="cuda").transpose(2, 3))
    pool = cp.page_pool(torch.zeros(1, 3, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 4)
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="strides"):
        cp.cpes_cache_append(cp.paged_cache(k, k.clone()), 0, pool, torch.zeros(2, 2, 8, device="cuda"),
                             torch.zeros(2, 4, 8, device="cuda")[:, :2], pos)
