"""How many bits a weight of the fp32 cache's attention keeps.

Queries with a single 1 make a score one entry of its key, and values with a single 1 make an output one weight over
the sum, so that nothing but the weights' own roundings is left.  Scores are multiples of 2^-10 in descending order:
their differences are exact, and no maximum grows on the way.  Roundings, in units of 2^-24 relative:

* an exponential of two ulps (the library function's one, doubled): 4;
* the sum over one tile of 16: those of its weights, 4 additions in a lane and 2 between lanes; one division or a
  reciprocal and a product: 2.  In all 4 + 4 + 4 + 2 + 2, and 2 to spare: 18;
* over more tiles pieces join with factors of their own, two at most, each an exponential and a product (5, on both
  sides of the quotient), 5 additions a tile and 12 where pieces join: 20 + 5 (tiles - 1) + 12 more.

A logarithm of two ulps and the roundings of the result lie on top of the sum's error for lse."""
import numpy as np
import pytest
import torch

from eval_helpers import EPS
from test_gpu_attend import F32, Case


def bound(n):
    tiles = -(-n // 16)
    return (18 if tiles == 1 else 18 + 20 + 5 * (tiles - 1) + 12) * EPS


def scores(n, heads, dim, seed):
    rng = np.random.default_rng(seed)
    return -np.sort(-rng.integers(-50 * 1024, 4 * 1024, size=(n, heads, dim)), axis=0) / 1024.0


def test_the_bound_tells_fewer_bits():
    """Weights kept as two bf16, or taken as 2^x of a rounded product, are beyond the bound; plain fp32 is within."""
    x = scores(16, 8, 64, 5).reshape(16, -1)
    d = (x - x[0]).astype(np.float32)
    exact = np.exp(x - x[0])
    exact /= exact.sum(0)

    def worst(w, total):
        return (np.abs(w.astype(np.float64) / total.astype(np.float64) - exact) / exact).max()

    w = np.exp(d)
    total = w.sum(0, dtype=np.float32)
    assert worst(w, total) <= bound(16)
    bf = lambda a: torch.from_numpy(a).bfloat16().float().numpy()
    assert worst(bf(w) + bf(w - bf(w)), total) > bound(16)
    assert worst(bf(w), total) > 100 * bound(16)
    two = np.exp2((d * np.float32(1.44269504088896340736)).astype(np.float32))
    assert worst(two, two.sum(0, dtype=np.float32)) > bound(16)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,page", [(8, 16), (64, 16), (64, 7), (80, 16), (128, 16), (128, 32), (256, 16), (256, 5)])
@pytest.mark.parametrize("width", [None, 5000], ids=["narrow", "wide"])
def test_weights_keep_their_bits(dim, page, width):
    """Rows of one workgroup, and rows of shares."""
    print(f"fp32 weights dim={dim} page={page} width={width}", flush=True)
    lens = [n for n in (1, 5, 8, 15, 16, 33, 64, 100, 200, 256) if n <= dim]
    kv, group = 2, 3
    c = Case(lens, kv, dim, page, F32, layers=1, layer=0, seed=dim + page, width=width)
    for s, n in enumerate(lens):
        x = torch.from_numpy(scores(n, kv, dim, 100 * s + dim)).float()
        j = torch.arange(n)
        ones = torch.zeros(n, kv, dim)
        ones[j, :, j] = 1.0
        at = c.table[s].long()[j // page].cuda(), (j % page).cuda()
        c.k[0][at[0], :, at[1]], c.v[0][at[0], :, at[1]] = x.cuda(), ones.cuda()
        c.keys[s] = x
    q = torch.zeros(len(lens), kv * group, dim)
    for i in range(kv * group):
        q[:, i, i] = 1.0
    out, lse = (t.cpu().double().numpy() for t in c.run(q, scale=1.0))
    for s, n in enumerate(lens):
        for i in range(kv * group):
            x = c.keys[s][:, i // group, i].double().numpy()
            w = np.exp(x - x[0])
            want = w / w.sum()
            off = np.abs(out[s, i, :n] - want) / want
            assert off.max() <= bound(n), (s, i, n, off.max() / EPS)
            assert not out[s, i, n:].any()
            exact = x[0] + np.log(w.sum())
            assert abs(lse[s, i] - exact) <= bound(n) + 4 * EPS * np.log(w.sum()) + 2 * EPS * abs(exact), (s, i, n)
