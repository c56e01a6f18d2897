"""Gradients of the scores at the sizes where loads and stores change their way through the caches: logits and
gradients of 256 MiB together, logits of 256 MiB."""
import math

import pytest
import torch

import eval_helpers as H
import paper_2608_02391_amd as cp
from test_gpu_logprobs import BF16, F32, check_gradient, score, sum_bound

pytestmark = pytest.mark.gpu
V = 50257
MIB = 1 << 20


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("limit", [128 * MIB, 256 * MIB], ids=["stores", "loads"])
@pytest.mark.parametrize("beyond", [0, 1])
@pytest.mark.parametrize("lead", [0, 3])
def test_gradients_on_either_side_of_the_caches(dtype, limit, beyond, lead):
    """Whole rows, and rows of an odd number of entries inside wider ones that start at odd elements."""
    row = V * (2 if dtype == BF16 else 4)
    rows = limit // row + beyond
    print(f"gradient rows={rows} {dtype} lead={lead}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + lead)
    wide = torch.empty(rows, V + 2 * lead, dtype=dtype, device="cuda").normal_(0.0, 2.5, generator=gen)
    x = wide[:, lead:lead + V]
    host = torch.Generator().manual_seed(rows)
    target = torch.randint(0, V, (rows,), generator=host)
    x[1, ::2] = float("-inf")
    x[2] = float("-inf")
    target[3] = -100
    x[4, 11] = 40.0
    target[4] = 11
    d_logp, d_entropy = torch.randn(rows, generator=host).cuda(), torch.randn(rows, generator=host).cuda()
    o = score(x, target, scale=1.25)
    grads = torch.full((rows, V + 2 * lead), 9.0, dtype=dtype, device="cuda")
    dx = grads[:, lead:lead + V]
    cp.cpes_logprobs_backward(x, target.cuda(), o["stats"], o["entropy"], d_logp, d_entropy, dx, scale=1.25)
    pick = [0, 1, 2, 3, 4, rows // 2, rows - 2, rows - 1]
    check_gradient(x[pick], target[pick], d_logp[pick], d_entropy[pick], dx[pick], 1.25)
    if lead:
        assert bool((grads[:, :lead] == 9).all()) and bool((grads[:, lead + V:] == 9).all())
    again = torch.empty_like(dx)                      # the rows that are not looked at: the same on every run, in place too
    cp.cpes_logprobs_backward(x, target.cuda(), o["stats"], o["entropy"], d_logp, d_entropy, again, scale=1.25)
    assert torch.equal(dx, again)
    edge = wide[:, :lead].clone(), wide[:, lead + V:].clone()
    cp.cpes_logprobs_backward(x, target.cuda(), o["stats"], o["entropy"], d_logp, d_entropy, x, scale=1.25)
    assert torch.equal(dx, x)
    if lead:
        assert torch.equal(wide[:, :lead], edge[0]) and torch.equal(wide[:, lead + V:], edge[1])
    # and every row adds up to 0: what its entries' roundings and its probabilities' bounds leave
    g, h = d_logp.double().abs(), d_entropy.double().abs()
    off = sum_bound(V) + 8 * H.EPS * (math.log(V) + 30)
    bound = H.rounding(dtype) * dx.double().abs().sum(-1) + 2 * off * 1.25 * (g + h * (2 * math.log(V) + 1))
    assert bool((dx.double().sum(-1).abs() <= bound).all())
