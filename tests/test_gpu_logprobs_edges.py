"""Scores and gradients at the edges: not-a-number and +inf wherever they stand, among masked logits too, and
the largest vocabularies."""
import math

import pytest
import torch

import paper_2608_02391_amd as cp
from test_gpu_logprobs import BF16, F32, check, check_gradient, logits, score

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,V", [(4, 1), (4, 3001), (800, 3001), (4, 140003), (300, 70001)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["all_nan", "nan_among_masked", "inf_among_masked", "nan_target"])
def test_rows_without_a_finite_logit(rows, V, dtype, kind):
    """Every number of such a row is NaN, its log probability too, whichever launch scores it; rows beside it are not
    touched."""
    print(f"broken {kind} rows={rows} V={V} {dtype}", flush=True)
    x, t = logits(rows, V, dtype, V + rows)
    if kind == "all_nan":
        x[1] = math.nan
    else:
        x[1] = -math.inf
        x[1, V // 2] = math.inf if kind == "inf_among_masked" else math.nan
    t[1] = V // 2 if kind == "nan_target" else V - 1
    x = x.cuda()
    o = score(x, t, top=4)
    for name in ("logp", "entropy", "lse", "top_logp"):
        assert bool(torch.isnan(o[name][1]).all()), name
    assert bool((o["top_ids"][1] == -1).all())
    pick = [0, 2, rows - 1]
    check(x[pick], t[pick], {k: v[pick] for k, v in o.items()}, top=4)
    one = torch.ones(rows, device="cuda")
    for d_logp, d_entropy in ((one, None), (None, one), (one, one)):
        dx = torch.zeros_like(x)
        cp.cpes_logprobs_backward(x, t.cuda(), o["stats"], o["entropy"], d_logp, d_entropy, dx)
        assert bool(torch.isnan(dx[1]).all())
        check_gradient(x[pick], t[pick], None if d_logp is None else one[pick], None if d_entropy is None else one[pick], dx[pick])


@pytest.mark.parametrize("V,dtype", [(2 ** 31 - 1, BF16), (2 ** 31 - 7, BF16), (2 ** 31 - 8, BF16), (2 ** 31 - 1, F32), (2 ** 31 - 4, F32)])
def test_largest_vocabularies(V, dtype):
    """One row up to the largest vocabulary the argument holds: every entry of the gradient is written.

    The logits are equal but for three, so the numbers have closed forms.  A thread's terms are relative to its own
    maximum: 1 each, and their sum of V / 2^14 exact, but for three threads, which hold 2^-12 of the whole at 2^-7.  Sums
    join in 14 steps, each an exponential's 2^-21 off; lse, near 21.5, and its parts are rounded a few times: below 2e-5.
    A probability carries that, its own 2^-21 and the roundings of an exponent of 23: below 4e-5."""
    off = 2e-5
    print(f"largest V={V} {dtype}", flush=True)
    x = torch.full((1, V), 0.0, dtype=dtype, device="cuda")
    special = {0: 1.0, V // 3: 2.0, V - 1: 1.5}
    for v, value in special.items():
        x[0, v] = value
    target = torch.tensor([V - 1])
    o = score(x, target, top=3)
    total = V - 3 + sum(math.exp(value) for value in special.values())
    lse = math.log(total)
    assert abs(float(o["lse"]) - lse) <= off and abs(float(o["logp"]) - (1.5 - lse)) <= off
    assert o["top_ids"][0].tolist() == [V // 3, V - 1, 0]
    one = torch.ones(1, device="cuda")
    dx = torch.full_like(x, 7.0)
    cp.cpes_logprobs_backward(x, target.cuda(), o["stats"], None, one, None, dx)
    rounding = 2 * off + (2.0 ** -8 if dtype == BF16 else 2.0 ** -24)
    for v in (0, 1, 12345, V // 3, V // 2, V - 9, V - 8, V - 7, V - 3, V - 2):
        want = -math.exp(special.get(v, 0.0) - lse)
        assert abs(float(dx[0, v]) - want) <= rounding * abs(want), v
    assert abs(float(dx[0, V - 1]) - 1.0) <= rounding
    plain = -math.exp(-lse)
    low, high = plain * (1 + rounding), plain * (1 - rounding)
    for s in range(0, V, 1 << 28):
        part = dx[0, s:s + (1 << 28)]
        here = sum(1 for v in special if s <= v < s + part.numel())
        assert int(((part < low) | (part > high)).sum()) <= here, s


@pytest.mark.parametrize("vocab", [151936, 70001])
def test_one_workspace_as_rows_end(vocab):
    """The workspace of the first batch scores what is left of it, whichever number that is."""
    top, most = 20, 300
    x, t = logits(most, vocab, BF16, 3)
    x, dt = x.cuda(), t.cuda()
    ws = torch.empty(cp.cpes_logprobs_workspace_bytes(most, vocab, top), dtype=torch.uint8, device="cuda")
    f = lambda *shape: torch.empty(*shape, device="cuda")
    for rows in (300, 257, 256, 200, 100, 65, 48, 33, 32, 8, 7, 2, 1):
        o = dict(logp=f(rows), entropy=f(rows), lse=f(rows), top_logp=f(rows, top),
                 top_ids=torch.empty(rows, top, dtype=torch.int64, device="cuda"))
        cp.cpes_logprobs(x[:rows], dt[:rows], workspace=ws, **o)
        pick = sorted({0, rows // 2, rows - 1})
        check(x[pick], t[pick], {k: v[pick] for k, v in o.items()}, top=top)
