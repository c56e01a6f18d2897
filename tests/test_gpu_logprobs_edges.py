"""Scores and gradients at the edges: not-a-number and +inf wherever they stand, among masked logits too."""
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
