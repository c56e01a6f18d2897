"""Scores of tokens -- log probabilities, entropies, alternatives -- and their
gradient, against a plain implementation in 64 bits and against differences.

Bounds.  A sum of V / 256 terms per thread and a tree of a few more: rounding
errors of random sign, six standard deviations of sqrt(V / 256 + 32) EPS,
relative; each exponential 2^-21 and the roundings of d = scale (x - max) and of
its product with log2 e, |d| 3 EPS, which the weights e^d hold below 3 EPS / e on
the sums and which a single token's log probability carries in full."""
import math

import numpy as np
import pytest
import torch

import eval_helpers as H
import paper_2608_02391_amd as cp

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def sum_bound(V):
    return 6 * math.sqrt(V / 256 + 32) * H.EPS + 2.0 ** -20


def logits(rows, V, dtype, seed, std=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, V, generator=g) * std).to(dtype), torch.randint(0, V, (rows,), generator=g)


def score(x, target, scale=1.0, top=0, stream=None):
    rows, V = x.shape
    f = lambda *shape: torch.full(shape, 7.0, device="cuda")
    o = dict(logp=f(rows), entropy=f(rows), lse=f(rows), stats=f(rows, 2))
    if top:
        o.update(top_logp=f(rows, top), top_ids=torch.full((rows, top), 7, dtype=torch.int64, device="cuda"))
    ws = torch.full((cp.cpes_logprobs_workspace_bytes(rows, V, top),), 0xFF, dtype=torch.uint8, device="cuda")
    cp.cpes_logprobs(x, target.cuda(), scale=scale, workspace=ws, stream=stream, **o)
    return o


def check(x, target, o, scale=1.0, top=0):
    host = x.cpu().double().numpy()
    got = {k: v.cpu().double().numpy() for k, v in o.items()}
    for r in range(host.shape[0]):
        ref = H.logprobs(host[r], int(target[r]), scale, top)
        b = sum_bound(host.shape[1])
        def near(a, e, extra=0.0):
            if math.isinf(e):
                assert a == e, (r, a, e)
            else:
                assert abs(a - e) <= b + 4 * H.EPS * abs(e) + extra, (r, a, e)
        near(got["lse"][r], ref["lse"], 0 if math.isinf(ref["lse"]) else 4 * H.EPS * scale * float(np.max(host[r])) if np.max(host[r]) > 0 else 4 * H.EPS * abs(scale * float(np.max(host[r]))))
        near(got["logp"][r], ref["logp"])
        near(got["entropy"][r], ref["entropy"], 2 * b * abs(ref["entropy"]))
        if top:
            assert np.array_equal(o["top_ids"][r].cpu().numpy(), ref["ids"]), r
            for j in range(top):
                near(got["top_logp"][r, j], ref["tops"][j])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 257, 2047, 2048, 4097, 8191, 50257, 151936])
def test_vocabularies(dtype, V):
    rows = 3
    print(f"logprobs V={V} {dtype}", flush=True)
    x, t = logits(rows, V, dtype, V)
    x = x.cuda()
    check(x, t, score(x, t, top=5), top=5)
    check(x, t, score(x, t, scale=0.7), scale=0.7)


@pytest.mark.parametrize("rows", [1, 2, 5, 100, 767, 768, 1500])
@pytest.mark.parametrize("top", [0, 1, 64])
def test_row_counts(rows, top):
    """Rows cut into slices and rows of one workgroup."""
    print(f"logprobs rows={rows} top={top}", flush=True)
    x, t = logits(rows, 5003, BF16, rows)
    x = x.cuda()
    o = score(x, t, top=top)
    pick = range(rows) if rows < 20 else [0, 1, rows // 2, rows - 1]
    sub = {k: v[list(pick)] for k, v in o.items()}
    check(x[list(pick)], t[list(pick)], sub, top=top)


@pytest.mark.parametrize("rows", [2, 900])
@pytest.mark.parametrize("kind", ["equal", "descending", "ascending", "one_thread", "few_values", "signed_zeros", "lowest"])
def test_alternatives_on_awkward_rows(rows, kind):
    """Ties go to the lowest token; a thread's share may hold every large logit."""
    V, top = 9001, 33
    print(f"alternatives {kind} rows={rows}", flush=True)
    v = torch.arange(V)
    if kind == "equal":
        x = torch.full((V,), 1.5)
    elif kind == "descending":
        x = -v / 100.0
    elif kind == "ascending":
        x = v / 100.0
    elif kind == "one_thread":
        x = torch.where(v // 8 % 256 == 77, 10 + (v % 13) / 8.0, -(v % 5) / 1.0)
    elif kind == "few_values":
        x = (v * 7919 % 3).float()
    elif kind == "signed_zeros":
        x = torch.where(v % 2 == 0, -0.0, 0.0)
    else:
        x = torch.full((V,), torch.finfo(BF16).min)
        x[V // 3:V // 3 + 10] = 2.0
    x = x.to(BF16)[None].repeat(rows, 1).contiguous().cuda()
    t = torch.full((rows,), V // 3)
    o = score(x, t, top=top)
    check(x[:2], t[:2], {k: y[:2] for k, y in o.items()}, top=top)
    assert all(torch.equal(y[0], y[-1]) for y in o.values())


@pytest.mark.parametrize("rows,V,dtype", [(3, 70000, BF16), (800, 70000, BF16), (800, 3001, F32)])
@pytest.mark.parametrize("levels", [3, 40, 1000])
def test_alternatives_among_many_ties(rows, V, dtype, levels):
    """Random logits of few values: the k-th largest ties with others all over the row."""
    print(f"ties rows={rows} V={V} levels={levels}", flush=True)
    top = 20
    g = torch.Generator(device="cuda").manual_seed(levels)
    x = torch.randn(rows, V, generator=g, device="cuda")
    x = ((x * levels / 8).round() * (8.0 / levels)).to(dtype)
    t = torch.zeros(rows, dtype=torch.int64)
    o = score(x, t, top=top)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(o["top_ids"], order)


@pytest.mark.parametrize("rows", [4, 1000])
def test_masked_rows(rows):
    """-inf in most places, in all but one, in all; the type's lowest value everywhere; a target outside."""
    V, top = 5000, 6
    x, t = logits(rows, V, F32, 3)
    x[0, torch.arange(V) % 37 != 5] = -math.inf
    t[0] = 6                                          # itself masked
    x[1] = -math.inf
    x[1, 4321] = -3.0
    t[1] = 4321
    x[2] = -math.inf
    x[3] = torch.finfo(F32).min
    x = x.cuda()
    o = score(x, t, top=top)
    check(x[:4], t[:4], {k: y[:4] for k, y in o.items()}, top=top)
    t[0], t[1] = -1, V
    o = score(x, t, top=top)
    check(x[:4], t[:4], {k: y[:4] for k, y in o.items()}, top=top)
    assert float(o["logp"][0]) == 0.0 and float(o["logp"][1]) == 0.0


@pytest.mark.parametrize("rows", [3, 800])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_broken_rows(rows, bad):
    V = 3001
    x, t = logits(rows, V, BF16, 4)
    x[1, 2999] = bad
    x = x.cuda()
    o = score(x, t, top=4)
    for n in ("logp", "entropy", "lse", "top_logp"):
        assert bool(torch.isnan(o[n][1]).all()), n
    assert bool((o["top_ids"][1] == -1).all())
    check(x[[0, 2]], t[[0, 2]], {k: y[[0, 2]] for k, y in o.items()}, top=4)
    dx = torch.empty_like(x)
    one = torch.ones(rows, device="cuda")
    cp.cpes_logprobs_backward(x, t.cuda(), o["stats"], o["entropy"], one, one, dx)
    assert bool(torch.isnan(dx[1]).all()) and bool(torch.isfinite(dx[0].float()).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_rows_inside_a_wider_tensor(dtype):
    """Rows further apart than they are long, starting at odd elements."""
    wide, t = logits(5, 4099, dtype, 9)
    t = t % 4001
    x = wide.cuda()[:, 3:4004]
    o = score(x, t, top=3)
    check(x, t, o, top=3)
    grads = torch.full((5, 5000), 9.0, dtype=dtype, device="cuda")
    dx = grads[:, 1:4002]
    one = torch.ones(5, device="cuda")
    cp.cpes_logprobs_backward(x, t.cuda(), o["stats"], None, one, None, dx)
    check_gradient(x, t, one, None, dx)
    assert bool((grads[:, 0] == 9).all()) and bool((grads[:, 4002:] == 9).all())


def check_gradient(x, target, d_logp, d_entropy, dx, scale=1.0):
    """dx against scale (g (onehot - p) - h p (ln p + H)) in 64 bits: the weight p is off by
    its exponential's bound times what multiplies it, the result rounded once."""
    host, got, dtype = x.cpu().double().numpy(), dx.cpu().double().numpy(), x.dtype
    V = host.shape[1]
    for r in range(host.shape[0]):
        ref = H.logprobs(host[r], int(target[r]), scale, 0)
        logp = ref["every"]
        if math.isinf(ref["lse"]):
            assert not got[r].any()
            continue
        p = np.exp(logp)
        g = float(d_logp[r]) if d_logp is not None else 0.0
        h = float(d_entropy[r]) if d_entropy is not None else 0.0
        t = int(target[r])
        if not 0 <= t < V:
            g = 0.0
        onehot = np.zeros(V)
        if 0 <= t < V:
            onehot[t] = 1
        lp = np.where(p > 0, logp, 0.0)
        exact = scale * (g * (onehot - p) - h * p * (lp + ref["entropy"]))
        e = sum_bound(V) + 8 * H.EPS * (np.abs(lp) + 1)
        size = scale * p * (abs(g) + abs(h) * (np.abs(lp) + ref["entropy"] + 1))
        tol = 2 * e * size + 8 * H.EPS * scale * abs(g) * onehot + H.rounding(dtype) * np.abs(exact) * 1.01 + 1e-37
        worst = np.argmax(np.abs(got[r] - exact) - tol)
        assert abs(got[r][worst] - exact[worst]) <= tol[worst], (r, worst, got[r][worst], exact[worst])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 5, 8, 1000, 4096, 4099, 50257])
@pytest.mark.parametrize("which", ["logp", "entropy", "both"])
def test_gradient(dtype, V, which):
    print(f"gradient V={V} {dtype} {which}", flush=True)
    rows, scale = 4, 1.25
    x, t = logits(rows, V, dtype, V + 1)
    if V > 5:
        x[1, ::2] = -math.inf
        x[2] = -math.inf
        t[3] = -100
    x = x.cuda()
    g = torch.Generator().manual_seed(5)
    d_logp = torch.randn(rows, generator=g).cuda() if which != "entropy" else None
    d_entropy = torch.randn(rows, generator=g).cuda() if which != "logp" else None
    o = score(x, t, scale=scale)
    dx = torch.full_like(x, 5.0)
    cp.cpes_logprobs_backward(x, t.cuda(), o["stats"], o["entropy"], d_logp, d_entropy, dx, scale=scale)
    check_gradient(x, t, d_logp, d_entropy, dx, scale)
    same = x.clone()                                  # in place
    cp.cpes_logprobs_backward(same, t.cuda(), o["stats"], o["entropy"], d_logp, d_entropy, same, scale=scale)
    assert torch.equal(same, dx)


def test_gradient_against_differences():
    """Central differences of the 64-bit forward: their own error is h^2 times a third
    derivative below 2, 2e-8 at h = 1e-4, and rounding of 1e-11."""
    V, scale, h = 23, 0.8, 1e-4
    x, t = logits(3, V, F32, 8, std=1.5)
    dx = torch.empty_like(x, device="cuda")
    d_logp, d_entropy = torch.tensor([1.0, 0.0, -0.7]).cuda(), torch.tensor([0.0, 1.0, 0.4]).cuda()
    xd = x.cuda()
    o = score(xd, t, scale=scale)
    cp.cpes_logprobs_backward(xd, t.cuda(), o["stats"], o["entropy"], d_logp, d_entropy, dx, scale=scale)
    for r in range(3):
        def f(row):
            y = H.logprobs(row, int(t[r]), scale, 0)
            return float(d_logp[r]) * y["logp"] + float(d_entropy[r]) * y["entropy"]
        for v in range(V):
            up, down = x[r].double().numpy().copy(), x[r].double().numpy().copy()
            up[v] += h
            down[v] -= h
            assert abs((f(up) - f(down)) / (2 * h) - float(dx[r, v])) <= 1e-6


def test_every_output_is_optional_and_no_rows():
    x, t = logits(3, 700, BF16, 1)
    x = x.cuda()
    full = score(x, t, top=2)
    ws = torch.empty(cp.cpes_logprobs_workspace_bytes(3, 700, 2), dtype=torch.uint8, device="cuda")
    entropy = torch.empty(3, device="cuda")
    cp.cpes_logprobs(x, None, None, entropy=entropy, workspace=ws)
    assert torch.equal(entropy, full["entropy"])
    ids, tops = torch.empty(3, 2, dtype=torch.int64, device="cuda"), torch.empty(3, 2, device="cuda")
    cp.cpes_logprobs(x, None, None, top_ids=ids, top_logp=tops, workspace=ws)
    assert torch.equal(ids, full["top_ids"]) and torch.equal(tops, full["top_logp"])
    cp.cpes_logprobs(x[:0], t[:0].cuda(), entropy[:0])
    torch.cuda.synchronize()


def test_captured_and_on_another_stream():
    x, t = logits(6, 40000, BF16, 2)
    dx, dt = x.cuda(), t.cuda()
    f = lambda *s: torch.empty(*s, device="cuda")
    o = dict(logp=f(6), entropy=f(6), lse=f(6), stats=f(6, 2), top_logp=f(6, 9),
             top_ids=torch.empty(6, 9, dtype=torch.int64, device="cuda"))
    ws = torch.empty(cp.cpes_logprobs_workspace_bytes(6, 40000, 9), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        cp.cpes_logprobs(dx, dt, workspace=ws, **o)
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(side)
    for seed in (5, 6, 7):
        x2, _ = logits(6, 40000, BF16, seed)
        dx.copy_(x2)
        graph.replay()
        torch.cuda.synchronize()
        eager = score(dx, t, top=9)
        assert all(torch.equal(o[k], eager[k]) for k in o)
        check(dx, t, o, top=9)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,V", [(3, 151936), (900, 30011), (2, 700)])
@pytest.mark.parametrize("lead", [16.0, 30.0, 60.0])
def test_near_certain_tokens(dtype, rows, V, lead):
    """One logit far above the others: its log probability -ln (1 + s), the entropy and its gradient
    g (1 - p) are of the size of s, and keep their digits.  Each term of s is off by its exponential's 2^-21 and by
    the roundings of an exponent of the size of the lead, relative."""
    print(f"near certain V={V} lead={lead} {dtype}", flush=True)
    x, t = logits(rows, V, dtype, 11, std=1.0)
    x[torch.arange(rows), t] = lead
    xd = x.cuda()
    o = score(xd, t, top=2)
    dx, one = torch.empty(rows, V, device="cuda", dtype=dtype), torch.ones(rows, device="cuda")
    cp.cpes_logprobs_backward(xd, t.cuda(), o["stats"], None, one, None, dx)
    rel = sum_bound(V) + 8 * H.EPS * (lead + 6)
    for r in range(0, rows, max(1, rows // 3)):
        d = x[r].double().numpy() - lead
        s = np.exp(np.delete(d, int(t[r]))).sum()
        logp, entropy = -math.log1p(s), math.log1p(s) - float((np.delete(d, int(t[r])) * np.exp(np.delete(d, int(t[r])))).sum()) / (1 + s)
        assert int(o["top_ids"][r, 0]) == int(t[r])
        for got, want in ((o["logp"][r], logp), (o["top_logp"][r, 0], logp), (o["entropy"][r], entropy)):
            assert abs(float(got) - want) <= rel * abs(want) + 1e-38, (r, float(got), want)
        want = s / (1 + s)
        assert abs(float(dx[r, t[r]]) - want) <= (rel + H.rounding(dtype)) * want + 1e-38, (r, float(dx[r, t[r]]), want)


@pytest.mark.parametrize("rows,V,dtype", [(770, 151936, F32), (770, 300007, BF16), (2, 5000011, BF16)])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_alternatives_of_long_rows(rows, V, dtype, top):
    """Rows of more steps than a thread keeps notes of: notes of several steps each."""
    print(f"long rows={rows} V={V} top={top} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(top)
    x = torch.randn(rows, V, generator=g, device="cuda").to(dtype)
    t = torch.randint(0, V, (rows,))
    o = score(x, t, top=top)
    for r in range(0, rows, 97):
        # ties by the lowest token: a stable sort
        order = torch.sort(x[r].double(), descending=True, stable=True).indices[:top]
        assert torch.equal(o["top_ids"][r], order), r
    check(x[:2], t[:2], {k: y[:2] for k, y in o.items()}, top=top)


@pytest.mark.parametrize("rows", [1, 3, 40, 200, 256, 257])
@pytest.mark.parametrize("V,dtype", [(65535, BF16), (65536, BF16), (140001, BF16), (32767, F32), (32768, F32), (70001, F32)])
def test_sliced_rows(rows, V, dtype):
    """Row counts and lengths on either side of the rule that cuts rows into slices."""
    print(f"sliced rows={rows} V={V} {dtype}", flush=True)
    x, t = logits(rows, V, dtype, rows + V)
    x = x.cuda()
    for top in (0, 7, 64):
        o = score(x, t, top=top, scale=0.9)
        pick = sorted({0, rows // 2, rows - 1})
        check(x[pick], t[pick], {k: v[pick] for k, v in o.items()}, scale=0.9, top=top)


@pytest.mark.parametrize("kind", ["equal", "descending", "one_slice", "few_values", "masked_but_few", "masked", "lowest", "nan", "inf"])
def test_awkward_sliced_rows(kind):
    """Ties across slices, slices of nothing but -inf, one slice that holds every large logit, broken ones."""
    V, top, rows = 140003, 33, 3
    print(f"awkward slices {kind}", flush=True)
    v = torch.arange(V)
    x = (v * 7919 % 101) / 16.0
    if kind == "equal":
        x = torch.full((V,), -2.5)
    elif kind == "descending":
        x = -v / 1000.0
    elif kind == "one_slice":
        x = torch.where((v > 100000) & (v < 100400), 20 + (v % 7) / 8.0, x)
    elif kind == "few_values":
        x = (v * 7919 % 2).float()
    elif kind == "masked_but_few":
        x = torch.where(v % 14000 == 9, x, torch.tensor(-math.inf))
    elif kind == "masked":
        x = torch.full((V,), -math.inf)
    elif kind == "lowest":
        x = torch.full((V,), torch.finfo(BF16).min)
        x[77777] = 1.0
    elif kind in ("nan", "inf"):
        x[V - 2] = float(kind)
    x = x.to(BF16)[None].repeat(rows, 1).contiguous().cuda()
    t = torch.tensor([77777, 0, V - 1])
    o = score(x, t, top=top)
    if kind in ("nan", "inf"):
        assert all(bool(torch.isnan(o[n]).all()) for n in ("logp", "entropy", "lse", "top_logp")) and bool((o["top_ids"] == -1).all())
        return
    check(x, t, o, top=top)


@pytest.mark.parametrize("rows", [5, 512, 513, 1100])
@pytest.mark.parametrize("V,dtype", [(60, BF16), (300, BF16), (2048, BF16), (2049, BF16), (6144, BF16), (6145, BF16), (8192, BF16),
                                     (8193, BF16), (24577, BF16), (1024, F32), (4097, F32), (12289, F32)])
def test_short_rows(rows, V, dtype):
    """Row lengths and counts on either side of the rule that picks a row's threads, ties among them."""
    print(f"short rows={rows} V={V} {dtype}", flush=True)
    x, t = logits(rows, V, dtype, rows + V)
    x[1] = (x[1].float() * 2).round().to(dtype) / 2          # few values
    x[2, 7:] = -math.inf
    t[2] = 3
    x[3] = 0.5
    x = x.cuda()
    for top in (0, 9, 64):
        o = score(x, t, top=top)
        pick = [0, 1, 2, 3, rows - 1]
        check(x[pick], t[pick], {k: v[pick] for k, v in o.items()}, top=top)


@pytest.mark.parametrize("rows,V,dtype", [(768, 24576, BF16), (769, 24577, BF16), (769, 102400, BF16), (1535, 102401, BF16),
                                          (1535, 8193, BF16), (1536, 8193, BF16), (1536, 102400, BF16), (4096, 102401, BF16),
                                          (4096, 32769, BF16), (4097, 32769, BF16), (4097, 32768, BF16), (1700, 51200, F32)])
def test_many_rows(rows, V, dtype):
    """Row counts and lengths on either side of the rule that picks a row's threads, and numbers of alternatives
    on either side of its limit."""
    print(f"many rows={rows} V={V} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + V)
    x = torch.empty(rows, V, dtype=dtype, device="cuda").normal_(0.0, 2.5, generator=gen)
    t = torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(rows))
    x[1] = x[1].mul(2).round() / 2                           # few values
    x[2, 7:] = -math.inf
    t[2] = 3
    x[3] = 0.5
    pick = [0, 1, 2, 3, rows // 2, rows - 1]
    for top in (0, 40, 41, 64):
        o = score(x, t, top=top)
        check(x[pick], t[pick], {k: v[pick] for k, v in o.items()}, top=top)


@pytest.mark.parametrize("rows,V,dtype", [(1024, 8193, BF16), (1025, 8193, BF16), (1024, 24576, BF16), (1025, 24577, BF16),
                                          (2621, 51200, BF16), (2622, 51200, BF16), (1400, 100000, BF16), (1025, 300, F32)])
def test_rows_and_cache(rows, V, dtype):
    """Row counts on either side of the rule that picks a row's threads where the logits fit the last-level cache, and
    do not."""
    print(f"cache rows={rows} V={V} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + V)
    x = torch.empty(rows, V, dtype=dtype, device="cuda").normal_(0.0, 2.5, generator=gen)
    t = torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(rows))
    x[1] = x[1].mul(2).round() / 2
    x[2, 7:] = -math.inf
    t[2] = 3
    x[3, 5] = 60.0                                           # a near-certain token
    t[3] = 5
    pick = [0, 1, 2, 3, rows // 2, rows - 1]
    for top in (0, 17, 64):
        o = score(x, t, top=top)
        check(x[pick], t[pick], {k: v[pick] for k, v in o.items()}, top=top)
