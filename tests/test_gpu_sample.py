"""Tokens drawn from rows of logits by given numbers, against a plain draw in 64 bits."""
import math

import numpy as np
import pytest
import torch

import draft_helpers as D
import paper_2608_02391_amd as cp

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# Weights are off by 2^-37.5 at most, those of a whole row's sum by as much again, and sums by some roundings of
# 64 bits: a draw nearer than this to a border (of the tokens, or of what top_p keeps), relative to the sum, may fall
# on either side.
NEAR = 2.0 ** -36


def run(x, u, top_k=0, top_p=1.0, min_p=0.0, scale=1.0, stream=None, logp=True):
    rows, vocab = x.shape
    ws = torch.full((cp.cpes_sample_workspace_bytes(rows, vocab),), 0xFF, dtype=torch.uint8, device="cuda")
    token = torch.full((rows,), -7, dtype=torch.int64, device="cuda")
    lp = torch.full((rows,), 77.0, device="cuda") if logp else None
    cp.cpes_sample(x, u, token, logp=lp, scale=scale, top_k=top_k, top_p=top_p, min_p=min_p, workspace=ws, stream=stream)
    return token, lp


def check(x, u, rows=None, **kw):
    """The draw of every row (or of some), but for those on a border; their number is returned."""
    token, logp = run(x, u, **kw)
    token, logp, host, hu, near = token.cpu(), logp.cpu(), x.double().cpu().numpy(), u.cpu().tolist(), 0
    for r in range(len(host)) if rows is None else rows:
        ref, ref_logp, margin = D.draw(host[r], hu[r], **kw)
        if margin < NEAR and int(token[r]) != ref:
            near += 1
            continue
        assert int(token[r]) == ref, (r, int(token[r]), ref, hu[r], margin, kw)
        if math.isnan(ref_logp):
            assert math.isnan(float(logp[r]))
        elif ref < 0:
            assert float(logp[r]) == ref_logp
        elif margin >= NEAR:
            # 64-bit sums as above, then one rounding to 32 bits
            assert abs(float(logp[r]) - ref_logp) <= 2.0 ** -24 * abs(ref_logp) + 2.0 ** -36, (r, float(logp[r]), ref_logp, kw)
    assert near <= 1
    return token, logp


def logits(rows, vocab, dtype, seed=0, std=2.5, likely=8):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * std
    for i in range(min(likely, vocab)):
        x[torch.arange(rows), torch.randint(0, vocab, (rows,), generator=g)] = 14.0 - 1.5 * math.log(i + 1) + 0.1 * torch.randn(rows, generator=g)
    return x.to(dtype).cuda(), torch.rand(rows, generator=g).cuda()


FILTERS = [dict(), dict(top_k=1), dict(top_k=7), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=20, top_p=0.8),
           dict(top_p=0.95, min_p=0.02, scale=0.7), dict(top_k=50, top_p=0.6, min_p=0.3, scale=1.5), dict(top_k=9, min_p=0.2),
           dict(scale=0.6), dict(top_p=0.3, scale=1.3), dict(min_p=1.0)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 300, 511, 2047, 2048, 2049, 8191, 8200, 32768, 50257])
def test_vocabularies(vocab, dtype):
    print(f"sample vocab={vocab} {dtype}", flush=True)
    for i, f in enumerate(FILTERS):
        x, u = logits(9, vocab, dtype, seed=vocab + i)
        check(x, u, **f)


@pytest.mark.parametrize("rows", [1, 2, 40, 256, 257, 600])
@pytest.mark.parametrize("filters", FILTERS[:7], ids=lambda f: ",".join(f) or "none")
def test_rows(rows, filters):
    """Rows cut into slices, and whole ones."""
    print(f"sample rows={rows} {filters}", flush=True)
    x, u = logits(rows, 40000, BF16, seed=rows)
    check(x, u, rows=range(0, rows, max(1, rows // 40)), **filters)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows", [3, 300])
def test_large_vocabulary(dtype, rows):
    x, u = logits(rows, 151936, dtype, seed=rows, likely=200)
    for f in FILTERS:
        check(x, u, rows=range(0, rows, max(1, rows // 12)), **f)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_a_vocabulary_of_a_million(dtype):
    for rows in (1, 4):
        x, u = logits(rows, 1 << 20, dtype, seed=rows, likely=200)
        for f in (dict(), dict(top_k=50), dict(top_p=0.9), dict(top_p=0.95, scale=0.3), dict(top_k=2000, top_p=0.7), dict(min_p=0.02)):
            check(x, u, **f)


@pytest.mark.parametrize("filters", [dict(top_p=0.95), dict(top_k=400), dict(top_k=3000), dict(top_k=1000, top_p=0.7), dict(min_p=0.001),
                                     dict(top_p=0.999, min_p=1e-4), dict(top_p=0.5, scale=0.25), dict(top_k=20000, min_p=0.01)],
                         ids=lambda f: ",".join(f"{k}={v}" for k, v in f.items()))
@pytest.mark.parametrize("dtype,rows,vocab", [(BF16, 5, 30000), (F32, 5, 30000), (BF16, 300, 9000), (F32, 300, 9001), (BF16, 2, 151936)])
def test_flat_rows(dtype, rows, vocab, filters):
    """Thousands of tokens stay: the bounding key is found by its digits."""
    print(f"sample flat {dtype} {rows}x{vocab} {filters}", flush=True)
    x, u = logits(rows, vocab, dtype, seed=vocab, likely=0)
    check(x, u, rows=range(0, rows, max(1, rows // 10)), **filters)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [100, 5000, 40000])
def test_ties(vocab, dtype):
    """Equal logits stay by the lowest token: all alike, few values, signs of zero."""
    g = torch.Generator().manual_seed(vocab)
    u = torch.rand(6, generator=g).cuda()
    same = torch.full((6, vocab), 1.25).to(dtype).cuda()
    few = torch.randint(0, 3, (6, vocab), generator=g).to(dtype).cuda()
    zeros = torch.where(torch.rand(6, vocab, generator=g) < 0.5, torch.tensor(0.0), torch.tensor(-0.0)).to(dtype).cuda()
    for x in (same, few, zeros):
        for f in [dict(), dict(top_k=1), dict(top_k=5), dict(top_k=vocab - 1), dict(top_p=0.25), dict(top_k=60, top_p=0.5), dict(min_p=1.0),
                  dict(min_p=0.9, top_k=3), dict(top_k=700, top_p=0.33)]:
            token, _ = check(x, u, **f)
            if f == dict(top_k=1):
                assert torch.equal(token, x.float().cpu().argmax(-1))


def last_kept(x, top_p):
    """(the last token that top_p of a row keeps, how near its border is, relative), of logits that fall with the token but
    for equal ones."""
    w = np.exp(x - x[0])
    upto = np.concatenate([[0.0], np.cumsum(w.astype(np.longdouble)).astype(np.float64)])
    enough = top_p * upto[-1]
    return int((upto[:-1] < enough).sum()) - 1, float(np.abs(upto - enough).min() / upto[-1])


@pytest.mark.parametrize("rows", [24, 260])
@pytest.mark.parametrize("behind,top_k", [(0, 0), (50000, 0), (50000, 151935)])
def test_a_cut_among_many_small_weights(behind, top_k, rows):
    """One likely token in front of some 100,000 equal fp32 logits, and others behind those: where top_p ends, their sum has
    to be right to its last bits, not each of them to as many as fit beside the likely one."""
    print(f"sample cut among small weights behind={behind} top_k={top_k} rows={rows}", flush=True)
    vocab = 151936
    rng = np.random.default_rng(behind)
    top_p = float(np.float32(0.9999 if behind else 0.93))
    found = []
    while len(found) < 24:
        # rows whose border lies between what sums of 44 bits a weight and what the call promises tell apart
        value = (-13.8 + 0.4 * rng.random(4000)).astype(np.float32)
        if not behind:
            # by the sum of equal ones, the candidates in the middle of that range
            w = np.exp(value.astype(np.float64))
            number = (top_p * (1 + (vocab - 1) * w) - 1) / w
            value = value[np.abs(np.log2(np.abs(number - number.round()) * w) + 32) < 2.5]
        x = np.full(vocab, value[0], dtype=np.float32)
        x[0] = 0.0
        if behind:
            x[-behind:] = np.sort((-18.0 - rng.random(behind)).astype(np.float32))[::-1]
        token, margin = last_kept(x.astype(np.float64)[:top_k or vocab], top_p)
        if 2.0 ** -35 < margin < 2.0 ** -29:
            found.append((x, token))
    x = torch.from_numpy(np.stack([f[0] for f in found])).repeat(-(-rows // 24), 1)[:rows].cuda()
    token, _ = run(x, torch.ones(rows, device="cuda"), top_p=top_p, top_k=top_k)
    assert token.tolist() == ([f[1] for f in found] * -(-rows // 24))[:rows]


def test_values_close_together():
    """fp32 logits that one bf16 number stands for."""
    g = torch.Generator().manual_seed(5)
    for sign in (1, -1):
        x = (sign * 5.0 + torch.rand(8, 20000, generator=g) * 2e-4).cuda()
        u = torch.rand(8, generator=g).cuda()
        for f in (dict(top_k=1), dict(top_k=3), dict(top_k=40), dict(top_k=300, top_p=0.5), dict(top_p=0.001), dict(top_p=0.5),
                  dict(top_k=50, scale=3e4), dict(min_p=0.9999), dict(top_p=0.9, scale=1e5), dict(scale=1e5)):
            check(x, u, **f)


@pytest.mark.parametrize("scale", [1e5, 1e6, 1e7])
@pytest.mark.parametrize("rows,vocab", [(48, 5000), (48, 40000), (300, 40000)])
def test_neighbours_that_are_octaves_apart(rows, vocab, scale):
    """fp32 logits a few steps of the type above those before them, which at a low temperature is octaves: the likelier
    ones come later in the row, in the same step of a wave, in the next and much later."""
    print(f"sample neighbours {rows}x{vocab} scale={scale}", flush=True)
    g = torch.Generator().manual_seed(rows + vocab)
    x = torch.randn(rows, vocab, generator=g)
    for r in range(rows):
        base = np.float32([10.0, 20.0, 31.0, 100.0, 600.0, -12.0, -100.0, 1000.0][r % 8])
        for place, ulps in ((5, 0), (300, 1 + r // 8 % 3), (1100, 2 + r // 8 % 5), (4500, 1 + r // 8)):
            y = base
            for _ in range(ulps):
                y = np.nextafter(y, np.float32(math.inf))
            x[r, place] = float(y)
        if base < 0:
            x[r][x[r] > -10.0] = 2.0 * float(base)
    x, u = x.cuda(), torch.rand(rows, generator=g).cuda()
    for f in (dict(), dict(top_p=0.9), dict(top_p=0.9999), dict(top_k=3), dict(min_p=0.01)):
        check(x, u, rows=range(min(rows, 48)), scale=scale, **f)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows", [12, 300])
def test_infinite_logits_behind_a_finite_base(rows, dtype):
    """A +inf, and one beside a NaN, long after the weights' base was found; the rows around are drawn as ever."""
    x, u = logits(rows, 40000, dtype, seed=13)
    x[1, 39000] = math.inf
    x[2, 30000], x[2, 30001] = math.nan, math.inf
    x[3, 30000], x[3, 30001] = math.inf, math.nan
    x[4, 700:] = math.inf
    x[5, 20000] = math.nan
    for f in (dict(), dict(top_p=0.9), dict(top_p=0.95, scale=0.2), dict(scale=1e6)):
        token, logp = check(x, u, rows=range(12), **f)
        assert token[1:6].tolist() == [-1] * 5 and bool(torch.isnan(logp[1:6]).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows", [12, 300])
def test_masks_and_broken_rows(dtype, rows):
    """-inf is never chosen; rows of nothing else, with NaN or +inf; the type's lowest value is a number."""
    x, u = logits(rows, 20000, dtype, seed=3)
    inf, lowest = math.inf, torch.finfo(dtype).min
    x[0] = -inf
    x[1, 7:] = -inf
    x[2, :19999] = -inf
    x[3, 100] = math.nan
    x[4, 19999] = inf
    x[5] = -inf
    x[5, 3] = math.nan
    x[6] = lowest
    x[6, ::3] = -inf
    x[7] = -inf
    x[7, 12345] = lowest
    x[8, ::2] = -inf
    x[9, 5000:] = lowest
    x[10, :] = -3e38
    x[10, 11] = 3e38
    x[11] = -inf
    x[11, 9000:9040] = 4.0
    for f in FILTERS + [dict(top_p=0.99, scale=0.25), dict(top_k=3000)]:
        token, logp = check(x, u, rows=range(12), **f)
        assert int(token[0]) == -1 and float(logp[0]) == -inf and token[3:6].tolist() == [-1, -1, -1]
        assert bool(torch.isnan(logp[3:6]).all()) and int(token[2]) == 19999 and int(token[7]) == 12345
        assert float(logp[2]) == 0.0 and float(logp[7]) == 0.0


@pytest.mark.parametrize("filters", [dict(), dict(top_k=4), dict(top_p=0.9), dict(top_p=0.95, scale=0.2), dict(min_p=0.1)],
                         ids=lambda f: ",".join(f) or "none")
def test_ends_of_the_uniform_numbers(filters):
    """0 and below, NaN, the last number below 1, 1 and above."""
    us = [0.0, -0.0, -3.0, math.nan, 1 - 2.0 ** -24, 1.0, 7.0, math.inf, -math.inf, 2.0 ** -149]
    for dtype in (BF16, F32):
        for rows in (10, 300):
            x, _ = logits(rows, 9000, dtype, seed=6)
            x[:, :2200] = -math.inf
            x[:, 8000:] = -math.inf
            u = torch.tensor((us * 30)[:rows]).cuda()
            token, _ = check(x, u, rows=range(10), **filters)
            assert int(token.min()) >= 2200 and int(token.max()) < 8000


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows", [5, 300])
def test_weights_at_the_edge_of_what_counts(rows, dtype):
    """Weights between 2^-56 and 2^-52 of the largest count as 0: where the number given ends among them, a token on
    either side is drawn, or the last; one of 2^-47 beside them is not lost."""
    print(f"sample edge rows={rows} {dtype}", flush=True)
    octave = math.log(2.0)

    def token_of(x, u):
        out, _ = run(x.to(dtype).repeat(rows, 1).cuda(), torch.full((rows,), u, device="cuda"))
        assert bool((out == out[0]).all())
        return int(out[0])

    for vocab in (3500, 40000, 100000):
        # nothing that counts lies between two pairs of the largest: half of the weight is in front of it
        x = torch.full((1, vocab), -54.0 * octave)
        x[0, 5] = x[0, 40] = x[0, vocab - 300] = x[0, vocab - 100] = 0.0
        assert token_of(x, 0.5) in (40, vocab - 300)
        assert token_of(x, 0.25) in (5, 40) and token_of(x, 0.75) in (vocab - 300, vocab - 100)
        # nor behind the last of them
        assert token_of(x, 1.0) == vocab - 100
        x[0, vocab - 300] = x[0, vocab - 100] = -54.0 * octave
        assert token_of(x, 1.0) == 40
        # the first token that counts stands behind others within 7 octaves that do not
        x = torch.full((1, vocab), -53.0 * octave)
        x[0, 2100] = -47.0 * octave
        x[0, vocab - 1] = 0.0
        assert token_of(x, 0.0) == 2100
        assert token_of(x, 2.0 ** -40) == vocab - 1


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 0.01, 30.0, 1e4, 1e20, 1.7e38])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_scales(scale, dtype):
    """From a uniform draw over what is not forbidden to the most likely token alone."""
    x, u = logits(6, 9000, dtype, seed=7)
    x[1, 4000:] = -math.inf
    x[2] *= 1e30
    x[3] *= 1e-30
    for f in (dict(), dict(top_k=6), dict(top_p=0.7), dict(min_p=0.5), dict(top_k=5, top_p=0.5)):
        check(x, u, scale=scale, **f)


def test_strides_alignment_and_missing_outputs():
    g = torch.Generator().manual_seed(8)
    for dtype in (BF16, F32):
        wide = torch.randn(7 * 3001 + 5, generator=g).to(dtype).cuda()
        x = wide[5:].view(7, 3001)[:, :2999]
        u = torch.rand(7, generator=g).cuda()
        for f in FILTERS:
            token, _ = check(x, u, **f)
            alone, _ = run(x, u, logp=False, **f)
            assert torch.equal(alone.cpu(), token)
    one = torch.randn(4000, generator=g).cuda()
    check(one[None], u[:1], top_k=30)
    check(one[None].expand(1, -1), u[:1])
    empty = torch.empty(0, 100, device="cuda")
    run(empty, torch.empty(0, device="cuda"))


def test_a_row_does_not_depend_on_the_others():
    """A row's draw is the same among few rows (cut into slices) and among many, but on a border."""
    x, u = logits(400, 30000, BF16, seed=9)
    for f in FILTERS:
        many, many_logp = run(x, u, **f)
        few, few_logp = run(x[:3], u[:3], **f)
        assert torch.equal(many[:3], few) and float((many_logp[:3] - few_logp).abs().max()) <= 2.0 ** -23 * float(few_logp.abs().max()) + 2.0 ** -36
        again, again_logp = run(x, u, **f)
        assert torch.equal(many, again) and torch.equal(many_logp, again_logp)


def test_draws_follow_the_distribution():
    """A grid of uniform numbers draws each token as often as its probability says, up to one."""
    x = torch.tensor([1.0, -math.inf, 3.0, 2.5, 0.0, 2.0], dtype=F32)
    n = 4096
    u = ((torch.arange(n) + 0.5) / n).float().cuda()
    token, logp = run(x.expand(n, -1).contiguous().cuda(), u, scale=0.8)
    p = torch.softmax(x.double() * float(np.float32(0.8)), -1)
    count = torch.bincount(token.cpu(), minlength=6)
    assert float((count - n * p).abs().max()) <= 1.0 + 1e-6
    assert bool((logp.cpu().double() - p.log()[token.cpu()]).abs().max() < 1e-6)


def test_captured_draws():
    """Replays read the logits and numbers of the moment; streams are respected."""
    for rows in (2, 300):
        x, u = logits(rows, 40000, BF16, seed=10)
        ws = torch.empty(cp.cpes_sample_workspace_bytes(rows, 40000), dtype=torch.uint8, device="cuda")
        for f in (dict(), dict(top_k=20, top_p=0.9), dict(top_p=0.9, scale=0.3)):
            token, logp = torch.empty(rows, dtype=torch.int64, device="cuda"), torch.empty(rows, device="cuda")
            cp.cpes_sample(x, u, token, logp=logp, workspace=ws, **f)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                cp.cpes_sample(x, u, token, logp=logp, workspace=ws, **f)
            for turn in range(3):
                fresh, fu = logits(rows, 40000, BF16, seed=20 + turn)
                x.copy_(fresh)
                u.copy_(fu)
                token.fill_(-9)
                graph.replay()
                torch.cuda.synchronize()
                eager, eager_logp = run(x, u, **f)
                assert torch.equal(token, eager) and torch.equal(logp, eager_logp)


def test_many_logits():
    """A row of more than 2^27 tokens, and rows that begin beyond 2^32 bytes."""
    n = (1 << 27) + 12345
    x = torch.zeros(1, n, dtype=BF16, device="cuda")
    x[0, n - 3] = 30.0
    token, logp = run(x, torch.tensor([0.5], device="cuda"))
    total = math.exp(-30.0) * (n - 1) + 1
    assert int(token) == n - 3 and abs(float(logp) + math.log(total)) < 1e-6
    token, _ = run(x, torch.tensor([0.5], device="cuda"), top_k=4, scale=1e-3)
    assert int(token) in (0, 1, 2, n - 3)
    token, _ = run(x[:, :1 << 27], torch.tensor([0.75], device="cuda"))
    assert int(token) == 3 << 25
    del x
    rows, vocab = 9, 1 << 28
    y = torch.zeros(rows, vocab, dtype=BF16, device="cuda")
    y[8, 99] = 40.0
    token, _ = run(y, torch.full((rows,), 0.5, device="cuda"))
    assert int(token[8]) == 99 and bool((token[:8] == vocab // 2).all())


def test_more_rows_than_are_taken_at_once():
    """8,192 rows are cut and kept together; the ones behind them draw from their own logits, strided."""
    x, u = logits(8192 + 37, 8300, BF16, seed=12)
    wide = torch.empty(8192 + 37, 8320, dtype=BF16, device="cuda")[:, :8300]
    wide.copy_(x)
    for f in (dict(), dict(top_k=20), dict(top_p=0.9)):
        check(wide, u, rows=[0, 1, 4095, 8190, 8191, 8192, 8193, 8200, 8228], **f)
