"""examples/member_rollouts.py: the evaluation operators together, as a program
uses them, against the same model without a cache in float32."""
import importlib.util
import os

import pytest
import torch

import paper_2608_02391_amd as cp

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("member_rollouts", os.path.join(ROOT, "examples", "member_rollouts.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def dense_logits(model, tokens, window, sinks):
    """Logits behind every token of one sequence, attention over all of them at once in float32."""
    n = len(tokens)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    x = model.embed(torch.tensor(tokens, device="cuda"), pos)
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    seen = (j <= i) & ((j > i - window) | (j < sinks)) if window else j <= i
    for layer in range(model.layers):
        q, k, v = (t.float().transpose(0, 1).contiguous() for t in model.qkv(layer, x))
        group = model.q_heads // model.kv_heads
        k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
        s = (q @ k.transpose(1, 2).contiguous()) * model.head_dim ** -0.5
        p = s.masked_fill(~seen, float("-inf")).softmax(-1)
        x = model.after(layer, x, (p @ v).transpose(0, 1).to(torch.bfloat16))
    return model.logits(x)


@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 2)])
def test_generation_through_the_cache_matches_the_dense_model(ex, window, sinks):
    """Greedy rollouts (the first alternative): every token's log probability is the dense model's, up to the
    activations' bf16 roundings: 2^-8 of a residual stream of a few layers, a few times, on logits of order one."""
    model = ex.Decoder(layers=3)
    prompts = [[5, 900, 17], list(range(40, 75)), [1] * 16]
    batch = ex.Rollouts(model, 3, 2, 64, window=window, sinks=sinks, alternatives=8)
    tokens, logps, entropies = batch.generate(prompts, 10, torch.zeros(6, 10, device="cuda"))
    assert torch.equal(tokens[0::2], tokens[1::2]) and torch.equal(logps[0::2], logps[1::2])     # rollouts of one prompt
    for i, p in enumerate(prompts):
        out = tokens[2 * i].tolist()
        ref = torch.log_softmax(dense_logits(model, p + out[:-1], window, sinks).float(), -1)[len(p) - 1:]
        got, want = logps[2 * i], ref[torch.arange(10), tokens[2 * i]]
        assert float((got - want).abs().max()) < 0.1, (i, got, want)
        assert float((want - ref.amax(-1)).min()) > -0.1                                          # the most likely token
        assert float((entropies[2 * i] + (ref.exp() * ref).sum(-1)).abs().max()) < 0.1
    assert int(batch.refs.sum()) > int((batch.refs > 0).sum())                                    # pages are shared
    # some rollouts end, the rest goes on from packed pages and says the same
    before = batch.step(batch.child_ids[:2], tokens[:2, -1], torch.tensor([12, 12], dtype=torch.int32, device="cuda"))
    batch.lengths[batch.child_ids[:2].long()] -= 1
    batch.drop(batch.child_ids[2:])
    live = int((batch.refs > 0).sum())
    assert int(batch.refs[:live].min()) > 0 and not bool(batch.refs[live:].any())
    after = batch.step(batch.child_ids[:2], tokens[:2, -1], torch.tensor([12, 12], dtype=torch.int32, device="cuda"))
    assert torch.equal(before, after)
    batch.clear()
    assert not bool(batch.refs.any()) and not bool(batch.lengths.any())


def test_training_steps(ex):
    """Members leave the weights as they were; a step's update changes its subspace alone."""
    lines = []
    means = ex.train(steps=2, members=4, prompts=2, each=2, new_tokens=5, report=lines.append)
    assert len(means) == 2 and len(lines) == 2 and all(0 <= m + 0.1 <= 1.2 for m in means)
    model = ex.Decoder()
    before = model.flat.clone()
    sub = cp.subspace(1000, 5000)
    backup = torch.empty(5000, dtype=torch.bfloat16, device="cuda")
    batch = ex.Rollouts(model, 1, 2, 32)
    plain = batch.generate([[1, 2, 3]], 4, torch.zeros(2, 4, device="cuda"))
    batch.clear()
    cp.cpes_perturb(model.flat, sub, 0.05, 7, 1, aux=backup, aux_mode=cp.AUX_SNAPSHOT)
    batch.generate([[1, 2, 3]], 4, torch.zeros(2, 4, device="cuda"))
    batch.clear()
    cp.cpes_restore(model.flat, sub, aux=backup, aux_mode=cp.AUX_SNAPSHOT)
    assert torch.equal(model.flat, before)
    again = batch.generate([[1, 2, 3]], 4, torch.zeros(2, 4, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(plain, again))
