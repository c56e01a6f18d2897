"""A CoPES step whose members are evaluated by generating text: the weights are
perturbed in place, rollouts run on the perturbed model through a paged
key-value cache, their tokens are scored, the weights are restored, and the
seed-replayed update follows.

The model is a small decoder (grouped-query attention, RMS norms, a gated
feed-forward block) whose weights are views of the one flat buffer that
perturbation, restore and update work on; its projections are plain matrix
products, everything else that touches the cache or the logits goes through
``paper_2608_02391_amd``:

    prompts -> cpes_pages_reserve, then token by token cpes_cache_append, cpes_attend
    rollouts of a prompt -> cpes_pages_fork
    each new token -> cpes_pages_reserve, cpes_cache_append, cpes_attend, cpes_logprobs
    finished rollouts -> cpes_pages_free, cpes_pages_compact

    python examples/member_rollouts.py --steps 3 --members 16
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_02391_amd as cp  # noqa: E402

BF16, INT32 = torch.bfloat16, torch.int32


class Decoder:
    """Weights as views of one flat bf16 buffer; one token per row and call."""

    def __init__(self, vocab=1024, hidden=256, layers=2, q_heads=8, kv_heads=2, head_dim=64, inner=512, seed=1):
        self.vocab, self.hidden, self.layers, self.inner = vocab, hidden, layers, inner
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        shapes = {"embed": (vocab, hidden)}
        for i in range(layers):
            shapes[f"{i}.qkv"] = (hidden, (q_heads + 2 * kv_heads) * head_dim)
            shapes[f"{i}.out"] = (q_heads * head_dim, hidden)
            shapes[f"{i}.gate"] = shapes[f"{i}.up"] = (hidden, inner)
            shapes[f"{i}.down"] = (inner, hidden)
        self.flat = torch.empty(sum(math.prod(s) for s in shapes.values()), dtype=BF16, device="cuda")
        cp.cpes_fill_normal(self.flat, seed, stddev=0.06)
        self.w, at = {}, 0
        for name, shape in shapes.items():
            n = math.prod(shape)
            self.w[name] = self.flat[at:at + n].view(shape)
            at += n

    @staticmethod
    def norm(x):
        return x * torch.rsqrt(x.float().pow(2).mean(-1, keepdim=True) + 1e-6).to(x.dtype)

    def positions(self, pos):
        """Sinusoidal position code, float32 [rows, hidden]."""
        f = torch.exp(torch.arange(0, self.hidden, 2, device="cuda") * (-math.log(1e4) / self.hidden))
        a = pos[:, None].float() * f
        return torch.cat([a.sin(), a.cos()], -1)

    def qkv(self, layer, x):
        y = (self.norm(x) @ self.w[f"{layer}.qkv"]).view(len(x), -1, self.head_dim)
        return y[:, :self.q_heads], y[:, self.q_heads:-self.kv_heads], y[:, -self.kv_heads:]

    def after(self, layer, x, heads):
        """The residual stream behind a layer's attention (heads [rows, q_heads, head_dim])."""
        x = x + heads.reshape(len(x), -1) @ self.w[f"{layer}.out"]
        y = self.norm(x)
        return x + (torch.nn.functional.silu(y @ self.w[f"{layer}.gate"]) * (y @ self.w[f"{layer}.up"])) @ self.w[f"{layer}.down"]

    def embed(self, tokens, pos):
        return self.w["embed"][tokens] + self.positions(pos).to(BF16)

    def logits(self, x):
        return self.norm(x) @ self.w["embed"].t()


class Rollouts:
    """The paged cache of a batch: `prompts` sequences and `each` rollouts of every one."""

    def __init__(self, model, prompts, each, longest, page_size=16, pages=None, window=0, sinks=0, alternatives=16):
        self.model, self.prompts, self.each, self.alternatives = model, prompts, each, alternatives
        self.window, self.sinks = window, sinks
        S, width = prompts * (1 + each), -(-longest // page_size)
        pages = pages or S * width
        shape = (model.layers, pages, model.kv_heads, page_size, model.head_dim)
        self.k, self.v = (torch.empty(shape, dtype=BF16, device="cuda") for _ in range(2))
        self.table = torch.full((S, width), -1, dtype=INT32, device="cuda")
        self.lengths, self.refs = (torch.zeros(n, dtype=INT32, device="cuda") for n in (S, pages))
        self.cache, self.pool = cp.paged_cache(self.k, self.v), cp.page_pool(self.table, self.lengths, page_size, self.refs)
        rows = max(prompts, prompts * each)
        self.page_ws = torch.empty(cp.cpes_pages_workspace_bytes(pages), dtype=torch.uint8, device="cuda")
        self.attend_ws = torch.empty(cp.cpes_attend_workspace_bytes(rows, model.q_heads, model.kv_heads, model.head_dim),
                                     dtype=torch.uint8, device="cuda")
        self.score_ws = torch.empty(cp.cpes_logprobs_workspace_bytes(rows, model.vocab, alternatives), dtype=torch.uint8,
                                    device="cuda")
        self.status, self.worst = (torch.zeros(1, dtype=INT32, device="cuda") for _ in range(2))
        self.moved = torch.zeros(1, dtype=INT32, device="cuda")
        self.prompt_ids = torch.arange(prompts, dtype=INT32, device="cuda")
        self.child_ids = torch.arange(prompts, S, dtype=INT32, device="cuda")
        self.parents = self.prompt_ids.repeat_interleave(each)

    def note(self):
        """A page call writes its own status over the last one's: the worst since the last check is kept beside it."""
        torch.maximum(self.worst, self.status, out=self.worst)

    def check(self):
        """Whether a page call has failed since the last check (a synchronisation: where a program may wait)."""
        worst = int(self.worst)
        if worst != cp.PAGES_OK:
            self.worst.zero_()
            raise RuntimeError(f"page call failed with status {worst}")

    def step(self, seqs, tokens, pos):
        """One new token for each listed sequence, at positions `pos`: logits [rows, vocabulary]."""
        m, rows = self.model, len(seqs)
        cp.cpes_pages_reserve(self.pool, seqs, pos + 1, self.page_ws, status=self.status)
        self.note()
        x = m.embed(tokens, pos)
        heads = torch.empty(rows, m.q_heads, m.head_dim, dtype=BF16, device="cuda")
        for layer in range(m.layers):
            q, k, v = m.qkv(layer, x)
            cp.cpes_cache_append(self.cache, layer, self.pool, k, v, pos, seqs=seqs)
            cp.cpes_attend(self.cache, layer, self.pool, q, heads, seqs=seqs, window=self.window, sinks=self.sinks,
                           workspace=self.attend_ws)
            x = m.after(layer, x, heads)
        return m.logits(x)

    def score(self, logits, targets=None, scale=1.0):
        """(log probabilities of targets or None, entropies, alternatives' log probabilities and tokens)"""
        f = lambda *shape: torch.empty(*shape, device="cuda")
        rows = len(logits)
        logp, entropy = f(rows) if targets is not None else None, f(rows)
        top = f(rows, self.alternatives), torch.empty(rows, self.alternatives, dtype=torch.int64, device="cuda")
        cp.cpes_logprobs(logits, targets, logp, entropy=entropy, top_logp=top[0], top_ids=top[1], scale=scale, workspace=self.score_ws)
        return logp, entropy, *top

    def prefill(self, prompts):
        """Prompts (lists of tokens) enter the cache; logits behind each one's last token."""
        lens = [len(p) for p in prompts]
        last = [None] * len(prompts)
        for t in range(max(lens)):
            live = [i for i, n in enumerate(lens) if n > t]
            seqs = torch.tensor(live, dtype=INT32, device="cuda")
            logits = self.step(seqs, torch.tensor([prompts[i][t] for i in live], device="cuda"), torch.full_like(seqs, t))
            for row, i in enumerate(live):
                if lens[i] == t + 1:
                    last[i] = logits[row]
        return torch.stack(last)

    def generate(self, prompts, new_tokens, uniforms, temperature=1.0):
        """(tokens [rollouts, new_tokens], their log probabilities, entropies); uniforms (same shape) in [0, 1)
        pick among the alternatives."""
        logits = self.prefill(prompts).repeat_interleave(self.each, 0)
        cp.cpes_pages_fork(self.cache, self.pool, self.parents, self.child_ids, self.page_ws, status=self.status)
        self.note()
        self.check()
        pos = torch.tensor([len(p) for p in prompts], dtype=INT32, device="cuda").repeat_interleave(self.each)
        tokens, logps, entropies = [], [], []
        for t in range(new_tokens):
            _, entropy, top_logp, top_ids = self.score(logits, scale=1.0 / temperature)
            mass = top_logp.exp().cumsum(-1)
            pick = (mass < uniforms[:, t:t + 1] * mass[:, -1:]).sum(-1, keepdim=True).clamp(max=self.alternatives - 1)
            tokens.append(top_ids.gather(1, pick)[:, 0])
            logps.append(top_logp.gather(1, pick)[:, 0])
            entropies.append(entropy)
            if t + 1 < new_tokens:
                logits = self.step(self.child_ids, tokens[-1], pos + t)
        self.check()
        return torch.stack(tokens, 1), torch.stack(logps, 1), torch.stack(entropies, 1)

    def drop(self, seqs):
        """Sequences end; the pages that stay move to the front of the cache."""
        cp.cpes_pages_free(self.pool, seqs, status=self.status)
        self.note()
        cp.cpes_pages_compact(self.cache, self.pool, self.pool, self.page_ws, moved=self.moved)

    def clear(self):
        cp.cpes_pages_free(self.pool, torch.arange(len(self.lengths), dtype=INT32, device="cuda"), status=self.status)
        self.note()


def reward(tokens, logps, goal):
    """Share of a rollout's tokens below `goal`, plus a little for confidence: a stand-in for a verifier."""
    return (tokens < goal).float().mean(-1) + 0.01 * logps.mean(-1)


def train(steps=2, members=8, subspaces=4, prompts=4, each=4, new_tokens=12, seed=0, report=print):
    """CoPES steps on contiguous subspaces; returns the mean reward of every step."""
    model = Decoder()
    g = torch.Generator().manual_seed(seed)
    texts = [torch.randint(0, model.vocab, (int(n),), generator=g).tolist() for n in torch.randint(3, 40, (prompts,), generator=g)]
    batch = Rollouts(model, prompts, each, max(map(len, texts)) + new_tokens, window=32, sinks=4)
    uniforms = torch.rand(prompts * each, new_tokens, generator=g).cuda()
    d = model.flat.numel()
    offsets = cp.cpes_partition(cp.PART_CONTIGUOUS, d, subspaces)
    rewards, rnorm = torch.empty(members, device="cuda"), torch.empty(members, device="cuda")
    means = []
    for step in range(steps):
        k = step % subspaces
        length = offsets[k + 1] - offsets[k]
        sub, sigma = cp.subspace(offsets[k], length), 2e-3 * math.sqrt(d / length)
        backup = torch.empty(length, dtype=BF16, device="cuda")
        seeds = [1000 * step + i + 1 for i in range(members)]
        for i, s in enumerate(seeds):
            cp.cpes_perturb(model.flat, sub, sigma, s, 1, aux=backup if i == 0 else None,
                            aux_mode=cp.AUX_SNAPSHOT if i == 0 else cp.AUX_NONE)
            tokens, logps, _ = batch.generate(texts, new_tokens, uniforms)
            rewards[i] = reward(tokens, logps, model.vocab // 4).mean()
            batch.clear()                      # another member's keys and values are worth nothing
            cp.cpes_restore(model.flat, sub, aux=backup, aux_mode=cp.AUX_SNAPSHOT)
        cp.cpes_normalize_rewards(rewards, rnorm, cp.NORM_Z)
        cp.cpes_update(model.flat, sub, seeds, [1] * members, rnorm, 2e-3, sigma)
        means.append(float(rewards.mean()))
        report(f"step {step}: subspace {k}, mean reward {means[-1]:.4f}, best {float(rewards.max()):.4f}")
    return means


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=3)
    ap.add_argument("--members", type=int, default=16)
    ap.add_argument("--rollouts", type=int, default=4, help="of each prompt")
    ap.add_argument("--tokens", type=int, default=12, help="generated by each rollout")
    a = ap.parse_args()
    train(steps=a.steps, members=a.members, each=a.rollouts, new_tokens=a.tokens)


if __name__ == "__main__":
    main()
