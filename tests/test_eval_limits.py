"""What the evaluation operators' host side promises beside refusals: workspaces that serve fewer rows, messages that
name the argument.  Nothing is launched here."""
import pytest
import torch

import paper_2608_02391_amd as cp


@pytest.mark.parametrize("vocab", [100, 50257, 65536, 151936, 1 << 20])
@pytest.mark.parametrize("top", [0, 1, 20, 64])
def test_a_score_workspace_serves_fewer_rows(vocab, top):
    """A batch loses rows as its rollouts end: what was enough for the largest is enough for all below."""
    most = 0
    for rows in range(0, 600):
        need = cp.cpes_logprobs_workspace_bytes(rows, vocab, top)
        assert need >= most, (rows, need, most)
        most = need
    for rows in (4096, 1 << 20, 2 ** 31 - 1):
        assert cp.cpes_logprobs_workspace_bytes(rows, vocab, top) == most


def test_a_score_workspace_serves_fewer_alternatives():
    for rows in (1, 32, 48, 256, 1000):
        sizes = [cp.cpes_logprobs_workspace_bytes(rows, 151936, top) for top in range(65)]
        assert sizes == sorted(sizes)


def test_an_attention_workspace_serves_fewer_rows():
    for heads in ((8, 2, 64), (32, 8, 128), (33, 1, 256)):
        sizes = [cp.cpes_attend_workspace_bytes(rows, *heads) for rows in range(0, 300)]
        assert sizes == sorted(sizes) and sizes[0] > 0


class FakeGpu:
    """A host tensor that says it is on the GPU, to reach the checks behind that one."""

    def __init__(self, t):
        self.t = t

    is_cuda = True

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_messages_name_what_has_the_wrong_type():
    half = lambda *s: FakeGpu(torch.zeros(*s, dtype=torch.float16))
    with pytest.raises(TypeError, match="^keys and values must be bfloat16 or float32, not torch.float16"):
        cp.paged_cache(half(1, 2, 2, 4, 8), half(1, 2, 2, 4, 8))
    with pytest.raises(TypeError, match="^logits must be bfloat16 or float32, not torch.float16"):
        cp.cpes_logprobs(half(2, 9), None, None)
    with pytest.raises(TypeError, match="^logits must be bfloat16 or float32, not torch.float16"):
        cp.cpes_logprobs_backward(half(2, 9), None, None, None, None, None, half(2, 9))
    with pytest.raises(TypeError, match="^weights must be bfloat16 or float32, not torch.float16"):
        cp.cpes_perturb(half(16), cp.subspace(0, 16), 0.1, 1, 1)
