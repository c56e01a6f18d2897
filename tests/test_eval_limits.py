"""What the evaluation operators' host side promises beside refusals: workspaces that serve fewer rows.  Nothing is
launched here."""
import pytest

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
