"""examples/member_rollouts.py: a page call that failed is reported, whatever calls came behind it."""
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


def test_a_failed_page_call_is_not_forgotten(ex):
    """Two prompts and one page: the first token of both finds no room, the second token of the longer one does."""
    model = ex.Decoder(layers=1)
    batch = ex.Rollouts(model, 2, 1, 16, pages=1, alternatives=4)
    for page in (batch.k, batch.v):
        page.zero_()                       # what a step reads where no token was entered
    with pytest.raises(RuntimeError, match=f"status {cp.PAGES_SHORT}"):
        batch.prefill([[5], [7, 9]])
        batch.check()
    batch.clear()
    batch.check()                          # reported once
    assert not bool(batch.refs.any())


def test_enough_pages_raise_nothing(ex):
    model = ex.Decoder(layers=1)
    batch = ex.Rollouts(model, 2, 2, 24, alternatives=4)
    tokens, _, _ = batch.generate([[5], [7, 9, 11]], 4, torch.zeros(4, 4, device="cuda"))
    assert tokens.shape == (4, 4)
    batch.drop(batch.child_ids)
    batch.clear()
    batch.check()
