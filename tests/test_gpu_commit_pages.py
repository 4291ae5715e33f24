"""Commits to pages outside the pool, and past the cache's end: the call reports them, the
sequence keeps its cache and its context length, and the others are committed."""
import pytest
import torch

from test_gpu_verify8 import _setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [0, 16])
def test_step8_reports_a_path_past_the_end(page):
    """A cache with room for the root alone: a longer path is not committed, and the step says
    so."""
    case, dims, t, step, cache, _ = _setup(page=page, ctx=(500, 1535, 0, 1300), seed=page + 1, tau=1e-20)
    before = [getattr(cache, x).clone() for x in ("k", "v", "k_exp", "v_exp")]
    out = step.run()
    torch.cuda.synchronize()
    assert (out["accept"] == 1).all()                    # every path is the tree's depth
    assert step.device_status() == 5
    got = out["ctx_len_out"].tolist()
    assert got[1] == 1535 and got[0] > 500 and got[3] > 1300
    for x, was in zip(("k", "v", "k_exp", "v_exp"), before):
        now = getattr(cache, x)
        mine = case.table[1] if page else 1
        assert torch.equal(now[mine], was[mine]), x
