"""Commits to pages outside the pool, and past the cache's end: the call reports them, the
sequence keeps its cache and its context length, and the others are committed."""
import numpy as np
import pytest
import torch

from _cases8 import Case, bf16
from test_gpu_kv8 import _append, _commit, _same
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


@pytest.mark.parametrize("page,B", [(8, 3), (16, 2), (64, 20)])
@pytest.mark.parametrize("which", ["first", "last"])
@pytest.mark.parametrize("value", [-1, "pages", 2 ** 31 - 1])
def test_commit8_writes_nothing_where_a_page_is_bad(page, B, which, value):
    """A path over several pages, one of them bad: no byte or scale of the sequence moves (its
    part-filled block would have been rescaled)."""
    from paper_2609_02897_gb300 import asd
    case = Case(page + B, [30] * B, [page + 5] * B, page=page, cap=-(-(page + 40) // page) * page, max_path=30)
    for b in range(B):                                   # chains, committed whole
        case.trees[b] = np.arange(-1, 29)
    case.nodes, case.T = [30] * B, 30 * B
    case.parent = np.concatenate(case.trees).astype(np.int32)
    case.cu = np.arange(0, 30 * B + 1, 30, dtype=np.int32)
    case.tree_k, case.tree_v = (bf16(10 * case._values((case.T, case.Hkv, case.D))) for _ in range(2))
    case.fill()
    at = (page + 5) // page if which == "first" else (page + 34) // page
    case.table[1, at] = case.num_pages if value == "pages" else value
    paths = [list(range(30))] * B
    cache, out, ws = _commit(case, paths)
    assert asd.asd_get_device_status(ws) == 5
    assert out.tolist() == [page + 5 if b == 1 else page + 35 for b in range(B)]
    _append(case, [p if b != 1 else [] for b, p in enumerate(paths)])
    _same(case, cache)


def test_step8_writes_nothing_where_a_page_is_bad():
    """The page that a step's path would begin in: reported, the other sequences committed."""
    case, dims, t, step, cache, _ = _setup(ctx=(500, 80, 0, 1300), seed=4, tau=1e-20)
    t["page_table"][1, 5] = case.num_pages
    before = [getattr(cache, x).clone() for x in ("k", "v", "k_exp", "v_exp")]
    out = step.run()
    torch.cuda.synchronize()
    assert step.device_status() == 5
    got = out["ctx_len_out"].tolist()
    assert got[1] == 80 and got[0] > 500 and got[3] > 1300
    mine = np.setdiff1d(case.table[1], [case.table[1, 5]])
    for x, was in zip(("k", "v", "k_exp", "v_exp"), before):
        now = getattr(cache, x)
        assert torch.equal(now[mine], was[mine]), x
