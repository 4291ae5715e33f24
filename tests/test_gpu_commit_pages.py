"""Commits to pages outside the pool, and past the cache's end: the call reports them, the
sequence keeps its cache and its context length, and the others are committed."""
import numpy as np
import pytest
import torch

from _cases8 import Case, bf16, dev
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


def _setup16(page, ctx, seed):
    """The step of _setup with a bf16 cache and weight."""
    from paper_2609_02897_gb300 import asd
    case, dims, t, _, _, (h, w, tok) = _setup(page=page, ctx=ctx, seed=seed, tau=1e-20)
    step, b = asd.VerifyStep(dims, case.T), torch.bfloat16
    t.update(k_cache=dev(case.k16, b), v_cache=dev(case.v16, b), hidden=dev(h, b), w_lm=dev(w, b),
             tokens=dev(tok, torch.int32))
    return case, dims, t, step


def _no_path(out, b, ctx):
    """Sequence b of a step committed nothing."""
    assert out["path_len"][b] == 0 and (out["path"][b] == -1).all()
    assert out["bonus"][b] == -1 and out["n_promoted"][b] == 0 and out["ctx_len_out"][b] == ctx


@pytest.mark.parametrize("page,ctx", [(0, 1535), (16, 1535), (16, 80)])
def test_step_commits_nothing_where_slots_are_missing(page, ctx):
    """The path's end past the cache, or (context 80) its page outside the pool."""
    case, dims, t, step = _setup16(page, (500, ctx, 0, 1300), seed=page + ctx)
    if ctx == 80:
        t["page_table"][1, 5] = -7
    before = t["k_cache"].clone(), t["v_cache"].clone()
    out = step.bind(tau=1e-20, **t).run()
    torch.cuda.synchronize()
    assert step.device_status() == 5
    _no_path(out, 1, ctx)
    assert (out["path_len"][[0, 3]] > 1).all() and out["path_len"][2] == 1
    mine = np.setdiff1d(case.table[1], [case.table[1, 5]] if ctx == 80 else []) if page else 1
    assert torch.equal(t["k_cache"][mine], before[0][mine]) and torch.equal(t["v_cache"][mine], before[1][mine])


@pytest.mark.parametrize("page,B", [(8, 3), (16, 2), (64, 20)])
@pytest.mark.parametrize("which", ["first", "last"])
def test_commit_writes_nothing_where_a_page_is_bad(page, B, which):
    """The bf16 commit: a path over several pages, one of them bad."""
    from paper_2609_02897_gb300 import asd
    case = Case(page + B, [30] * B, [page + 5] * B, page=page, cap=-(-(page + 40) // page) * page, max_path=30)
    n = [min(len(t), 30) for t in case.trees]
    case.table[1, (page + 5) // page if which == "first" else (page + 4 + n[1]) // page] = case.num_pages
    dims, t, b16, i32 = case.dims(), case.tensors(), torch.bfloat16, torch.int32
    k, v = dev(case.k16, b16), dev(case.v16, b16)
    want = [k.clone(), v.clone()]
    path = torch.arange(30, dtype=i32, device="cuda").repeat(B, 1)
    out, ws = torch.zeros(B, dtype=i32, device="cuda"), asd.alloc_workspace(dims, case.T)
    asd.asd_kv_compact(dims, t["tree_k"], t["tree_v"], t["cu_nodes"], case.T, path, torch.tensor(n, dtype=i32).cuda(),
                       t["ctx_len"], t["page_table"], k, v, out, ws)
    assert asd.asd_get_device_status(ws) == 5
    assert out.tolist() == [page + 5 + (n[b] if b != 1 else 0) for b in range(B)]
    for b in range(B):
        for j in range(n[b] if b != 1 else 0):
            at = case.table[b, (page + 5 + j) // page], slice(None), (page + 5 + j) % page
            want[0][at], want[1][at] = t["tree_k"][case.cu[b] + j], t["tree_v"][case.cu[b] + j]
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_commit_context_lengths_at_the_end_of_the_range():
    """The largest and the smallest context lengths of the type: reported, nothing written."""
    from paper_2609_02897_gb300 import asd
    for page in (0, 16):
        case = Case(3, [5] * 3, [20] * 3, page=page, cap=64)
        dims, t, b16, i32 = case.dims(), case.tensors(), torch.bfloat16, torch.int32
        k, v = dev(case.k16, b16), dev(case.v16, b16)
        before = k.clone(), v.clone()
        lens = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 4], dtype=torch.int64, device="cuda").to(i32)
        path = torch.arange(case.max_path, dtype=i32, device="cuda").repeat(3, 1)
        out, ws = torch.zeros(3, dtype=i32, device="cuda"), asd.alloc_workspace(dims, case.T)
        plen = torch.full((3,), min(case.nodes + [case.max_path]), dtype=i32, device="cuda")
        asd.asd_kv_compact(dims, t["tree_k"], t["tree_v"], t["cu_nodes"], case.T, path, plen, lens,
                           t["page_table"], k, v, out, ws)
        assert asd.asd_get_device_status(ws) == 5
        assert torch.equal(out, lens) and torch.equal(k, before[0]) and torch.equal(v, before[1])


@pytest.mark.parametrize("page,ctx", [(0, 1535), (16, 1535), (16, 80)])
def test_step8_has_no_path_where_slots_are_missing(page, ctx):
    case, dims, t, step, cache, _ = _setup(page=page, ctx=(500, ctx, 0, 1300), seed=page + ctx, tau=1e-20)
    if ctx == 80:
        t["page_table"][1, 5] = -7
    out = step.run()
    torch.cuda.synchronize()
    assert step.device_status() == 5
    _no_path(out, 1, ctx)
    assert (out["path_len"][[0, 3]] > 1).all() and out["path_len"][2] == 1
