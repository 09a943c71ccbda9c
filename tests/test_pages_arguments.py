"""What the calls of selected pages and of drafted tokens refuse before anything is launched, both ways into the library.  No GPU: tensors are stand-ins, and a
plan made on the host only, which the C call refuses, shows that the tensors themselves were accepted."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200 import workload as W
from test_kv8_arguments import BF16, F32, I32, I64, STREAM, U8, Fake, accepted, refused, way  # noqa: F401

SHAPE, PAGES, TOKENS = W.Shape(8, 2, 64, 16), 9, 5
BATCH = ([0, 1, 4, 5], [20, 30, 0], [0, 2, 5, 6], [0, 1, 2, 3, 4, 5])
BOUNDS = (PAGES, 2, 2, 64)


@pytest.fixture(scope="module")
def plan():
    return B.plan_host(SHAPE, PAGES, *BATCH, sparse=(3, 1, 1))


def test_bounds(way, plan):  # noqa: F811
    pool, scales = Fake((PAGES, 2, 2, 16, 64)), Fake((PAGES, 2, 2, 16), U8)
    accepted(lambda: B.asynclm_kv_bounds(plan, pool, Fake(BOUNDS), stream=STREAM))
    accepted(lambda: B.asynclm_kv8_bounds(plan, Fake(pool.shape, U8), scales, Fake(BOUNDS), True, stream=STREAM))
    for bad in (Fake(BOUNDS, F32), Fake((PAGES - 1, 2, 2, 64)), Fake(BOUNDS, strides=(1, 2, 3, 4))):
        refused(lambda: B.asynclm_kv_bounds(plan, pool, bad, stream=STREAM), "key_bounds")
        refused(lambda: B.asynclm_kv8_bounds(plan, Fake(pool.shape, U8), scales, bad, stream=STREAM), "key_bounds")
    refused(lambda: B.asynclm_kv_bounds(plan, Fake((PAGES + 1, 2, 2, 16, 64)), Fake(BOUNDS), stream=STREAM), "kv_pool")
    refused(lambda: B.asynclm_kv_bounds(plan, Fake(pool.shape, U8), Fake(BOUNDS), stream=STREAM), "kv_pool")
    refused(lambda: B.asynclm_kv8_bounds(plan, Fake(pool.shape, U8), Fake((PAGES, 2, 2, 15), U8), Fake(BOUNDS), stream=STREAM), "kv8_scales")


def test_select(way, plan):  # noqa: F811
    q, out = Fake((TOKENS, 8, 64)), Fake((TOKENS, 2, 3), I32)
    accepted(lambda: B.asynclm_select_pages(plan, q, Fake(BOUNDS), out, stream=STREAM))
    accepted(lambda: B.asynclm_select_pages(plan, q, Fake(BOUNDS), stream=STREAM))
    refused(lambda: B.asynclm_select_pages(plan, Fake((TOKENS, 8, 63)), Fake(BOUNDS), stream=STREAM), "q")
    refused(lambda: B.asynclm_select_pages(plan, q, Fake(BOUNDS, F32), stream=STREAM), "key_bounds")
    refused(lambda: B.asynclm_select_pages(plan, q, Fake(BOUNDS), Fake((TOKENS, 2, 4), I32), stream=STREAM), "pages_out")
    refused(lambda: B.asynclm_select_pages(plan, q, Fake(BOUNDS), Fake((TOKENS, 2, 3), I64), stream=STREAM), "pages_out")
    ordinary = B.plan_host(SHAPE, PAGES, *BATCH)
    accepted(lambda: B.asynclm_select_pages(ordinary, q, Fake(BOUNDS), stream=STREAM))      # (the C call says that the plan is of another kind)


def test_verify(way):  # noqa: F811
    batch, drafts, vocab = 2, 5, 100
    good = dict(draft_indptr=Fake((batch + 1,), I32), target=Fake((drafts + batch, vocab), F32), draft=Fake((drafts, vocab), F32), draft_tokens=Fake((drafts,), I32),
                accept_u=Fake((drafts,), F32), sample_u=Fake((batch,), F32), accepted=Fake((batch,), I32), tokens_out=Fake((drafts + batch,), I32),
                workspace=Fake((B.draft_verify_workspace_bytes(batch, vocab),), U8))
    for name, bad, what in (("target", Fake((drafts + batch, vocab), torch.float16), "target"), ("target", Fake((drafts, vocab), F32), "target"),
                            ("target", Fake((drafts + batch, vocab), F32, (1, drafts + batch)), "target"), ("target", Fake((drafts + batch, vocab), F32, (50, 1)), "target"),
                            ("draft", Fake((drafts, vocab), BF16), "draft"), ("draft", Fake((drafts, vocab + 1), F32), "draft"),
                            ("draft", Fake((drafts, vocab), F32, (0, 1)), "draft"), ("draft_indptr", Fake((batch + 1,), I64), "draft_indptr"),
                            ("draft_indptr", Fake((batch + 2,), I32), "target"), ("draft_tokens", Fake((drafts,), I64), "draft_tokens"),
                            ("draft_tokens", Fake((drafts + 1,), I32), "target"), ("accept_u", Fake((drafts - 1,), F32), "accept_u"),
                            ("sample_u", Fake((batch,), BF16), "sample_u"), ("accepted", Fake((batch + 1,), I32), "accepted"),
                            ("tokens_out", Fake((drafts,), I32), "tokens_out"), ("workspace", Fake((1000,), U8), "workspace")):
        refused(lambda: B.asynclm_draft_verify(**{**good, name: bad}, stream=STREAM), what)


def test_c_calls_refuse():
    """From C: null pointers, sizes, strides, alignment."""
    lib, at = B.load(), 1 << 20
    rows = lambda **kw: ctypes.byref(B.CDraftRows(**{**dict(target=at, draft=at, target_stride=100, draft_stride=100, vocab=100, dtype=1), **kw}))      # noqa: E731
    call = lambda r, indptr=at, batch=2, drafts=5, tokens=at, au=at, su=at, acc=at, out=at, ws=at: lib.asynclm_draft_verify(      # noqa: E731
        r, indptr, batch, drafts, tokens, au, su, acc, out, ws, None)
    for kw in (dict(target=None), dict(vocab=0), dict(vocab=-1), dict(dtype=2), dict(target_stride=99), dict(draft_stride=99), dict(target=at + 2), dict(draft=at + 1),
               dict(vocab=2 ** 31 - 1, target_stride=2 ** 31, draft_stride=2 ** 31)):
        assert call(rows(**kw)) == -1, kw
    for kw in (dict(indptr=None), dict(batch=-1), dict(batch=65536), dict(drafts=-1), dict(tokens=None), dict(au=None), dict(su=None), dict(acc=None), dict(out=None),
               dict(ws=None), dict(ws=at + 8), dict(acc=at + 2), dict(batch=0)):
        assert call(rows(), **kw) == -1, kw
    assert call(None) == -1 and call(rows(), batch=0, drafts=0) == 0
    assert B.draft_verify_workspace_bytes(0, 10) == B.draft_verify_workspace_bytes(10, 0) == 0
    for handle in (None, B.plan_host(SHAPE, PAGES, *BATCH).handle):
        assert lib.asynclm_kv_bounds(handle, at, at, 0, None) == -1
        assert lib.asynclm_kv8_bounds(handle, at, at, at, 0, None) == -1
        assert lib.asynclm_select_pages(handle, at, at, None, None) == -1
        assert lib.asynclm_plan_get_sparse(handle, ctypes.byref(B.CSparse())) == -1
    pages = B.CSparse()
    plan = B.plan_host(SHAPE, PAGES, *BATCH, sparse=(3, 1, 1))
    assert lib.asynclm_plan_get_sparse(plan.handle, ctypes.byref(pages)) == 0 and (pages.budget_pages, pages.first_pages, pages.last_pages) == (3, 1, 1)


def test_groups_and_pages_of_the_binding():
    for groups in ([(0, 3)], [(0, 1, 2, 3)]):
        with pytest.raises(ValueError, match="groups"):
            B.plan_host(SHAPE, PAGES, *BATCH, groups=groups)
    with pytest.raises(ValueError, match="groups and sparse"):
        B.plan_host(SHAPE, PAGES, *BATCH, groups=[], sparse=(3, 1, 1))
    lib, out, ws = B.load(), ctypes.c_void_p(), np.zeros(1 << 14, np.int64)
    cs, co = B._cshape(SHAPE, PAGES), B._copts(num_sms=148)
    cb, _keep = B._cbatch(*BATCH)
    front, back = (ctypes.byref(cs), ctypes.byref(co), ctypes.byref(cb)), (ws.ctypes.data, ws.nbytes, None, 0, None, ctypes.byref(out))
    assert lib.asynclm_plan_prefix(*front, None, 1, *back) == -1 and lib.asynclm_plan_prefix(*front, None, -1, *back) == -1
    assert lib.asynclm_plan_prefix(*front, None, 0, *back) == 0
    assert lib.asynclm_plan_sparse(*front, None, *back) == -1
    assert lib.asynclm_plan_sparse(*front, ctypes.byref(B.CSparse(3, 1, 1, 7)), *back) == -1
    assert lib.asynclm_plan_prefix(*front, (B.CPrefixGroup * 1)(B.CPrefixGroup(0, 2, 16, 1)), 1, *back) == -1
