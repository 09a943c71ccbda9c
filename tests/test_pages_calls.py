"""Selected pages and drafted tokens, called in the other ways that their documentation allows (GPU)."""
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2412_07017_b200 import binding as B
from cache_util import Cache, check
from test_draft_verify import Case
from test_select_pages import as_mask, chosen_pages, update_bounds

pytestmark = pytest.mark.gpu


def selected(heads, kv8=False, **options):
    c = Cache(heads, [3000, 15, 700, 9000], [1, 2, 4, 1], kv8=kv8, seed=4)
    plan = B.asynclm_plan_sparse(*c.args, 24, 1, 2, kv8=kv8, **options)
    bounds = torch.zeros((c.num_pages, c.hkv, 2, c.d), dtype=torch.bfloat16, device="cuda")
    update_bounds(c, plan, bounds, True)
    B.asynclm_select_pages(plan, c.q, bounds)
    return c, plan, bounds, as_mask(c, chosen_pages(c, c.bounds().nan_to_num(0.0), 24, 1, 2))


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 4, 64)])
def test_selected_pages_in_the_fixed_scratch(heads):
    c, plan, _, mask = selected(heads)
    got = c.attend(plan)
    check(got, c.exact(mask))
    static = c.attend(plan, call=lambda p, q, pool, out, lse: B.asynclm_attn_mixed_static(p, q, pool, out, lse))
    assert torch.equal(got[0], static[0]) and torch.equal(got[1], static[1])


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("num_sms", [1, 5])
def test_selected_pages_on_few_sms(num_sms, kv8):
    c, plan, _, mask = selected((32, 8, 128), kv8, num_sms=num_sms)
    check(c.attend(plan), c.exact(mask))


def test_selected_pages_and_another_scale():
    c, plan, bounds, mask = selected((8, 1, 128))
    scaled = B.asynclm_plan_sparse(*c.args, 24, 1, 2, sm_scale=0.5 * c.d ** -0.5)
    B.asynclm_select_pages(scaled, c.q, bounds)      # (the scale is positive: the same choice)
    got = c.attend(scaled)
    c.q.mul_(0.5)                                    # exact in bf16
    check(got, c.exact(mask))


def test_a_budget_of_every_page_is_the_ordinary_attention():
    c = Cache((32, 8, 128), [900, 31, 2000], [1, 3, 2], seed=8)
    plan, ordinary = B.asynclm_plan_sparse(*c.args, 200, 1, 1), B.asynclm_plan(*c.args)
    bounds = torch.zeros((c.num_pages, 8, 2, 128), dtype=torch.bfloat16, device="cuda")
    B.asynclm_select_pages(plan, c.q, bounds)
    want = c.exact()
    check(c.attend(plan), want)
    check(c.attend(ordinary), want)


def test_two_selections_at_once():
    """Two plans on two streams, each with its own workspace, over one cache and its bounds."""
    c, first, bounds, mask = selected((32, 8, 128))
    second = B.asynclm_plan_sparse(*c.args, 24, 1, 2)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    outs = [(torch.empty_like(c.q), torch.empty((c.total, c.hq), device="cuda")) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, plan, (out, lse) in zip(streams, (first, second), outs):
            with torch.cuda.stream(s):
                B.asynclm_select_pages(plan, c.q, bounds)
                c.attend(plan, out, lse)
    torch.cuda.synchronize()
    want = c.exact(mask)
    for got in outs:
        check(got, want)


def test_two_verifications_at_once():
    cases = [Case([3, 0, 5] * 20, 30000, seed=1), Case([1, 2] * 40, 50001, torch.bfloat16, seed=2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                c.call()
    torch.cuda.synchronize()
    for c in cases:
        assert (c.accepted.cpu().tolist(), c.out.cpu().tolist()) == c.want()


def test_the_most_sequences():
    c = Case([1] + [0] * 65534, 3, with_draft=False)
    c.check()
    one_more = Case([0] * 65536, 3, with_draft=False)
    with pytest.raises(B.AsynclmError) as e:
        one_more.call()
    assert e.value.status == -1


@pytest.mark.parametrize("indptr", [[0, 5, 2, 6], [3, 3, 99, 6], [-7, 2, 4, 6], [6, 6, 6, 6], [0, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 6, 0]])
def test_rows_that_are_no_rows(indptr):
    """draft_indptr is device memory and held to the drafts that there are: some tokens of the vocabulary, and nothing else is written."""
    c = Case([2, 2, 2], 700, seed=3)
    c.indptr.copy_(torch.tensor(indptr, dtype=torch.int64).to(torch.int32))
    around = torch.full((c.out.numel() + 64,), 77, dtype=torch.int32, device="cuda")
    c.out = around[32:32 + c.out.numel()]
    c.out.fill_(-1)
    c.call()
    assert ((c.out >= -1) & (c.out < 700)).all() and (around[:32] == 77).all() and (around[32 + c.out.numel():] == 77).all()
    assert ((c.accepted >= 0) & (c.accepted <= 6)).all()
    c.indptr.copy_(torch.tensor([0, 2, 4, 6]))
    c.check()      # the workspace is fit for the next call


CHILD = """
import sys
sys.path.insert(0, "tests")
import torch
from test_draft_verify import Case
c = Case([3, 0, 2], 40000, {dtype}, {draft}, 5)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    c.call()
graph.replay()
torch.cuda.synchronize()
assert (c.accepted.cpu().tolist(), c.out.cpu().tolist()) == c.want()
print("ok")
"""


@pytest.mark.parametrize("dtype", ["torch.float32", "torch.bfloat16"])
@pytest.mark.parametrize("draft", [True, False])
def test_first_call_in_a_capture(dtype, draft):
    p = subprocess.run([sys.executable, "-c", CHILD.format(dtype=dtype, draft=draft)], capture_output=True, text=True, timeout=200, cwd=__file__.rsplit("/tests/", 1)[0])
    assert p.stdout.split() == ["ok"], p.stderr[-600:]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("heads,n,ctx", [((32, 8, 128), 64, 1500), ((8, 2, 64), 200, 300), ((8, 8, 64), 100, 40)])
def test_calls_one_behind_the_other(heads, n, ctx, kv8):
    """Attention, append, bounds and selection again and again under one plan, with nothing between them: every call sees what the ones in front of it wrote."""
    c = Cache(heads, ctx + np.arange(n) % 16, [1] * n, kv8=kv8, seed=3)
    plan = B.asynclm_plan_sparse(*c.args, 24, 1, 2, kv8=kv8)
    bounds = torch.zeros((c.num_pages, c.hkv, 2, c.d), dtype=torch.bfloat16, device="cuda")
    update_bounds(c, plan, bounds, True)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = [(torch.randn((c.total, c.hkv, c.d), generator=g, device="cuda") * 2.0 ** (i % 5 - 2)).bfloat16() for i in range(12)]      # (a row's scale differs from time to time)
    pages = torch.zeros((c.total, c.hkv, 24), dtype=torch.int32, device="cuda")
    B.asynclm_select_pages(plan, c.q, bounds, pages)
    out, lse = c.attend(plan)
    torch.cuda.synchronize()
    for i in range(0, 12, 3):
        for k in rows[i:i + 3]:
            c.attend(plan, out, lse)
            if kv8:
                B.asynclm_kv8_append(plan, k, k, c.pool, c.scales)
            else:
                B.asynclm_kv_append(plan, k, k, c.pool)
            update_bounds(c, plan, bounds, False)
            B.asynclm_select_pages(plan, c.q, bounds, pages)
        torch.cuda.synchronize()
        want, used = c.bounds(), c.used.any(-1)
        assert torch.equal(bounds[used].double(), want[used])
    assert pages.cpu().tolist() == [[h + [-1] * (24 - len(h)) for h in row] for row in chosen_pages(c, c.bounds().nan_to_num(0.0), 24, 1, 2)]
