"""The selection of pages where its form changes with the row's length, where scores cancel, and where calls are repeated (GPU)."""
import numpy as np
import pytest
import torch

from paper_2412_07017_b200 import binding as B
from cache_util import PAGE, Cache, check
from test_select_pages import as_mask, chosen_pages, update_bounds

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", [[1024], [1025], [2048], [2049], [4096], [4097], [1024, 4097], [2048, 1025, 4100, 9]])
@pytest.mark.parametrize("heads", [(4, 1, 64), (2, 2, 128)])
def test_lengths_at_which_the_choice_changes(pages, heads):
    """Keys of up to 128, 256 and 512 threads in registers, or in memory; rows of several kinds under one plan.  The last page has one key."""
    c = Cache(heads, [(n - 1) * PAGE for n in pages], [1] * len(pages), seed=pages[0])
    plan = B.asynclm_plan_sparse(*c.args, 40, 1, 2)
    bounds = torch.zeros((c.num_pages, c.hkv, 2, c.d), dtype=torch.bfloat16, device="cuda")
    update_bounds(c, plan, bounds, True)
    chosen = torch.full((c.total, c.hkv, 40), 99, dtype=torch.int32, device="cuda")
    B.asynclm_select_pages(plan, c.q, bounds, chosen)
    lists = chosen_pages(c, c.bounds().nan_to_num(0.0), 40, 1, 2)
    assert chosen.cpu().tolist() == [[h + [-1] * (40 - len(h)) for h in row] for row in lists]
    check(c.attend(plan), c.exact(as_mask(c, lists)))


@pytest.mark.parametrize("step", range(0, 31, 2))
@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_cancel(d, step):
    """Products of about 2^20 that cancel in pairs, in an order that differs from page to page, and one more by which the scores differ, 64 to 255 times 2^(14 - step): from
    beyond the bound of the tensor cores' error, 2^-14 of the sum of magnitudes (2^12 or 2^13 here), to far below the steps of a sum in 32 bits (1/8 at 2^20)."""
    c = Cache((2, 2, d), [16 * 600, 16 * 1500], [1, 1], seed=step)
    r = np.random.RandomState(step)
    sign = r.choice([-1.0, 1.0], (2, 2, d))      # queries
    bounds = np.zeros((c.num_pages, 2, 2, d))
    rows = np.zeros(c.num_pages, int)
    rows[c.ids[c.indptr[1]:]] = 1
    for page in range(c.num_pages):
        for h in range(2):
            at, x = r.permutation(d), np.zeros(d)
            most = 2.0 ** 20 * (1 + r.randint(0, 128, d // 2 - 1) / 128)
            x[at[:d // 2 - 1]], x[at[d // 2 - 1:d - 2]] = most, -most
            x[at[-1]] = r.randint(64, 256) * 2.0 ** (14 - step)
            bounds[page, h] = x * sign[rows[page], h]
    bounds = torch.tensor(bounds, device="cuda").bfloat16()
    c.q.copy_(torch.tensor(sign))
    plan = B.asynclm_plan_sparse(*c.args, 60, 1, 2)
    chosen = torch.zeros((c.total, 2, 60), dtype=torch.int32, device="cuda")
    B.asynclm_select_pages(plan, c.q, bounds, chosen)
    assert chosen.cpu().tolist() == chosen_pages(c, bounds, 60, 1, 2)


@pytest.mark.parametrize("kv8", [False, True])
def test_the_same_call_twice(kv8):
    """The same inputs give the same bits, whichever CTA ran what: choice and attention, and attention behind a shared prefix with spans beside it."""
    c = Cache((32, 8, 128), [9000, 30000, 77, 4000], [1, 2, 1, 4], kv8=kv8)
    plan = B.asynclm_plan_sparse(*c.args, 64, 1, 4, kv8=kv8)
    bounds = torch.zeros((c.num_pages, 8, 2, 128), dtype=torch.bfloat16, device="cuda")
    update_bounds(c, plan, bounds, True)
    groups = [(0, 24, 3008)]
    s = Cache((32, 8, 128), 3008 + np.arange(24) * 37, [1] * 18 + [40, 3, 1, 70, 1, 1], groups, kv8, 2)
    shared = B.asynclm_plan_prefix(*s.args, groups, kv8=kv8)
    first = None
    for _ in range(12):
        chosen = torch.full((c.total, 8, 64), 99, dtype=torch.int32, device="cuda")
        B.asynclm_select_pages(plan, c.q, bounds, chosen)
        got = [chosen.clone(), *c.attend(plan), *s.attend(shared)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))
