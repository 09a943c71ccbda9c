"""Child process of test_checked_pages.py: with the checked build of the library, bounds and selections of plans with a page id beyond the pool in their device copy.
Prints one JSON line."""
import json
import os

import numpy as np
import torch

from checked_build_child import B
from cache_util import Cache
from test_select_pages import chosen_pages, update_bounds


def table_at(plan, ids):
    """Word offset of the page table inside the plan's device workspace."""
    words = plan.dev_ws[: plan.dev_ws.numel() // 4 * 4].view(torch.int32).cpu().numpy()
    hits = [int(i) for i in np.flatnonzero(words[: len(words) - len(ids) + 1] == ids[0]) if np.array_equal(words[i:i + len(ids)], ids)]
    assert len(hits) == 1, hits
    return hits[0]


def main():
    assert "debug" in os.path.basename(os.environ.get("ASYNCLM_LIBRARY", "")), "the checked build must be the one loaded"
    torch.cuda.set_device(0)
    result = {}
    for kv8 in (False, True):
        c = Cache((8, 2, 128), [5000, 900], [2, 1], kv8=kv8, seed=1)
        bounds = torch.zeros((c.num_pages, 2, 2, 128), dtype=torch.bfloat16, device="cuda")

        def sparse_plan(bad_entry=None):
            plan = B.asynclm_plan_sparse(*c.args, 20, 1, 2, kv8=kv8)
            torch.cuda.synchronize()
            if bad_entry is not None:
                plan.dev_ws[: plan.dev_ws.numel() // 4 * 4].view(torch.int32)[table_at(plan, c.ids) + bad_entry] = c.num_pages + 7
            return plan

        def select(plan):
            chosen = torch.zeros((c.total, 2, 20), dtype=torch.int32, device="cuda")
            B.asynclm_select_pages(plan, c.q, bounds, chosen)
            return B.last_device_status(plan), chosen.cpu().tolist()
        plan = sparse_plan()
        update_bounds(c, plan, bounds, True)
        status, chosen = select(plan)
        assert status == 0 and chosen == chosen_pages(c, c.bounds().nan_to_num(0.0), 20, 1, 2)
        # bounds of a page beyond the pool: left out
        entry = 100
        plan = sparse_plan(entry)
        before = bounds.clone()
        bounds[int(c.ids[entry])] = 5.0
        update_bounds(c, plan, bounds, True)
        result[f"bounds {kv8}"] = B.last_device_status(plan)
        assert (bounds[int(c.ids[entry])] == 5.0).all()
        bounds.copy_(before)
        # a score of one: page 0's in its place
        status, chosen = select(sparse_plan(entry))
        result[f"select {kv8}"] = status
        keep, c.ids = c.ids, c.ids.copy()
        c.ids[entry] = 0
        assert chosen == chosen_pages(c, bounds.double().nan_to_num(0.0), 20, 1, 2)
        c.ids = keep
        # all scores equal, so that every page is scored again in 64 bits
        bounds.fill_(1.0)
        status, chosen = select(sparse_plan(entry))
        result[f"equal {kv8}"] = status
        assert chosen == chosen_pages(c, bounds, 20, 1, 2)
        bounds.copy_(before)
    print(json.dumps(result))


if __name__ == "__main__":
    main()
