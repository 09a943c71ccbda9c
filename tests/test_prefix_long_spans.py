"""Batches that share a prefix with spans beyond the length that always shares it, planned without flags: what such a plan reads, and its results."""
import numpy as np
import pytest

from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200.workload import Shape
from test_prefix_plan import PAGE, batch, coverage


def plans(new, prefix, heads=(32, 8, 128), kv8=False, own=100):
    rows, args = batch([(len(new), prefix)], [own] * len(new), new)
    shape = Shape(*heads, PAGE)
    return shape, args, B.plan_host(shape, 1 << 20, *args, groups=rows, kv8=kv8), B.plan_host(shape, 1 << 20, *args, kv8=kv8)


def keys_read(plan):
    return sum(int(i["kv1"] - i["kv0"]) for i in plan.items())


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("new,prefix", [([1, 300] * 10, 16000), ([1, 257] * 20, 8000), ([300, 1, 1] * 4, 30000), ([1, 300, 1, 300], 30000)])
def test_the_order_of_a_batch_loses_nothing(new, prefix, kv8):
    """Single tokens between long spans, or in front of them: no stretch of either kind by itself need share anything."""
    _, _, mixed, ordinary = plans(new, prefix, kv8=kv8)
    _, _, in_order, _ = plans(sorted(new), prefix, kv8=kv8)
    assert keys_read(mixed) <= keys_read(in_order) < keys_read(ordinary)


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 1, 64)])
@pytest.mark.parametrize("new,prefix", [([1, 300] * 6, 6400), ([300] * 3, 8000), ([1, 400, 0, 1, 2, 300, 7], 12000), ([1, 1, 1, 300, 1, 1], 3008)])
def test_every_key_once(new, prefix, heads):
    shape, args, plan, ordinary = plans(new, prefix, heads)
    for r in coverage(shape, plan, args[0], args[1]):
        for h in r:
            assert (h == 1).all()
    assert keys_read(plan) <= keys_read(ordinary)


@pytest.mark.gpu
@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("new,prefix,heads,shares", [([1, 140] * 4, 16000, (8, 1, 128), None), ([1, 140] * 4, 16000, (16, 2, 64), None), ([150, 1, 1, 0, 160, 2], 40000, (8, 1, 128), None),
                                                     ([1, 140] * 4, 60000, (8, 1, 128), True), ([1, 140] * 6, 30000, (16, 2, 64), True), ([1, 130] * 4, 40000, (32, 4, 64), True)])
def test_results(new, prefix, heads, shares, kv8):
    """shares: whether the plan has to share something (None: as its model has it)."""
    import torch
    from cache_util import Cache, check
    own = np.arange(len(new)) * 37 % 300
    groups = [(0, len(new), prefix)]
    c = Cache(heads, own + prefix, new, groups, kv8)
    plan, ordinary = B.asynclm_plan_prefix(*c.args, groups, kv8=kv8), B.asynclm_plan(*c.args, kv8=kv8)
    assert keys_read(plan) < keys_read(ordinary) or not shares
    got = c.attend(plan)
    check(got, c.exact())
    again = c.attend(plan)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    assert B.last_device_status(plan) == 0
