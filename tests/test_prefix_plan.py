"""Plans for batches that share a prefix, and for selected pages: what they cover, and what they refuse (host only)."""
import numpy as np
import pytest

from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200.workload import Shape

PAGE = 16


def batch(groups, own, new, alone=()):
    """groups: (sequences, prefix tokens); own[b] context tokens behind the prefix, new[b] new tokens; alone: contexts of sequences in no group, behind."""
    prefix = np.concatenate([[p] * n for n, p in groups] + [[0] * len(alone)]).astype(int)
    ctx = prefix + np.concatenate([own, alone]).astype(int)
    new = np.asarray(new)
    pages = -(-(ctx + new) // PAGE)
    indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    ids = np.arange(int(indptr[-1]), dtype=np.int32)
    rows, first = [], 0
    for n, p in groups:
        for b in range(first, first + n):
            ids[indptr[b]:indptr[b] + p // PAGE] = ids[indptr[first]:indptr[first] + p // PAGE]
        rows.append((first, n, p))
        first += n
    q_indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return rows, (q_indptr, ctx.astype(np.int32), indptr, ids)


def coverage(shape, plan, q_indptr, ctx):
    """Times that each (row, kv head) has each of its keys in an item."""
    seq = np.repeat(np.arange(len(ctx)), np.diff(q_indptr))
    sees = ctx[seq] + np.arange(len(seq)) - q_indptr[seq] + 1
    seen = [[np.zeros(n, int) for _ in range(shape.num_kv_heads)] for n in sees]
    for it in plan.items():
        for r in range(q_indptr[it["seq"]] + it["tok0"], q_indptr[it["seq"]] + it["tok0"] + it["ntok"]):
            seen[r][it["kv_head"]][it["kv0"]:it["kv1"]] += 1
    return seen


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (4, 4, 64), (8, 1, 128)])
@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("groups,own,new,alone", [
    ([(6, 8192)], [0, 1, 15, 16, 17, 900], [1, 1, 1, 1, 1, 1], []),
    ([(5, 6400), (4, 9600)], [3, 40, 0, 200, 7, 100, 2, 60, 31], [1, 0, 4, 1, 33, 1, 300, 2, 1, 1, 5], [700, 4000]),
    ([(40, 16000)], [20] * 40, [3] * 40, []),
])
def test_every_key_once(heads, kv8, groups, own, new, alone):
    shape = Shape(*heads, PAGE)
    rows, args = batch(groups, own, new, alone)
    plan = B.plan_host(shape, 1 << 20, *args, groups=rows, kv8=kv8, flags=B.PLAN_SHARE_ALL)
    for r in coverage(shape, plan, args[0], args[1]):
        for h in r:
            assert (h == 1).all()
    ordinary = B.plan_host(shape, 1 << 20, *args, kv8=kv8)
    read = lambda p: sum(int(i["kv1"] - i["kv0"]) for i in p.items())      # noqa: E731
    assert read(plan) < read(ordinary)
    assert plan.info["partial_rows"] > 0


def test_nothing_worth_sharing_is_the_ordinary_plan():
    shape = Shape(32, 8, 128, PAGE)
    for groups, own, new in (([(2, 16)], [4, 9], [1, 1]), ([(1, 8192)], [4], [1]), ([(3, 0)], [5, 6, 7], [1, 1, 1]), ([(4, 3008)], [5, 6, 7, 8], [900, 1300, 1000, 700])):
        rows, args = batch(groups, own, new)
        a, b = B.plan_host(shape, 1 << 20, *args, groups=rows), B.plan_host(shape, 1 << 20, *args)
        assert (a.items() == b.items()).all() and a.info["partial_rows"] == b.info["partial_rows"]
    assert len(B.plan_host(shape, 1 << 20, *args, groups=[]).items()) == len(b.items())


def test_groups_refused():
    shape = Shape(32, 8, 128, PAGE)
    rows, args = batch([(3, 8192)], [5, 6, 7], [1, 1, 1])
    for bad, status in (([(0, 3, 8190)], -1), ([(0, 4, 8192)], -1), ([(-1, 2, 8192)], -1), ([(0, 0, 8192)], -1), ([(1, 2, 16), (0, 1, 16)], -1),
                        ([(0, 2, 16), (1, 2, 16)], -1), ([(0, 3, 8208)], -1), ([(0, 3, -16)], -1), ([(0, 2 ** 31 - 1, 16)], -1)):
        with pytest.raises(B.AsynclmError) as e:
            B.plan_host(shape, 1 << 20, *args, groups=bad)
        assert e.value.status == status, bad
    ids = args[3].copy()
    ids[args[2][2] + 100] = 3
    with pytest.raises(B.AsynclmError) as e:
        B.plan_host(shape, 1 << 20, *args[:3], ids, groups=rows)
    assert e.value.status == -3
    with pytest.raises(ValueError):
        B.plan_host(shape, 1 << 20, *args, groups=[(0, 3)])
    # a paused sequence's pages are not looked at
    rows, args = batch([(3, 8192)], [5, 6, 7], [1, 0, 1])
    args[3][args[2][1] + 100] = 77777777
    B.plan_host(shape, 1 << 20, *args, groups=rows)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("heads", [(32, 8, 128), (4, 4, 64)])
def test_sparse_plan(heads, kv8):
    shape = Shape(*heads, PAGE)
    _, args = batch([], [], [1, 4, 0, 1, 2], [0, 5000, 300, 15, 160000])
    plan = B.plan_host(shape, 1 << 20, *args, sparse=(64, 1, 4), kv8=kv8)
    seq = np.repeat(np.arange(5), [1, 4, 0, 1, 2])
    pos = args[1][seq] + np.arange(8) - args[0][seq]
    keys = np.minimum(pos // PAGE, 63) * PAGE + pos % PAGE + 1
    seen = [[np.zeros(n, int) for _ in range(shape.num_kv_heads)] for n in keys]
    for it in plan.items():
        assert it["ntok"] == 1 and it["path"] == 0
        seen[args[0][it["seq"]] + it["tok0"]][it["kv_head"]][it["kv0"]:it["kv1"]] += 1
    assert all((h == 1).all() for r in seen for h in r)
    for bad in ((4, 2, 3), (4, -1, 1), (4, 0, 0), (0, 0, 1), (2 ** 31 - 1, 2 ** 31 - 1, 2)):
        with pytest.raises(B.AsynclmError) as e:
            B.plan_host(shape, 1 << 20, *args, sparse=bad)
        assert e.value.status == -1
    with pytest.raises(B.AsynclmError) as e:
        B.plan_host(shape, 1 << 20, *args, sparse=(64, 1, 4), kv_chunk_tokens=128)
    assert e.value.status == -1
    with pytest.raises(B.AsynclmError) as e:      # lists beyond what an index of the page table reaches
        B.plan_host(shape, 1 << 20, *args, sparse=(2 ** 30, 1, 4))
    assert e.value.status == -4


def test_empty_batch():
    shape = Shape(32, 8, 128, PAGE)
    none = np.zeros(1, np.int32)
    empty = np.zeros(0, np.int32)
    assert len(B.plan_host(shape, 16, none, empty, none, empty, groups=[]).items()) == 0
    assert len(B.plan_host(shape, 16, none, empty, none, empty, sparse=(4, 1, 1)).items()) == 0
