"""Bounds of pages, the selection by them, and attention over what was selected (GPU)."""
import numpy as np
import pytest
import torch

from paper_2412_07017_b200 import binding as B
from cache_util import PAGE, Cache, check

pytestmark = pytest.mark.gpu
HEADS = [(32, 8, 128), (8, 8, 128), (8, 4, 64), (8, 1, 128), (8, 1, 64), (4, 4, 64), (4, 1, 64)]
CTX, NEW = [0, 15, 16, 400, 5000, 3, 2047, 6 * PAGE], [1, 1, 2, 5, 1, 0, 33, 1]


def chosen_pages(c, bounds, budget, first, last):
    """[rows][kv heads] lists from the definition, in 64 bits."""
    out, row = [], 0
    for b in range(len(c.ctx)):
        pages = torch.as_tensor(c.ids[c.indptr[b]:c.indptr[b + 1]].astype(np.int64)).cuda()
        edges = bounds[pages].transpose(0, 1)[:, None].double()      # [kv heads][1][pages][2][dim]
        for t in range(int(c.new[b])):
            n = (int(c.ctx[b]) + t) // PAGE + 1
            q = c.q[row].double().reshape(c.hkv, -1, 1, c.d)
            score = torch.maximum(q * edges[:, :, :n, 0], q * edges[:, :, :n, 1]).sum(-1).amax(1).cpu().numpy()
            lists = []
            for h in range(c.hkv):
                always = [j for j in range(n) if n <= budget or j < first or j >= n - last]
                rest = [j for j in range(n) if j not in set(always)]
                rest.sort(key=lambda j: (-score[h][j], j))
                lists.append(sorted(always + rest[:max(0, budget - len(always))]))
            out.append(lists)
            row += 1
    return out


def as_mask(c, lists):
    most = int((c.ctx + c.new).max())
    mask = torch.zeros((c.total, c.hkv, most + PAGE), dtype=torch.bool)
    for r, row in enumerate(lists):
        for h, pages in enumerate(row):
            for j in pages:
                mask[r, h, j * PAGE:(j + 1) * PAGE] = True
    return mask.cuda()


def update_bounds(c, plan, bounds, from_start):
    if c.kv8:
        B.asynclm_kv8_bounds(plan, c.pool, c.scales, bounds, from_start)
    else:
        B.asynclm_kv_bounds(plan, c.pool, bounds, from_start)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("heads", HEADS)
def test_bounds(heads, kv8):
    c = Cache(heads, CTX, NEW, kv8=kv8)
    plan = B.asynclm_plan(*c.args, kv8=kv8)
    want = c.bounds()
    touched = torch.zeros(c.num_pages, dtype=torch.bool)
    active = torch.zeros(c.num_pages, dtype=torch.bool)
    for b in range(len(CTX)):
        if NEW[b]:
            active[c.ids[c.indptr[b]:c.indptr[b + 1]]] = True
            touched[c.ids[c.indptr[b] + CTX[b] // PAGE:c.indptr[b + 1]]] = True
    for from_start, pages in ((False, touched), (True, active)):
        got = torch.full((c.num_pages, c.hkv, 2, c.d), 77.0, dtype=torch.bfloat16, device="cuda")
        update_bounds(c, plan, got, from_start)
        assert torch.equal(got[pages].double(), want[pages.cuda()])
        assert (got[~pages] == 77).all()      # others are left alone
    assert B.last_device_status(plan) == 0


def test_bounds_of_odd_values():
    c = Cache((8, 4, 64), [100], [1])
    page = int(c.ids[2])
    c.pool[page, 0, 1, 3, 5] = float("nan")
    c.pool[page, 0, 2, 0, 7] = float("inf")
    c.pool[page, 0, 3, 9, 8:10] = torch.tensor([1e-40, -1e-40])      # subnormal numbers stay
    c.pool[page, 0, 3, :, 8:10] = c.pool[page, 0, 3, 9:10, 8:10].clone()
    got = torch.zeros((c.num_pages, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
    update_bounds(c, B.asynclm_plan(*c.args), got, True)
    assert got[page, 1, 0, 5] == -float("inf") and got[page, 1, 1, 5] == float("inf")
    assert got[page, 2, 1, 7] == float("inf") and torch.isfinite(got[page, 2, 0]).all()
    assert got[page, 3, 0, 8] == c.pool[page, 0, 3, 0, 8] != 0 and got[page, 3, 1, 9] == c.pool[page, 0, 3, 0, 9] != 0
    assert torch.isfinite(got[page, 0]).all()
    k8 = Cache((8, 4, 64), [100], [1], kv8=True)
    page = int(k8.ids[2])
    k8.scales.view(torch.uint8)[page, 1, 0, 3] = 255
    update_bounds(k8, B.asynclm_plan(*k8.args), got, True)
    assert (got[page, 1, 0] == -float("inf")).all() and (got[page, 1, 1] == float("inf")).all() and torch.isfinite(got[page, 2]).all()


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("budget,first,last", [(1, 0, 1), (6, 1, 2), (7, 3, 4), (40, 0, 1), (300, 2, 8), (1000, 1, 1)])
def test_selection_and_attention(heads, kv8, budget, first, last):
    c = Cache(heads, CTX, NEW, kv8=kv8, seed=budget)
    plan = B.asynclm_plan_sparse(*c.args, budget, first, last, kv8=kv8)
    bounds = torch.zeros((c.num_pages, c.hkv, 2, c.d), dtype=torch.bfloat16, device="cuda")
    update_bounds(c, plan, bounds, True)
    pages = torch.full((c.total, c.hkv, budget), 99, dtype=torch.int32, device="cuda")
    B.asynclm_select_pages(plan, c.q, bounds, pages)
    lists = chosen_pages(c, c.bounds().nan_to_num(0.0), budget, first, last)
    want = torch.tensor([[h + [-1] * (budget - len(h)) for h in row] for row in lists], dtype=torch.int32)
    assert torch.equal(pages.cpu(), want)
    check(c.attend(plan), c.exact(as_mask(c, lists)))
    # another layer's queries with the same plan, without the list
    c.q.copy_(torch.randn_like(c.q.float()))
    B.asynclm_select_pages(plan, c.q, bounds)
    check(c.attend(plan), c.exact(as_mask(c, chosen_pages(c, c.bounds().nan_to_num(0.0), budget, first, last))))
    assert B.last_device_status(plan) == 0


def test_ties_and_odd_scores():
    """Equal scores go to the lowest page; infinite bounds come first; scores of zero."""
    c = Cache((8, 2, 128), [1600, 70000], [1, 1])
    plan = B.asynclm_plan_sparse(*c.args, 20, 1, 2)
    bounds = torch.zeros((c.num_pages, 2, 2, 128), dtype=torch.bfloat16, device="cuda")
    pages = torch.zeros((2, 2, 20), dtype=torch.int32, device="cuda")

    def select():
        B.asynclm_select_pages(plan, c.q, bounds, pages)
        return pages.cpu().tolist()
    n = [1600 // PAGE + 1, 70000 // PAGE + 1]
    assert select() == [[list(range(18)) + [m - 2, m - 1]] * 2 for m in n]
    bounds.fill_(1.0)
    assert select() == [[list(range(18)) + [m - 2, m - 1]] * 2 for m in n]
    bounds[c.ids[50]], bounds[c.ids[c.indptr[1] + 4321]] = 2.0, 2.0      # same bounds above and below: q . 2, larger or smaller than q . 1 by q's sum
    got = select()
    for r in range(2):
        for h in range(2):
            up = bool(c.q[r, 4 * h:4 * h + 4].double().sum(-1).amax() > 0)
            page = (50, 4321)[r]
            assert (page in got[r][h]) == up
    bounds.fill_(1.0)
    for at in (int(c.ids[77]), int(c.ids[c.indptr[1] + 4100])):
        bounds[at, 1, 0], bounds[at, 1, 1] = -float("inf"), float("inf")
    got = select()
    assert 77 in got[0][1] and 77 not in got[0][0] and 4100 in got[1][1] and 4100 not in got[1][0]
    c.q[0, 5] = float("nan")      # a choice all the same, of valid pages
    got = select()
    assert all(sorted(set(h)) == h and 0 <= h[0] and h[-1] == n[r] - 1 for r, row in enumerate(got) for h in row)


def test_tiny_and_huge_values():
    """Bounds and queries at the ends of their range: scores whose 32 bits say nothing are decided in 64; beyond 2^56 all count as 2^56."""
    c = Cache((8, 2, 128), [4000, 9000], [1, 2])
    plan = B.asynclm_plan_sparse(*c.args, 30, 1, 2)
    pages = torch.zeros((3, 2, 30), dtype=torch.int32, device="cuda")
    plain, q = c.bounds().nan_to_num(0.0), c.q.clone()
    for scale_b, scale_q in ((2.0 ** -126, 1.0), (2.0 ** -126, 2.0 ** 50), (2.0 ** 50, 2.0 ** 50), (2.0 ** -70, 2.0 ** -60), (1.0, 0.0)):
        bounds = (plain * scale_b).bfloat16()
        c.q.copy_(q.float() * scale_q)
        B.asynclm_select_pages(plan, c.q, bounds, pages)
        assert pages.cpu().tolist() == chosen_pages(c, bounds, 30, 1, 2), (scale_b, scale_q)
    c.q.copy_(q)
    bounds = plain.bfloat16()
    bounds[c.ids[c.indptr[1] + 300], :, 0], bounds[c.ids[c.indptr[1] + 300], :, 1] = -3e38, 3e38
    bounds[c.ids[c.indptr[1] + 301]] = bounds[c.ids[c.indptr[1] + 300]]
    B.asynclm_select_pages(plan, c.q, bounds, pages)
    assert pages.cpu().tolist() == chosen_pages(c, bounds.double().clamp(-2.0 ** 56, 2.0 ** 56), 30, 1, 2)


def test_many_equal_scores():
    """Far more pages at the threshold than a CTA ranks at once, in 32 bits and in 64, also where a row's keys are not held in registers."""
    c = Cache((4, 1, 64), [80000, 30000], [1, 1])
    plan = B.asynclm_plan_sparse(*c.args, 900, 3, 4)
    pages = torch.zeros((2, 1, 900), dtype=torch.int32, device="cuda")
    bounds = torch.zeros((c.num_pages, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    for kinds in (1, 2, 5):
        kind = torch.randint(0, kinds, (c.num_pages,), generator=g, device="cuda")
        bounds[:] = (1.0 + kind.float() * 2.0 ** -7).bfloat16()[:, None, None, None]      # neighbours in bf16
        B.asynclm_select_pages(plan, c.q, bounds, pages)
        assert pages.cpu().tolist() == chosen_pages(c, bounds, 900, 3, 4), kinds


def test_long_sequence():
    """More pages than the selection holds in shared memory, more keys than one list."""
    c = Cache((4, 1, 64), [90000, 66000], [2, 1])
    plan = B.asynclm_plan_sparse(*c.args, 333, 1, 5)
    bounds = torch.zeros((c.num_pages, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    update_bounds(c, plan, bounds, True)
    pages = torch.zeros((3, 1, 333), dtype=torch.int32, device="cuda")
    B.asynclm_select_pages(plan, c.q, bounds, pages)
    lists = chosen_pages(c, c.bounds().nan_to_num(0.0), 333, 1, 5)
    assert pages.cpu().tolist() == lists
    check(c.attend(plan), c.exact(as_mask(c, lists)))


@pytest.mark.parametrize("kv8", [False, True])
def test_graph_of_layers(kv8):
    """Two layers captured: append, bounds, selection, attention, each with its own cache and one plan; replayed with other inputs."""
    layers = [Cache((32, 8, 128), [3000, 77, 1200], [1, 1, 3], kv8=kv8, seed=s) for s in (0, 0)]
    for c in layers:
        c.out, c.lse = torch.zeros_like(c.q), torch.zeros((c.total, c.hq), device="cuda")
        c.kb = torch.zeros((c.num_pages, c.hkv, 2, c.d), dtype=torch.bfloat16, device="cuda")
        c.k, c.v = (torch.randn((c.total, c.hkv, c.d), device="cuda").bfloat16() for _ in range(2))
        c.pages = torch.zeros((c.total, c.hkv, 24), dtype=torch.int32, device="cuda")
    plan = B.asynclm_plan_sparse(*layers[0].args, 24, 1, 2, kv8=kv8)
    for c in layers:
        update_bounds(c, plan, c.kb, True)

    def step():
        for c in layers:
            if kv8:
                B.asynclm_kv8_append(plan, c.k, c.v, c.pool, c.scales)
            else:
                B.asynclm_kv_append(plan, c.k, c.v, c.pool)
            update_bounds(c, plan, c.kb, False)
            B.asynclm_select_pages(plan, c.q, c.kb, c.pages)
            c.attend(plan, c.out, c.lse)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for c in layers:
            for t in (c.q, c.k, c.v):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for c in layers:
            lists = chosen_pages(c, c.bounds().nan_to_num(0.0), 24, 1, 2)
            assert torch.equal(c.pages.cpu(), torch.tensor([[h + [-1] * (24 - len(h)) for h in row] for row in lists], dtype=torch.int32))
            check((c.out, c.lse), c.exact(as_mask(c, lists)))


def test_offsets_beyond_32_bits():
    """Pages whose keys lie beyond 2^31 values and whose bounds lie beyond 2^31 bytes."""
    small = Cache((8, 1, 128), [3000, 700], [1, 2], seed=11)
    num_pages = 4_300_000
    far = (np.arange(small.num_pages) * 13 % small.num_pages).astype(np.int64)
    far[far % 2 == 0] += num_pages - small.num_pages      # half of them at the end, the others at the start
    pool = torch.empty((num_pages, 2, 1, PAGE, 128), dtype=torch.bfloat16, device="cuda")
    pool[torch.as_tensor(far).cuda()] = small.pool
    bounds = torch.empty((num_pages, 1, 2, 128), dtype=torch.bfloat16, device="cuda")
    assert bounds.numel() * 2 > 2 ** 31 and pool.numel() > 2 ** 31
    args = (small.shape, num_pages, small.q_indptr, small.ctx, small.indptr, far[small.ids].astype(np.int32))
    plan = B.asynclm_plan_sparse(*args, 20, 1, 2)
    B.asynclm_kv_bounds(plan, pool, bounds, True)
    want = small.bounds()
    used = torch.as_tensor(np.unique(small.ids).astype(np.int64)).cuda()
    assert torch.equal(bounds[torch.as_tensor(far).cuda()[used]].double(), want[used])
    pages = torch.zeros((3, 1, 20), dtype=torch.int32, device="cuda")
    B.asynclm_select_pages(plan, small.q, bounds, pages)
    lists = chosen_pages(small, want.nan_to_num(0.0), 20, 1, 2)
    assert pages.cpu().tolist() == lists
    out, lse = small.attend(plan, call=lambda p, q, _, o, z: B.asynclm_attn_mixed(p, q, pool, o, z))
    check((out, lse), small.exact(as_mask(small, lists)))


def test_refusals():
    c = Cache((8, 4, 64), [100], [1])
    plan, ordinary = B.asynclm_plan_sparse(*c.args, 4, 1, 1), B.asynclm_plan(*c.args)
    bounds = torch.zeros((c.num_pages, 4, 2, 64), dtype=torch.bfloat16, device="cuda")

    def status(f, *args, **kw):
        with pytest.raises(B.AsynclmError) as e:
            f(*args, **kw)
        return e.value.status
    out = torch.empty_like(c.q)
    assert status(B.asynclm_attn_mixed, plan, c.q, c.pool, out) == -1                   # nothing selected yet
    assert status(B.asynclm_attn_mixed_static, plan, c.q, c.pool, out) == -1
    assert status(B.asynclm_select_pages, ordinary, c.q, bounds) == -1
    assert status(B.asynclm_step, plan, c.q, c.q[:, :4].contiguous(), c.q[:, :4].contiguous(), c.pool, out) == -1
    B.asynclm_select_pages(plan, c.q, bounds)
    B.asynclm_attn_mixed(plan, c.q, c.pool, out)
    for bad in (bounds.float(), bounds[:-1], bounds.cpu(), bounds.transpose(2, 3)):
        with pytest.raises(ValueError):
            B.asynclm_select_pages(plan, c.q, bad)
        with pytest.raises(ValueError):
            B.asynclm_kv_bounds(plan, c.pool, bad)
    with pytest.raises(ValueError):
        B.asynclm_kv_bounds(plan, c.pool[:-1], bounds)
    with pytest.raises(ValueError):
        B.asynclm_select_pages(plan, c.q[:, :4], bounds)
    with pytest.raises(ValueError):
        B.asynclm_select_pages(plan, c.q, bounds, torch.zeros(3, dtype=torch.int32, device="cuda"))
