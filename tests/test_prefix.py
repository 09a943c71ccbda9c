"""Attention of sequences that begin with the same pages, against 64 bits (GPU)."""
import numpy as np
import pytest
import torch

from paper_2412_07017_b200 import binding as B
from cache_util import Cache, check

pytestmark = pytest.mark.gpu
HEADS = [(32, 8, 128), (8, 8, 128), (8, 4, 64), (8, 1, 128), (8, 1, 64), (4, 1, 64)]
# (context behind the prefix, new tokens) of the sequences, groups
BATCHES = {
    "two": ([0, 5], [1, 1], [(0, 2, 16)]),
    "ragged": ([0, 1, 15, 16, 17, 300], [1] * 6, [(0, 6, 48)]),
    "long": ([3, 40, 777, 129], [1, 2, 1, 5], [(0, 4, 5008)]),
    "paused": ([3, 40, 50, 129, 9], [1, 0, 3, 0, 1], [(0, 5, 640)]),
    "many rows": ([7] * 70, [1, 2, 3, 1, 1, 8, 1] * 10, [(0, 70, 272)]),
    "spans": ([30, 0, 9, 100, 8], [16, 17, 1, 40, 3], [(0, 5, 400)]),
    "groups": ([1, 20, 3, 64, 500, 33, 60], [1, 1, 2, 1, 1, 1, 150], [(0, 2, 128), (2, 2, 256), (5, 2, 16)]),
    "a row tile and more": ([5, 5, 5, 5], [1, 130, 1, 2], [(0, 4, 320)]),
}


def make(name, heads, kv8, seed=0):
    own, new, groups = BATCHES[name]
    ctx = np.array(own)
    for first, n, tokens in groups:
        ctx[first:first + n] += tokens
    return Cache(heads, ctx, new, groups, kv8, seed), groups


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("name", BATCHES)
def test_exact(name, heads, kv8):
    c, groups = make(name, heads, kv8)
    plan = B.asynclm_plan_prefix(*c.args, groups, kv8=kv8, flags=B.PLAN_SHARE_ALL)
    want = c.exact()
    first = c.attend(plan)
    check(first, want, name)
    again = c.attend(plan)      # the same plan, as a model's next layer
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    assert B.last_device_status(plan) == 0


@pytest.mark.parametrize("options", [dict(kv_chunk_tokens=64), dict(tensor_min_rows=1), dict(flags=B.PLAN_SHARE_ALL | B.PLAN_NO_TENSOR_PATH), dict(num_sms=7)])
@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 4, 64)])
def test_plan_options(options, heads):
    c, groups = make("long", heads, False)
    plan = B.asynclm_plan_prefix(*c.args, groups, **{"flags": B.PLAN_SHARE_ALL, **options})
    check(c.attend(plan), c.exact(), str(options))


@pytest.mark.parametrize("kv8", [False, True])
def test_scale_and_no_lse(kv8):
    c, groups = make("ragged", (32, 8, 128), kv8)
    a = B.asynclm_plan_prefix(*c.args, groups, sm_scale=0.01, kv8=kv8, flags=B.PLAN_SHARE_ALL)
    b = B.asynclm_plan(*c.args, sm_scale=0.01, kv8=kv8)
    x, y = c.attend(a), c.attend(b)
    assert (x[1] - y[1]).abs().max() <= 8e-4
    assert ((x[0].double() - y[0].double()).abs() <= 2 * 2.1 * 2.0 ** -8 * 4.0).all()      # (|V| is below 6, its weighted mean below 4)
    out = torch.empty_like(x[0])
    if kv8:
        B.asynclm_kv8_attn_mixed(a, c.q, c.pool, c.scales, out)
    else:
        B.asynclm_attn_mixed(a, c.q, c.pool, out)
    assert torch.equal(out, x[0])


def test_step_append_and_static():
    """The other calls that take the plan: append, the whole step, the fixed scratch."""
    c, groups = make("groups", (32, 8, 128), False)
    plan = B.asynclm_plan_prefix(*c.args, groups, flags=B.PLAN_SHARE_ALL)
    rows = [torch.randn((c.total, c.hkv, c.d), device="cuda").bfloat16() for _ in range(2)]
    before = c.pool.clone()
    B.asynclm_kv_append(plan, *rows, c.pool)
    appended = c.pool.clone()
    B.asynclm_kv_append(B.asynclm_plan(*c.args), *rows, before)
    assert torch.equal(appended.view(torch.int16), before.view(torch.int16))
    want = c.exact()
    got = c.attend(plan)
    check(got, want)
    static = c.attend(plan, call=lambda p, q, pool, out, lse: B.asynclm_attn_mixed_static(p, q, pool, out, lse))
    assert torch.equal(got[0], static[0]) and torch.equal(got[1], static[1])
    step = c.attend(plan, call=lambda p, q, pool, out, lse: B.asynclm_step(p, q, *rows, pool, out, lse))
    assert torch.equal(got[0], step[0]) and torch.equal(got[1], step[1])


def test_small_step_is_not_fused():
    """A step of single tokens has its append apart from the attention: the units' keys are not all of their sequence's."""
    c, groups = make("ragged", (32, 8, 128), False)
    plan = B.asynclm_plan_prefix(*c.args, groups, flags=B.PLAN_SHARE_ALL)
    rows = [torch.randn((c.total, c.hkv, c.d), device="cuda").bfloat16() for _ in range(2)]
    got = c.attend(plan, call=lambda p, q, pool, out, lse: B.asynclm_step(p, q, *rows, pool, out, lse))
    check(got, c.exact())


@pytest.mark.parametrize("kv8", [False, True])
def test_graph(kv8):
    """Captured, replayed with other queries, between calls of an ordinary plan on the same stream."""
    c, groups = make("long", (32, 8, 128), kv8)
    plan, other = B.asynclm_plan_prefix(*c.args, groups, kv8=kv8), B.asynclm_plan(*c.args, kv8=kv8)
    out, lse = c.attend(plan)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for p in (plan, other, plan):
            c.attend(p, out, lse)
    for seed in (1, 2):
        c.q.copy_(torch.randn(c.q.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        check((out, lse), c.exact())


def test_side_stream():
    c, groups = make("groups", (8, 4, 64), False)
    want = c.exact()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        plan = B.asynclm_plan_prefix(*c.args, groups, flags=B.PLAN_SHARE_ALL)
        got = c.attend(plan)
    s.synchronize()
    check(got, want)


@pytest.mark.parametrize("kv8", [False, True])
def test_weights_on_either_side(kv8):
    """All of a row's weight in the prefix for some heads, behind it for others: the join of sums that are 2^100 apart and more."""
    c, groups = make("long", (8, 1, 128), kv8)
    v = c.q.view(c.total, 8, 128)
    v[:, ::2] *= 30
    v[:, 1::2] *= 12
    plan = B.asynclm_plan_prefix(*c.args, groups, kv8=kv8, flags=B.PLAN_SHARE_ALL)
    out, lse = c.attend(plan)
    ref, ref_lse, a_sum = c.exact()
    assert ((out.double() - ref).abs() <= (2.1 * 2.0 ** -8 + 2e-3) * a_sum).all()      # (scores of 500: their fp32 error of 2^-21 * 500 is in the weights)
    assert ((lse.double() - ref_lse).abs() <= 4e-4 + 2.0 ** -20 * ref_lse.abs()).all()
