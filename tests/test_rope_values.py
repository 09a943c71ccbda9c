"""Rotary rows with values that are not finite, too small to be normal numbers, or behind a rotary_dim that ends inside a vector of eight."""
import numpy as np
import pytest
import torch

from gpu_util import to_bits, to_dev
from oracle import kv8
from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200 import workload as W
from test_kv8 import bits_of, codes_of_random_pool, dev8, plan_of, ulp_diff

pytestmark = pytest.mark.gpu
ROTARY = [(64, "half", 20), (64, "half", 62), (128, "half", 2), (128, "half", 122), (64, "half", 64), (128, "half", 32), (64, "interleaved", 20), (128, "interleaved", 128),
          (64, "interleaved", 62)]


def turned_both_ways(q, ctx, table):
    """Query rows q (bits [T][H][d]) at positions ctx .. ctx + T - 1 by asynclm_rope_apply and by the append: bits of each."""
    T, H, d = q.shape
    x = to_dev(q)
    alone = torch.zeros_like(x)
    B.asynclm_rope_apply(table, torch.arange(ctx, ctx + T, dtype=torch.int32, device="cuda"), x, alone)
    wl = W.make_single_step("values", W.Shape(H, 1, d, 16), [ctx], [T], seed=61)
    pool, scales = dev8(*codes_of_random_pool(wl, 62))
    appended = torch.zeros_like(x)
    B.asynclm_kv8_append(plan_of(wl, wl.steps[0], kv8=True), to_dev(wl.steps[0].k_new), to_dev(wl.steps[0].v_new), pool, scales, table, x, appended)
    torch.cuda.synchronize()
    return to_bits(alone), to_bits(appended)


@pytest.mark.parametrize("d,layout,rotary", ROTARY)
def test_what_lies_behind_rotary_dim_passes_through_bit_for_bit(d, layout, rotary):
    q = np.random.default_rng(rotary).integers(0, 1 << 16, (7, 4, d)).astype(np.uint16)
    q[..., :rotary] = bits_of(np.random.default_rng(1).standard_normal(q[..., :rotary].shape))
    special = np.array([0x7F80, 0xFF80, 0x7FC1, 0xFFBF, 0x0001, 0x8003, 0x007F, 0x8000], np.uint16)      # infinities, NaN, subnormal numbers, -0
    if rotary < d:
        q[0, 0, rotary:] = np.resize(special, d - rotary)
        q[3, 2, rotary:] = np.resize(special[::-1], d - rotary)
    for got in turned_both_ways(q, 11, B.asynclm_rope_table(d, 10000.0, rotary, layout)):
        assert np.array_equal(got[..., rotary:], q[..., rotary:])


@pytest.mark.parametrize("d,layout,rotary", ROTARY)
def test_values_that_are_not_finite_turn_as_the_formula_has_it(d, layout, rotary):
    """x cos a - y sin a with an infinite x is infinite (NaN beside 0 * infinity, at position 0, or beside another infinity), and the other pairs of the row
    are what they are without it, bit for bit."""
    r = np.random.default_rng(rotary + d)
    T, H = 6, 4
    x = W.bf16_bits_to_f64(bits_of(r.standard_normal((T, H, d))))
    table = B.asynclm_rope_table(d, 10000.0, rotary, layout)
    f, m = kv8.frequencies(rotary, 10000.0)
    clean = turned_both_ways(bits_of(x), 0, table)
    for t in range(T):
        for h in range(H):
            x[t, h, r.integers(rotary)] = r.choice([np.inf, -np.inf, np.nan])
    x[5, 3, :rotary] = np.where(r.random(rotary) < 0.3, np.inf, x[5, 3, :rotary])
    with np.errstate(invalid="ignore"):
        want = kv8.turn(x, np.arange(T), f, m, layout)
    odd = ~np.isfinite(want)
    assert odd.any() and np.isinf(want).any() and np.isnan(want[0]).any()
    for got, without in zip(turned_both_ways(bits_of(x), 0, table), clean):
        value = W.bf16_bits_to_f64(got)
        assert np.array_equal(value[odd], want[odd], equal_nan=True)
        assert np.array_equal(got[~odd], without[~odd])


@pytest.mark.parametrize("d,layout,rotary", [(128, "half", 128), (64, "interleaved", 32), (64, "half", 20)])
@pytest.mark.parametrize("T", [1, 40, 1500])
def test_queries_turned_where_they_lie(d, layout, rotary, T):
    """q_out = q gives what a q_out of its own gives, bit for bit."""
    wl = W.make_single_step("in place", W.Shape(8, 2, d, 16), [5, 100], [T, 1], seed=63)
    st = wl.steps[0]
    table = B.asynclm_rope_table(d, 10000.0, rotary, layout)
    plan = plan_of(wl, st, kv8=True)
    left = []
    for same in (False, True):
        pool, scales = dev8(*codes_of_random_pool(wl, 64))
        q = to_dev(st.q)
        q_out = q if same else torch.zeros_like(q)
        B.asynclm_kv8_append(plan, to_dev(st.k_new), to_dev(st.v_new), pool, scales, table, q, q_out)
        torch.cuda.synchronize()
        left.append([to_bits(q_out), pool.view(torch.uint8).cpu().numpy(), scales.view(torch.uint8).cpu().numpy()])
    assert all(np.array_equal(a, b) for a, b in zip(*left))
    pos = np.concatenate([5 + np.arange(T), [100]])
    want = bits_of(kv8.turn(W.bf16_bits_to_f64(st.q), pos, *kv8.frequencies(rotary, 10000.0), layout))
    assert ulp_diff(left[0][0], want).max() <= 1
