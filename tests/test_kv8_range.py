"""Attention over the quantised cache where weights and the scales of V's rows span far more than f16 or fp32 do, against the definition in fp64.

Tolerances, before the first run.  With p the softmax weights, A_j = sum_k p_k |V_kj| and top = max_k p_k max_j |V_kj|:
    |error_j| <= 1.2 * 2^-8 A_j + n * floor * top
  1.2 * 2^-8: the output's rounding to bf16 (2^-8), a weight's to f16 (2^-11 = 0.125 * 2^-8) and the scores' fp32 sums (d products of 20 in all:
  2^-24 * 128 * 20 = 0.04 * 2^-8).
  floor: a weight is an f16 number times 2^-7 of the reference's, so at its lower end it is off by 2^-25 * 2^-7 = 2^-32 of that, whose code is 224 at least
  in its row, where the key's own is 448 at most: 2^-31 on the warp body.  On the span body a reference may count a row of V as if it were as
  large as its tile's largest, which is 2^8 times as large at most: 2^-23.
lse: as in test_kv8.py, 4e-4."""
import numpy as np
import pytest
import torch

from gpu_util import to_bits, to_dev
from oracle import kv8
from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200 import workload as W
from test_kv8 import LSE_ABS, bits_of, dev8, plan_of

pytestmark = pytest.mark.gpu
HQ, HKV = 8, 2
# tokens, flags, whether the span body runs: a decode row; a span on the warp body; of one row tile; of two
BODIES = {"decode": (1, 0, False), "warp span": (9, B.PLAN_NO_TENSOR_PATH, False), "one tile": (20, 0, True), "two tiles": (60, 0, True)}


def rounded(x):
    return W.bf16_bits_to_f64(bits_of(x))


def definition(q, k, v, ctx, scale):
    """out, A, top [T][Hq][..] and lse of queries [T][Hq][d] over all rows k, v [n][Hkv][d], token t seeing ctx + t + 1 of them."""
    T, hq, d = q.shape
    g = hq // k.shape[1]
    out, a, top, lse = (np.zeros(s) for s in ((T, hq, d), (T, hq, d), (T, hq), (T, hq)))
    for h in range(hq):
        kh, vh = k[:, h // g], v[:, h // g]
        s = q[:, h] @ kh.T * scale
        s[np.arange(len(kh))[None] > ctx + np.arange(T)[:, None]] = -np.inf
        m = s.max(-1, keepdims=True)
        p = np.exp(s - m)
        total = p.sum(-1, keepdims=True)
        p /= total
        out[:, h], a[:, h], lse[:, h] = p @ vh, p @ np.abs(vh), (m + np.log(total))[:, 0]
        top[:, h] = (p * np.abs(vh).max(-1)).max(-1)
    return out, a, top, lse


def attend(q, k, v, tokens, sm_scale=0.0, stale=130, **opts):
    """Rows k, v (fp64 [n][Hkv][d], bf16 values), of which the last `tokens` are new, appended and attended to; scales of unused slots are
    `stale`.  -> out fp64, lse, plan, K's and V's values."""
    n, d = len(k), k.shape[-1]
    wl = W.make_single_step("range", W.Shape(q.shape[1], HKV, d, 16), [n - tokens], [tokens], seed=51)
    st = wl.steps[0]
    (kc, kb), (vc, vb) = kv8.quantise(k), kv8.quantise(v)
    codes = np.full((wl.num_pages, 2, HKV, 16, d), 0x7F, np.uint8)
    byte = np.full((wl.num_pages, HKV, 2, 16), stale, np.uint8)
    pos = np.arange(n - tokens)
    pages, slots = np.asarray(st.page_indices)[pos // 16], pos % 16
    for which, c, b in ((0, kc, kb), (1, vc, vb)):
        codes[pages, which, :, slots], byte[pages, :, which, slots] = c[:n - tokens], b[:n - tokens]
    pool, scales = dev8(codes, byte)
    plan = plan_of(wl, st, sm_scale=sm_scale, kv8=True, **opts)
    out = torch.zeros((tokens, q.shape[1], d), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((tokens, q.shape[1]), device="cuda")
    B.asynclm_kv8_append(plan, to_dev(bits_of(k[n - tokens:])), to_dev(bits_of(v[n - tokens:])), pool, scales)
    B.asynclm_kv8_attn_mixed(plan, to_dev(bits_of(q)), pool, scales, out, lse)
    torch.cuda.synchronize()
    assert B.last_device_status(plan) == 0
    return W.bf16_bits_to_f64(to_bits(out)), lse.cpu().numpy().astype(np.float64), plan, kv8.values(kc, kb), kv8.values(vc, vb)


def check(q, k, v, body, what, rows=None, sm_scale=0.0, **opts):
    tokens, flags, spans = BODIES[body]
    got, lse, plan, kv, vv = attend(q, k, v, tokens, sm_scale, flags=flags, **opts)
    assert (plan.info["num_items_tensor"] > 0) == spans
    rows = np.ones(q.shape[:2], bool) if rows is None else rows
    out, a, top, want = definition(np.where(rows[..., None], q, 0.0), kv, vv, len(k) - tokens, sm_scale or k.shape[-1] ** -0.5)
    bound = 1.2 * 2.0 ** -8 * a + len(k) * (2.0 ** -23 if spans else 2.0 ** -31) * top[..., None]
    err = (np.abs(got - out) / (bound + 1e-30))[rows]
    assert np.isfinite(got[rows]).all() and err.max() <= 1, f"{what}: {err.max():.3g} of the bound"
    assert np.abs(lse - want)[rows].max() <= LSE_ABS, f"{what}: lse {np.abs(lse - want)[rows].max():.3g}"
    return got, lse


@pytest.mark.parametrize("body", BODIES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("chunk", [0, 1 << 20])
def test_one_key_with_a_small_value_takes_nearly_all_weight(body, d, chunk):
    """The key that an attention sink is: the others' weights are 2^-24 .. 2^-29 of its own and count all the same, by their number and because its V is small."""
    r = np.random.default_rng(d)
    n, tokens = 8000, BODIES[body][0]
    q = np.ones((tokens, HQ, d))
    for shift in (0, 5, 8, 15):
        for gap, at in ((17.0, 3), (20.0, 3), (17.0, 5000)):
            k, v = r.standard_normal((n, HKV, d)) * 0.4, 1.0 + r.standard_normal((n, HKV, d))
            k[at], v[at] = gap * d ** -0.5, r.standard_normal((HKV, d)) * 2.0 ** -shift
            v[at, :, ::2] = 0.0      # (there the others are all that there is)
            check(q, rounded(k), rounded(v), body, f"2^-{shift}, {gap} nats, key {at}", kv_chunk_tokens=chunk)


@pytest.mark.parametrize("body", BODIES)
@pytest.mark.parametrize("chunk", [0, 1 << 20])
def test_a_sink_without_any_value(body, chunk):
    """Its row of V is zero: all of the output is what the others leave."""
    r = np.random.default_rng(9)
    n, d, tokens = 3000, 128, BODIES[body][0]
    for gap, at in ((9.0, 0), (18.0, 3), (18.0, 2000)):
        k, v = r.standard_normal((n, HKV, d)) * 0.4, 1.0 + r.standard_normal((n, HKV, d))
        k[at], v[at] = gap * d ** -0.5, 0.0
        check(np.ones((tokens, HQ, d)), rounded(k), rounded(v), body, f"{gap} nats, key {at}", kv_chunk_tokens=chunk)


@pytest.mark.parametrize("body", BODIES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("first,second", [(None, 27), (None, 40), (27, None), (40, None), (-30, 100), (100, -30), (110, -28), (-90, 30), (60, -60), (None, 125), (125, None), (125, 3)])
def test_scales_of_v_that_change_along_a_sequence(body, d, first, second):
    """Scores alike, the first half of the keys with V's rows at 2^first (None: zeros), the second half at 2^second: whichever comes first, each half has half
    of the weight."""
    r = np.random.default_rng(77)
    n, tokens = 1530, BODIES[body][0]
    q, k = (rounded(r.standard_normal((m, h, d)) * 0.5) for m, h in ((tokens, HQ), (n, HKV)))
    v = 1.0 + r.standard_normal((n, HKV, d))
    v[:n // 2] *= 0.0 if first is None else 2.0 ** first
    v[n // 2:] *= 0.0 if second is None else 2.0 ** second
    for chunk in (0, 1 << 20):
        check(q, k, rounded(v), body, f"chunk {chunk}", kv_chunk_tokens=chunk)


@pytest.mark.parametrize("body", BODIES)
@pytest.mark.parametrize("d", [64, 128])
def test_queries_that_are_not_finite_give_nan_and_only_their_own_rows(body, d):
    r = np.random.default_rng(5)
    n, tokens = 500, BODIES[body][0]
    q, k, v = (rounded(r.standard_normal((m, h, d))) for m, h in ((tokens, HQ), (n, HKV), (n, HKV)))
    for bad in (np.inf, -np.inf, np.nan):
        x = q.copy()
        rows = np.ones((tokens, HQ), bool)
        for t, h, j in ((0, 2, 5), (tokens - 1, 0, d - 1), (tokens // 2, 7, 0)):
            x[t, h, j], rows[t, h] = bad, False
        got, lse = check(x, k, v, body, f"{bad}", rows=rows)
        assert np.isnan(got[~rows]).all() and np.isnan(lse[~rows]).all(), bad
        # keys of one sign: every score of such a row is infinite, and of one sign; small keys, and keys without those channels: a largest number in its place
        # would not overflow
        none = k.copy()
        none[..., [0, 5, d - 1]] = 0.0
        for what, other in (("positive", np.abs(k) + 0.1), ("small", k * 0.02), ("sparse", none)):
            got, lse = check(x, rounded(other), v, body, f"{bad}, {what} keys", rows=rows)
            assert np.isnan(got[~rows]).all() and np.isnan(lse[~rows]).all(), (bad, what)


@pytest.mark.parametrize("body", BODIES)
def test_the_largest_finite_queries(body):
    """Up to the largest bf16 number, against keys near 2^-100 under a scale that brings the scores to a few nats."""
    r = np.random.default_rng(6)
    n, d, tokens = 700, 64, BODIES[body][0]
    big = W.bf16_bits_to_f64(np.array([0x7F7F], np.uint16))[0]
    q = r.choice([0.9, 0.95, 1.0], (tokens, HQ, d)) * big
    q[:, :, 1:] *= 2.0 ** -9
    k = r.standard_normal((n, HKV, d)) * 2.0 ** -99
    check(rounded(q), rounded(k), rounded(r.standard_normal((n, HKV, d))), body, "largest", sm_scale=2.0 ** -28)


@pytest.mark.parametrize("body", BODIES)
@pytest.mark.parametrize("d", [64, 128])
def test_scales_behind_the_end_have_no_say(body, d):
    """Bit for bit: neither in the values nor in the form that a page's sums take."""
    r = np.random.default_rng(8)
    tokens, flags, _ = BODIES[body]
    for n in (75, 403, 2005):
        q, k, v = (rounded(r.standard_normal((m, h, d))) for m, h in ((tokens, HQ), (n, HKV), (n, HKV)))
        one, *others = (attend(q, k, v, tokens, stale=stale, flags=flags)[:2] for stale in (130, 0, 27, 254, 255))
        assert all(np.array_equal(a, b) for other in others for a, b in zip(one, other))
