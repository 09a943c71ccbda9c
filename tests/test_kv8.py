"""The quantised cache on the GPU against its fp64 oracle (oracle/kv8.py), and attention over it against the bf16 oracle, to which the cache's
values, which are bf16 values, are handed.

Tolerances, before the first run.  Codes and scales of unrotated rows, read-back and untouched bytes: exact.  Rotated rows: both sides round the same
real number once, ours from an fp32 value within 2^-20 of itself, so a value may fall on the other side of a rounding boundary, by one step, with
a probability of about that error over the step: 2^-20 / 2^-9 = 0.2 % for bf16, 2^-20 / 2^-4 for codes; and a row's exponent may differ where its
maximum is 448 * 2^e to that accuracy, which no case has.
Attention: the output is rounded to bf16 (by 2^-8 of it at most) and the weights to f16 on the way (by 2^-11 of each at most, and not all the same way), so
with A = sum_j p_j |V_j| >= |out|:  |error| <= 1.1 * 2^-8 A + 1e-30.
lse: fp32 sums of d products, 2^-24 * d * sum|q_i k_i| * scale <= 2^-17 * 40 here, and the exponentials' 2^-22: 4e-4."""
import numpy as np
import pytest
import torch

from gpu_util import to_bits, to_dev
from oracle import kv8, oracle
from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200 import workload as W

pytestmark = pytest.mark.gpu
LSE_ABS = 4e-4


def codes_of_random_pool(wl, seed, spread=0):
    """Codes and scale bytes of the workload's pool, every slot quantised; `spread`: rows are scaled by powers of two up to 2^+-spread."""
    x = W.bf16_bits_to_f64(wl.kv_pool)
    x = np.where(np.isfinite(x), x, 1.0)
    if spread:
        x = x * np.exp2(np.random.default_rng(seed).integers(-spread, spread + 1, x.shape[:-1] + (1,)))
    codes, byte = kv8.quantise(x)
    return codes, np.ascontiguousarray(byte.transpose(0, 2, 1, 3))


def poison(wl, st, codes, byte, seed):
    """NaN codes and any scale bytes in every slot that the step does not read or write."""
    used = np.zeros((wl.num_pages, 16), bool)
    for b in range(st.batch):
        if st.q_len[b] == 0:
            continue
        for pos in range(int(st.kv_len_before[b] + st.q_len[b])):
            used[st.page_indices[st.page_indptr[b] + pos // 16], pos % 16] = True
    r = np.random.default_rng(seed)
    codes.transpose(0, 3, 1, 2, 4)[~used] = 0x7F
    byte.transpose(0, 3, 1, 2)[~used] = r.choice([0, 254, 255, 130], size=(int((~used).sum()),) + byte.shape[1:3])
    return codes, byte


def dev8(codes, byte):
    return (torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn), torch.from_numpy(byte).cuda().view(torch.float8_e8m0fnu))


def plan_of(wl, st, **opts):
    return B.asynclm_plan(wl.shape, wl.num_pages, st.q_indptr, st.kv_len_before, st.page_indptr, st.page_indices, **opts)


def bits_of(values):
    return W.f32_to_bf16_bits(values.astype(np.float32))


def run_and_check(wl, codes, byte, st=None, sm_scale=0.0, lse=True, k_new=None, v_new=None, what="", **opts):
    """append + attention on the GPU against the oracles; codes and byte are changed to what the append leaves."""
    st = st or wl.steps[0]
    pool, scales = dev8(codes, byte)
    k_new, v_new = st.k_new if k_new is None else k_new, st.v_new if v_new is None else v_new
    out = torch.full((st.total_q, wl.shape.num_q_heads, wl.shape.head_dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse_dev = torch.full((st.total_q, wl.shape.num_q_heads), float("nan"), device="cuda") if lse else None
    plan = plan_of(wl, st, sm_scale=sm_scale, kv8=True, **opts)
    B.asynclm_kv8_append(plan, to_dev(k_new), to_dev(v_new), pool, scales)
    B.asynclm_kv8_attn_mixed(plan, to_dev(st.q), pool, scales, out, lse_dev)
    torch.cuda.synchronize()
    assert B.last_device_status(plan) == 0
    kv8.append(codes, byte, st.q_indptr, st.kv_len_before, st.page_indptr, st.page_indices, W.bf16_bits_to_f64(k_new), W.bf16_bits_to_f64(v_new))
    assert np.array_equal(pool.view(torch.uint8).cpu().numpy(), codes), f"{what}: codes"
    assert np.array_equal(scales.view(torch.uint8).cpu().numpy(), byte), f"{what}: scales"
    values = kv8.pool_values(codes, byte)
    with np.errstate(over="ignore", invalid="ignore"):
        bf16 = bits_of(values)
        sides = bits_of(np.concatenate([values[:, :1], np.abs(values[:, 1:])], 1))
    args = (st.q, st.q_indptr, st.kv_len_before, st.page_indptr, st.page_indices, sm_scale)
    ref, ref_lse = oracle.attn_mixed(bf16, *args)
    weight, _ = oracle.attn_mixed(sides, *args)
    got = W.bf16_bits_to_f64(to_bits(out))
    seen = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN where the oracle has none, or none where it has"
    err = np.abs(got - ref)[seen]
    assert (err <= 1.1 * 2.0 ** -8 * weight[seen] + 1e-30).all(), f"{what}: {(err / (weight[seen] + 1e-30)).max() * 2 ** 8:.3f} of the bound"
    if lse:
        d = np.abs(lse_dev.cpu().numpy().astype(np.float64) - ref_lse)
        rows = seen.all(-1)
        assert (d[rows] <= LSE_ABS).all(), f"{what}: lse {d[rows].max():.3g}"
    return plan, got


CTX = [0, 1, 15, 16, 17, 129, 700, 0, 300, 47, 2500]
Q = [1, 1, 1, 1, 12, 5, 1, 33, 0, 70, 1]


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (4, 4, 64), (8, 1, 64), (2, 1, 128), (32, 8, 128), (16, 2, 128), (4, 2, 128), (8, 8, 128)])
def test_append_and_attention_over_shapes_and_ragged_lengths(Hq, Hkv, d):
    shape = W.Shape(Hq, Hkv, d, 16)
    wl = W.make_single_step("ragged", shape, CTX, Q, seed=2000 + Hq * 7 + d, extra_pages=[0, 1, 0, 0, 2, 0, 0, 1, 3, 0, 1], interleave_pages=True)
    codes, byte = poison(wl, wl.steps[0], *codes_of_random_pool(wl, 5), seed=6)
    plan, _ = run_and_check(wl, codes, byte, what=f"ragged {Hq}/{Hkv}/{d}")
    assert plan.info["total_q"] == sum(Q)


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (8, 2, 64), (8, 8, 64)])
def test_long_contexts_are_cut_and_joined(Hq, Hkv, d):
    wl = W.make_single_step("long", W.Shape(Hq, Hkv, d, 16), [9000, 33, 4111], [1, 1, 2], seed=2100 + d)
    codes, byte = codes_of_random_pool(wl, 7)
    plan, _ = run_and_check(wl, codes, byte, what="long")
    assert plan.info["num_split_units"] > 0


@pytest.mark.parametrize("chunk", [64, 192, 512, 1 << 20])
@pytest.mark.parametrize("d", [64, 128])
def test_fixed_chunk_lengths(chunk, d):
    wl = W.make_single_step("chunks", W.Shape(8, 2, d, 16), [1500, 64, 127, 900], [1, 1, 40, 7], seed=2200)
    run_and_check(wl, *codes_of_random_pool(wl, 8), what=f"chunk {chunk}", kv_chunk_tokens=chunk)


@pytest.mark.parametrize("Hq", [2, 4, 8, 16])
def test_spans_on_the_warp_body(Hq):
    wl = W.make_single_step("spans", W.Shape(Hq, 2, 128, 16), [300, 0, 40, 700], [64, 130, 9, 1], seed=2300)
    plan, _ = run_and_check(wl, *codes_of_random_pool(wl, 9), what="warp body", flags=B.PLAN_NO_TENSOR_PATH)
    assert plan.info["num_items_tensor"] == 0


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (8, 1, 64), (8, 8, 128), (4, 2, 64)])
def test_spans_of_every_kind_beside_decode_rows(Hq, Hkv, d):
    wl = W.make_single_step("mixed", W.Shape(Hq, Hkv, d, 16), [300, 2000, 0, 17, 900, 63, 4000, 1], [64, 1, 300, 1, 129, 128, 1, 31], seed=2400 + d,
                            interleave_pages=True)
    codes, byte = poison(wl, wl.steps[0], *codes_of_random_pool(wl, 10), seed=11)
    run_and_check(wl, codes, byte, what="mixed")
    # and spans alone
    wl = W.make_single_step("spans", W.Shape(Hq, Hkv, d, 16), [300, 0, 77], [130, 515, 64], seed=2500 + d)
    codes, byte = poison(wl, wl.steps[0], *codes_of_random_pool(wl, 12), seed=13)
    run_and_check(wl, codes, byte, what="spans")


@pytest.mark.parametrize("spread", [6, 40, 60])
@pytest.mark.parametrize("q_lens", [[1, 1, 1], [40, 1, 90]])
def test_row_scales_far_apart(spread, q_lens):
    """Rows of V whose scales lie up to 2^80 apart: the small ones count where the large ones have no weight, and only there.  Scores are small."""
    wl = W.make_single_step("spread", W.Shape(8, 2, 128, 16), [700, 40, 1200], q_lens, seed=2600)
    codes, byte = codes_of_random_pool(wl, 14, spread)
    byte[:, :, 0] = np.random.default_rng(15).integers(116, 120, byte[:, :, 0].shape)
    run_and_check(wl, codes, byte, what="spread")


@pytest.mark.parametrize("q_lens", [[1, 1, 1], [40, 1, 90]])
def test_scores_far_apart(q_lens):
    """One key takes all the weight, another one's score lies hundreds below: exponentials under- and overflow on the way without a trace."""
    wl = W.make_single_step("scores", W.Shape(8, 2, 64, 16), [700, 40, 1200], q_lens, seed=2700)
    codes, byte = codes_of_random_pool(wl, 16)
    st = wl.steps[0]
    q = W.bf16_bits_to_f64(st.q) * np.exp2(np.random.default_rng(17).integers(-12, 5, (st.total_q, 8, 1)))
    st.q[...] = bits_of(q)
    pool, scales = dev8(codes, byte)
    out = torch.empty((st.total_q, 8, 64), dtype=torch.bfloat16, device="cuda")
    plan = plan_of(wl, st, kv8=True)
    B.asynclm_kv8_append(plan, to_dev(st.k_new), to_dev(st.v_new), pool, scales)
    B.asynclm_kv8_attn_mixed(plan, to_dev(st.q), pool, scales, out)
    torch.cuda.synchronize()
    bf16 = bits_of(kv8.pool_values(pool.view(torch.uint8).cpu().numpy(), scales.view(torch.uint8).cpu().numpy()))
    ref, _ = oracle.attn_mixed(bf16, st.q, st.q_indptr, st.kv_len_before, st.page_indptr, st.page_indices)
    # scores up to 2^4 * 8: their fp32 sums are off by 2^-24 * 64 * 130 at most, and weights by that factor; |V| < 6
    err = np.abs(W.bf16_bits_to_f64(to_bits(out)) - ref)
    assert err.max() <= 6 * (1.1 * 2.0 ** -8 + 64 * 130 * 2.0 ** -24)


def test_rows_that_are_not_finite_reach_those_that_see_them_only():
    """A span whose middle rows hold NaN and infinity (K of one, V of another): tokens in front are untouched, the others NaN; so is a decode row behind
    a NaN key; and zero rows, whose scale is the least, change nothing."""
    for d, q_len in ((128, 7), (128, 60), (64, 90)):
        wl = W.make_single_step("nan", W.Shape(8, 2, d, 16), [100, 33, 50], [q_len, 1, 1], seed=2800)
        st = wl.steps[0]
        k, v = st.k_new.copy(), st.v_new.copy()
        k[q_len // 2, 0, 3], v[q_len // 3, 1, 5] = 0x7FC0, 0xFF80       # a NaN key of kv head 0, an infinite value of kv head 1
        v[1] = 0
        codes, byte = codes_of_random_pool(wl, 18)
        page = st.page_indices[st.page_indptr[1]]
        byte[page, 0, 0, 5] = 255                                         # an old NaN key of the second sequence's first page, kv head 0
        codes[page, 0, 0, 5] = 0
        byte[page, 1, 1, :16], codes[page, 1, 1, :16] = 27, 0             # and 16 zero rows of V of kv head 1
        _, got = run_and_check(wl, codes, byte, k_new=k, v_new=v, what=f"not finite, {d}")
        nan = np.isnan(got).all(-1)
        assert nan[q_len // 2:q_len, :4].all() and not nan[:q_len // 2, :4].any()
        assert nan[q_len // 3:q_len, 4:].all() and not nan[:q_len // 3, 4:].any()
        assert nan[q_len, :4].all() and not nan[q_len, 4:].any() and not nan[q_len + 1].any()


@pytest.mark.parametrize("d", [64, 128])
def test_append_of_odd_rows(d):
    """Zero rows, values that become zeros, maxima at and beside 448 * 2^e, the largest bf16, negative zeros, infinities and NaN."""
    wl = W.make_single_step("odd", W.Shape(2, 2, d, 16), [0, 15, 32], [20, 3, 17], seed=2900)
    st = wl.steps[0]
    x = W.bf16_bits_to_f64(st.k_new).copy()
    x[0], x[1, 0], x[1, 1, 1:] = 0.0, 448.0, 0.0
    x[2], x[3, 0], x[3, 1, 0] = -450.0, 2.0 ** -115, 3.38e38
    x[4, 0, ::2], x[5, 0, 7], x[6, 1, 0], x[7] = -0.0, np.inf, np.nan, 2.0 ** -100
    x[8:16] *= np.exp2(np.random.default_rng(1).integers(-60, 60, (8, 2, 1)))
    k, v = bits_of(x), bits_of(x[::-1])
    codes, byte = codes_of_random_pool(wl, 20)
    pool, scales = dev8(codes, byte)
    plan = plan_of(wl, st, kv8=True)
    B.asynclm_kv8_append(plan, to_dev(k), to_dev(v), pool, scales)
    kv8.append(codes, byte, st.q_indptr, st.kv_len_before, st.page_indptr, st.page_indices, W.bf16_bits_to_f64(k), W.bf16_bits_to_f64(v))
    torch.cuda.synchronize()
    assert np.array_equal(pool.view(torch.uint8).cpu().numpy(), codes) and np.array_equal(scales.view(torch.uint8).cpu().numpy(), byte)


def ulp_diff(a, b):
    key = lambda x: np.where(x & 0x8000, 0x8000 - (x & 0x7FFF).astype(np.int32), 0x8000 + (x & 0x7FFF).astype(np.int32))  # noqa: E731
    return np.abs(key(a) - key(b))


def nearly(got_bits, values):
    """bf16 rows: equal to fp64 values rounded once, but for a step where a value lies on a boundary (see above)."""
    ref = bits_of(values)
    diff = got_bits != ref
    return diff.mean() < 4e-3 and ulp_diff(got_bits[diff], ref[diff]).max(initial=0) <= 1


def far(shape, ctx, q_lens, seed):
    """A step at positions `ctx` of which a small pool holds the last pages only: the ones in front are all the sequence's first, which an append does
    not touch."""
    near = [c if c <= 256 else 112 + c % 16 for c in ctx]
    wl = W.make_single_step("far", shape, near, q_lens, seed=seed)
    st = wl.steps[0]
    pages = [np.concatenate([np.full((c - n) // 16, st.page_indices[a], np.int32), st.page_indices[a:b]])
             for c, n, a, b in zip(ctx, near, st.page_indptr[:-1], st.page_indptr[1:])]
    st.page_indices, st.page_indptr = np.concatenate(pages).astype(np.int32), np.concatenate([[0], np.cumsum([len(x) for x in pages])]).astype(np.int32)
    st.kv_len_before = np.array(ctx, np.int32)
    return wl


SCALINGS = [(None, {}), ("linear", dict(factor=8.0)), ("bands", dict(factor=8.0, context=8192)), ("yarn", dict(factor=4.0, context=4096))]


@pytest.mark.parametrize("scaling,more", SCALINGS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("Hq,Hkv,d,rotary", [(32, 8, 128, 0), (8, 2, 64, 32), (5, 5, 64, 20), (16, 2, 128, 8), (8, 8, 64, 62), (2, 1, 128, 2)])
def test_rotated_append(Hq, Hkv, d, rotary, layout, scaling, more):
    """Keys turned and quantised, queries turned, out of a fused projection's output, at positions up to 131 K."""
    wl = far(W.Shape(Hq, Hkv, d, 16), [0, 5, 131, 4000, 131000], [9, 1, 18, 1, 3], seed=3000 + d)
    st = wl.steps[0]
    qkv = torch.cat([to_dev(st.q), to_dev(st.k_new), to_dev(st.v_new)], 1).contiguous()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    codes, byte = codes_of_random_pool(wl, 21)
    pool, scales = dev8(codes, byte)
    q_out = torch.full((st.total_q, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    table = B.asynclm_rope_table(d, 500000.0, rotary, layout, scaling, **more)
    B.asynclm_kv8_append(plan_of(wl, st, kv8=True), k, v, pool, scales, table, q, q_out)
    torch.cuda.synchronize()
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(st.kv_len_before, st.q_len)])
    turn = lambda bits: kv8.turn(W.bf16_bits_to_f64(bits), pos, *kv8.frequencies(rotary or d, 500000.0, scaling, **more), layout)  # noqa: E731
    assert nearly(to_bits(q_out), turn(st.q))
    assert np.array_equal(to_bits(qkv), np.concatenate([st.q, st.k_new, st.v_new], 1))
    kv8.append(codes, byte, st.q_indptr, st.kv_len_before, st.page_indptr, st.page_indices, turn(st.k_new), W.bf16_bits_to_f64(st.v_new))
    assert np.array_equal(scales.view(torch.uint8).cpu().numpy(), byte)
    got = pool.view(torch.uint8).cpu().numpy()
    diff = got != codes
    assert not diff[:, 1].any() and diff.mean() < 1e-3
    assert np.abs(got[diff].astype(int) - codes[diff].astype(int)).max(initial=0) <= 1      # (neighbouring codes of one sign)


@pytest.mark.parametrize("tokens", [0, 1, 3, 593, 5000])
@pytest.mark.parametrize("Hq,Hkv,d,rotary,layout", [(32, 8, 128, 128, "half"), (3, 1, 64, 24, "half"), (7, 2, 80, 40, "interleaved"), (4, 4, 256, 192, "half"),
                                                    (2, 1, 8, 6, "half"), (9, 3, 72, 20, "half"), (33, 1, 64, 64, "interleaved")])
def test_rope_apply(tokens, Hq, Hkv, d, rotary, layout):
    r = np.random.default_rng(31)
    q, k = (bits_of(r.standard_normal((tokens, h, d))) for h in (Hq, Hkv))
    pos = r.integers(-5, 200000, tokens).astype(np.int32)
    table = B.asynclm_rope_table(d, 10000.0, rotary, layout, "yarn", factor=4.0, context=4096)
    f, m = kv8.frequencies(rotary, 10000.0, "yarn", 4.0, 4096)
    want = [kv8.turn(W.bf16_bits_to_f64(x), pos, f, m, layout) for x in (q, k)]
    p = torch.from_numpy(pos).cuda()
    # rows of a wider tensor in, a wider one out; then one tensor by itself, in place
    both = torch.cat([to_dev(q), to_dev(k)], 1).contiguous()
    out = torch.full((tokens, Hq + Hkv + 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
    B.asynclm_rope_apply(table, p, both[:, :Hq], out[:, 1:Hq + 1], both[:, Hq:], out[:, Hq + 1:-1])
    here = to_dev(q)
    B.asynclm_rope_apply(table, p, here, here)
    torch.cuda.synchronize()
    if tokens == 0:
        return
    assert nearly(to_bits(out[:, 1:Hq + 1].contiguous()), want[0]) and nearly(to_bits(out[:, Hq + 1:-1].contiguous()), want[1])
    assert (out[:, 0] == 7.0).all() and (out[:, -1] == 7.0).all()
    assert np.array_equal(to_bits(here), to_bits(out[:, 1:Hq + 1].contiguous()))
    assert np.array_equal(to_bits(here)[..., rotary:], q[..., rotary:])


def test_values_that_do_not_turn_pass_through_bit_for_bit():
    """NaN payloads, infinities and subnormal numbers beyond rotary_dim."""
    q = np.arange(2 * 3 * 128, dtype=np.uint16).reshape(2, 3, 128) * 91
    for layout in ("half", "interleaved"):
        t = to_dev(q.copy())
        B.asynclm_rope_apply(B.asynclm_rope_table(128, rotary_dim=32, layout=layout), torch.tensor([5, 900], dtype=torch.int32, device="cuda"), t, t)
        torch.cuda.synchronize()
        assert np.array_equal(to_bits(t)[..., 32:], q[..., 32:])


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (32, 8, 128), (3, 3, 128)])
@pytest.mark.parametrize("lengths", [[0, 1, 0], [40, 700, 17], [1, 0, 3000]])
def test_read_back_is_exact(Hq, Hkv, d, lengths):
    """Ranges from any position, empty ones, ones that end inside a page or reach over the step's new rows; untouched rows around them."""
    wl = W.make_single_step("gather", W.Shape(Hq, Hkv, d, 16), [120, 720, 3100], [1, 0, 5], seed=3300, interleave_pages=True)
    st = wl.steps[0]
    codes, byte = codes_of_random_pool(wl, 33, 30)
    pool, scales = dev8(codes, byte)
    first = np.array([81 - min(lengths[0], 1), 13, 77], np.int32)
    if lengths[2] == 3000:
        first[2] = 105      # up to the last of the new rows
    indptr = np.concatenate([[0], np.cumsum(lengths)])
    k, v = (torch.full((int(indptr[-1]), Hkv, d), -1.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    plan = plan_of(wl, st, kv8=True)
    B.asynclm_kv8_gather(plan, torch.from_numpy(indptr).cuda(), torch.from_numpy(first).cuda(), pool, scales, k, v)
    torch.cuda.synchronize()
    assert B.last_device_status(plan) == 0
    values = kv8.pool_values(codes, byte)
    for b in range(3):
        for i in range(lengths[b]):
            pos = int(first[b]) + i
            row = values[st.page_indices[st.page_indptr[b] + pos // 16], :, :, pos % 16]
            assert np.array_equal(k[indptr[b] + i].double().cpu().numpy(), row[0]) and np.array_equal(v[indptr[b] + i].double().cpu().numpy(), row[1])


def test_read_back_leaves_out_and_reports_what_lies_outside():
    wl = W.make_single_step("gather", W.Shape(2, 2, 64, 16), [40, 30], [1, 1], seed=3400)
    st = wl.steps[0]
    pool, scales = dev8(*codes_of_random_pool(wl, 34))
    for first, pages in (([30, 0], None), ([-3, 0], None), ([0, 0], 999999)):
        plan = plan_of(wl, st, kv8=True)
        if pages is not None:      # a sequence without new tokens, whose pages the planner does not look at
            ids = st.page_indices.copy()
            ids[int(st.page_indptr[0])] = pages
            plan = B.asynclm_plan(wl.shape, wl.num_pages, [0, 0, 1], st.kv_len_before, st.page_indptr, ids, kv8=True)
        k, v = (torch.full((25, 2, 64), -1.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        B.asynclm_kv8_gather(plan, torch.tensor([0, 20, 25], device="cuda"), torch.tensor(first, dtype=torch.int32, device="cuda"), pool, scales, k, v)
        torch.cuda.synchronize()
        assert B.last_device_status(plan) == 45
        left = {30: range(11, 20), -3: range(0, 3), 0: range(0, 16)}[first[0]]
        assert all((k[i] == -1).all() and (v[i] == -1).all() for i in left)
        assert not any((k[i] == -1).all() for i in range(25) if i not in left)


def test_another_stream_a_graph_and_repeated_launches():
    """The calls go to the stream that they are given; a captured step replays to the same bits, split contexts among it."""
    wl = W.make_single_step("graph", W.Shape(8, 2, 128, 16), [9000, 100, 31], [1, 40, 1], seed=3500)
    st = wl.steps[0]
    codes, byte = codes_of_random_pool(wl, 35)
    pool, scales = dev8(codes, byte)
    q, k, v = to_dev(st.q), to_dev(st.k_new), to_dev(st.v_new)
    q2, out, lse = torch.empty_like(q), torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    table = B.asynclm_rope_table(128)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    plan = plan_of(wl, st, kv8=True, stream=side)

    def step(stream=None):
        B.asynclm_kv8_append(plan, k, v, pool, scales, table, q, q2, stream=stream)
        B.asynclm_kv8_attn_mixed(plan, q2, pool, scales, out, lse, stream=stream)
    step(side)
    side.synchronize()
    first = out.clone(), lse.clone()
    assert not (out == 0).all() and plan.info["num_split_units"] > 0
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
        step()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert B.last_device_status(plan) == 0
    # without the log-sum-exps
    out.zero_()
    B.asynclm_kv8_attn_mixed(plan, q2, pool, scales, out)
    torch.cuda.synchronize()
    assert torch.equal(out, first[0])


def test_refusals():
    shape = W.Shape(8, 2, 64, 16)
    wl = W.make_single_step("refuse", shape, [20], [1], seed=3600)
    st = wl.steps[0]
    pool, scales = dev8(*codes_of_random_pool(wl, 36))
    q, k, v, out = to_dev(st.q), to_dev(st.k_new), to_dev(st.v_new), to_dev(st.q)
    plan = plan_of(wl, st, kv8=True)
    table, other = B.asynclm_rope_table(64), B.asynclm_rope_table(128)
    wide = torch.zeros(4, 8, 72, dtype=torch.bfloat16, device="cuda")

    def refused(call, *args, **kw):
        with pytest.raises(B.AsynclmError) as e:
            call(*args, **kw)
        assert e.value.status == -1, (call, e.value)
    refused(B.asynclm_kv8_append, plan, k, v, pool, scales, other)                              # made for another head_dim
    refused(B.asynclm_kv8_append, plan, k, v, pool, scales, B.CRopeTable())                    # not initialised
    refused(B.asynclm_kv8_append, plan, k, v, pool, scales, None, q, out)                      # queries without positions to turn by
    flat = torch.zeros(1000, dtype=torch.uint8, device="cuda")
    refused(B.asynclm_kv8_append, plan, k, v, flat[1:], scales)                                # misaligned
    refused(B.asynclm_kv8_attn_mixed, plan, q, flat[1:], scales, out)
    refused(B.asynclm_kv8_attn_mixed, plan, q, pool, flat[1:], out)
    refused(B.asynclm_rope_apply, other, torch.zeros(1, dtype=torch.int32, device="cuda"), q, out)
    with pytest.raises(ValueError, match="q_out"):
        B.asynclm_kv8_append(plan, k, v, pool, scales, table, q)
    for bad in (dict(k_new=k.float()), dict(k_new=k.cpu()), dict(v_new=wide[:1, :2, :64]), dict(kv8_pool=pool.view(torch.uint8).int()),
                dict(kv8_scales=scales.transpose(0, 1))):
        args = dict(k_new=k, v_new=v, kv8_pool=pool, kv8_scales=scales) | bad
        with pytest.raises(ValueError, match=list(bad)[0]):
            B.asynclm_kv8_append(plan, **args)
    with pytest.raises(ValueError, match="positions"):
        B.asynclm_rope_apply(table, torch.zeros(3, dtype=torch.int32, device="cuda"), q, out)
    with pytest.raises(ValueError, match="positions"):
        B.asynclm_rope_apply(table, torch.zeros(1, dtype=torch.int64, device="cuda"), q, out)
    lib = B.load()
    import ctypes
    rows = B.CKv8Rows(k.data_ptr(), v.data_ptr(), None, None, 4, 0, 0)                         # a stride below a row
    assert lib.asynclm_kv8_append(plan.handle, ctypes.byref(rows), pool.data_ptr(), scales.data_ptr(), None, None) == -1
    assert lib.asynclm_kv8_gather(plan.handle, None, None, 3, pool.data_ptr(), scales.data_ptr(), k.data_ptr(), v.data_ptr(), None) == -1
    assert lib.asynclm_kv8_gather(plan.handle, None, None, 0, None, None, None, None, None) == 0
    torch.cuda.synchronize()


def test_steps_without_tokens():
    shape = W.Shape(8, 2, 64, 16)
    plan = B.asynclm_plan(shape, 4, [0, 0], [20], [0, 2], [1, 2], kv8=True)
    pool, scales = torch.zeros(4, 2, 2, 16, 64, dtype=torch.uint8, device="cuda"), torch.full((4, 2, 2, 16), 127, dtype=torch.uint8, device="cuda")
    none = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    B.asynclm_kv8_append(plan, none, none, pool, scales)
    B.asynclm_kv8_attn_mixed(plan, torch.zeros(0, 8, 64, dtype=torch.bfloat16, device="cuda"), pool, scales, torch.zeros(0, 8, 64, dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    assert B.last_device_status(plan) == 0
