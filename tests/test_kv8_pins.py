"""Pins of oracle/kv8.py, and the host side of the quantised cache's calls (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kv8, rope
from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200 import workload as W


def test_codes_are_those_of_torch():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, kv8.CODES, equal_nan=True)


def rows(seed=1, n=400, d=64):
    r = np.random.default_rng(seed)
    x = r.standard_normal((n, d)) * np.exp2(r.integers(-30, 30, (n, 1)))
    x[0], x[1, 1:], x[2], x[3], x[4, ::2] = 0.0, 0.0, 448.0, np.nextafter(448.0, 1e9), 2.0 ** -9
    x[5], x[6, 3], x[7, 5], x[8] = 2.0 ** -115, np.nan, -np.inf, 3e38
    return x


def test_quantise_picks_the_nearest_code_and_the_least_scale():
    x = rows()
    codes, byte = kv8.quantise(x)
    fine = np.isfinite(x).all(1)
    assert (byte[~fine] == 255).all() and (codes[~fine] == 0).all() and not fine[6] and not fine[7]
    e = byte[fine].astype(int) - 127
    most = np.abs(x[fine]).max(1)
    assert (most <= 448 * 2.0 ** e).all() and (e >= -100).all()
    assert ((most > 448 * 2.0 ** (e - 1)) | (e == -100)).all()
    y = x[fine] / 2.0 ** e[:, None]
    finite = kv8.CODES[np.isfinite(kv8.CODES)]
    assert np.array_equal(np.abs(kv8.CODES[codes[fine]] - y), np.abs(y[..., None] - finite).min(-1))
    again, byte2 = kv8.quantise(kv8.values(codes, byte)[fine])      # nothing moves a second time
    assert np.array_equal(kv8.values(again, byte2), kv8.values(codes, byte)[fine])
    # ties as torch's cast has them
    t = torch.from_numpy(y).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    same = torch.from_numpy(y).float().double().numpy() == y
    assert np.array_equal(t[same], codes[fine][same])
    assert np.array_equal(kv8.CODES[kv8.quantise(np.array([[448.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10]]))[0]], [[448.0, 1.0, 1.25, 0.0, 2.0 ** -8]])


def test_values_are_bf16_values():
    x = rows(2)
    codes, byte = kv8.quantise(x)
    v = kv8.values(codes, byte)[np.isfinite(x).all(1)]
    assert np.array_equal(torch.from_numpy(v).bfloat16().double().numpy(), v)


def test_turns_against_the_rotate_half_oracle_and_complex_products():
    r = np.random.default_rng(3)
    x, pos = r.standard_normal((5, 3, 64)), np.array([0, 1, 17, 4000, 131000])
    f, m = kv8.frequencies(64, 500000.0)
    assert m == 1.0 and np.allclose(kv8.turn(x, pos, f, m, "half"), rope.rotate(x, pos, 500000.0), rtol=0, atol=1e-9)
    f, m = kv8.frequencies(24, 10000.0, "yarn", 4.0, 2048)
    y = kv8.turn(x, pos, f, m, "interleaved")
    z = (x[..., 0:24:2] + 1j * x[..., 1:24:2]) * m * np.exp(1j * pos[:, None, None] * f)
    assert np.allclose(y[..., 0:24:2], z.real, atol=1e-9) and np.allclose(y[..., 1:24:2], z.imag, atol=1e-9) and np.array_equal(y[..., 24:], x[..., 24:])


@pytest.mark.parametrize("scaling,more", [(None, {}), ("linear", dict(factor=8.0)), ("bands", dict(factor=8.0, context=8192)),
                                          ("yarn", dict(factor=4.0, context=4096)), ("yarn", dict(factor=16.0, context=2048, attention_factor=1.5))])
@pytest.mark.parametrize("head_dim,rotary_dim,theta", [(128, 0, 500000.0), (64, 24, 10000.0), (256, 256, 1e6), (80, 2, 10000.0)])
def test_table_of_frequencies(head_dim, rotary_dim, theta, scaling, more):
    t = B.asynclm_rope_table(head_dim, theta, rotary_dim, "interleaved", scaling, **more)
    f, m = kv8.frequencies(rotary_dim or head_dim, theta, scaling, **more)
    assert t.rotary_dim == (rotary_dim or head_dim) and t.layout == 1 and abs(t.factor - m) < 1e-12
    got = np.array(t.turns) * 2 * np.pi
    # both sides work in fp64, with a power, a few products and a mixture
    assert np.allclose(got[:len(f)], f, rtol=1e-12, atol=0) and not got[len(f):].any()


@pytest.mark.parametrize("bad", [dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(rotary_dim=3), dict(rotary_dim=130), dict(rotary_dim=-2),
                                 dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(scaling="linear", factor=0.5),
                                 dict(scaling="linear", factor=float("nan")), dict(scaling="bands", factor=8.0), dict(scaling="bands", factor=8.0, context=8192, high_freq_factor=1.0),
                                 dict(scaling="yarn", factor=4.0), dict(scaling="yarn", factor=4.0, context=4096, beta_fast=0.5),
                                 dict(scaling="yarn", factor=4.0, context=4096, attention_factor=-1.0)])
def test_table_refusals(bad):
    with pytest.raises(B.AsynclmError) as e:
        B.asynclm_rope_table(**{"head_dim": 128, **bad})
    assert e.value.status == -1


def test_unknown_layout_and_scaling_are_named():
    with pytest.raises(ValueError, match="layout"):
        B.asynclm_rope_table(128, layout="quarter")
    with pytest.raises(ValueError, match="scaling"):
        B.asynclm_rope_table(128, scaling="ntk")


def test_struct_sizes():
    assert ctypes.sizeof(B.CRope) == 72 and ctypes.sizeof(B.CRopeTable) == 24 + 1024
    assert ctypes.sizeof(B.CRopeRows) == 40 and ctypes.sizeof(B.CKv8Rows) == 56


def test_calls_refuse_plans_that_cannot_run():
    """A plan made on the host only, and no plan at all: an error, and no CUDA call."""
    shape = W.Shape(8, 2, 64, 16)
    plan = B.plan_host(shape, 8, [0, 1], [20], [0, 2], [3, 4], kv8=True)
    lib, rows = B.load(), B.CKv8Rows()
    for handle in (None, plan.handle):
        assert lib.asynclm_kv8_append(handle, ctypes.byref(rows), 256, 256, None, None) == -1
        assert lib.asynclm_kv8_attn_mixed(handle, 256, 256, 256, 256, None, None) == -1
        assert lib.asynclm_kv8_gather(handle, 256, 256, 1, 256, 256, 256, 256, None) == -1


def test_tensors_that_do_not_fit_are_named():
    """Shapes, types and strides that the C call cannot see."""
    with pytest.raises(ValueError, match="k_new"):
        B.asynclm_kv8_append(None, torch.zeros(2, 2, 64, dtype=torch.bfloat16), None, None, None)      # not on the GPU
    with pytest.raises(ValueError, match="kv8_pool"):
        B._cache8(torch.zeros(4, dtype=torch.uint8), torch.zeros(4, dtype=torch.uint8))
