"""CPU oracle of the quantised cache and of the rotary forms (TEST INFRASTRUCTURE ONLY).

Plain fp64 statements, in numpy, of what the calls on the 8-bit cache are defined to do: a row of values is held as e4m3 codes and one power of
two, the least 2^e (e >= -100) with max|x| <= 448 * 2^e; a code is the e4m3 number nearest to x * 2^-e (ties to the even code).  The cache stands in for
the bf16 one while a sequence's function calls run (paper Section 5.4: the cache is kept in GPU memory if that is cheapest).  Attention over it is
attention over the values that it stands for, which are bf16 values, so the bf16 oracle evaluates it.

Nothing here imports, or is imported by, the CUDA package.  Pins (tests/test_kv8_pins.py): the table of all 256 codes against torch's; rounding against a
search over that table; the scale's two inequalities; idempotence; rotations against complex multiplication and oracle/rope.py.
"""
from __future__ import annotations

import math

import numpy as np


def _code_table() -> np.ndarray:
    """Value of every byte: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7f and 0xff are NaN."""
    t = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        t[b] = math.nan if b & 0x7F == 0x7F else -x if b & 0x80 else x
    return t


CODES = _code_table()


def quantise(x: np.ndarray):
    """x: float64 [..., d] -> (codes uint8 [..., d], scale bytes uint8 [...])."""
    most = np.abs(x).max(axis=-1)
    fine = np.isfinite(x).all(axis=-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        _, e = np.frexp(np.where(fine & (most > 0), most, 2.0 ** -120) / 448.0)      # most / 448 in [2^(e-1), 2^e)
    e = np.where(most <= 448.0 * 2.0 ** (e - 1.0), e - 1, e)
    e = np.maximum(e, -100)
    y = np.where(fine[..., None], x, 0.0) * 2.0 ** -e[..., None].astype(np.float64)
    # a's binade (from 2^-6 on, below it the subnormal one) has eight steps: whole steps, ties to even, count the codes up from it
    a = np.abs(y)
    power = np.where(a > 0, np.maximum(np.frexp(a)[1] - 1, -6), -6)
    steps = np.rint(np.ldexp(a, 3 - power)).astype(np.int32)
    code = ((power + 6) * 8 + steps).astype(np.uint8) | np.where(np.signbit(y), 0x80, 0).astype(np.uint8)
    byte = np.where(fine, e + 127, 255).astype(np.uint8)
    return np.where(fine[..., None], code, 0).astype(np.uint8), byte


def values(codes: np.ndarray, byte: np.ndarray) -> np.ndarray:
    """What codes [..., d] and scale bytes [...] stand for, float64."""
    scale = np.where(byte == 255, math.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return CODES[codes] * scale[..., None]


def append(pool: np.ndarray, scales: np.ndarray, q_indptr, kv_len_before, page_indptr, page_indices, k: np.ndarray, v: np.ndarray) -> None:
    """pool uint8 [pages][2][Hkv][16][d], scales uint8 [pages][Hkv][2][16]; k, v float64 [T][Hkv][d] (turned already), in place."""
    for b in range(len(kv_len_before)):
        for i in range(q_indptr[b + 1] - q_indptr[b]):
            pos = kv_len_before[b] + i
            page, slot = page_indices[page_indptr[b] + pos // 16], pos % 16
            for which, x in ((0, k), (1, v)):
                pool[page, which, :, slot], scales[page, :, which, slot] = quantise(x[q_indptr[b] + i])


def pool_values(pool: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """float64 [pages][2][Hkv][16][d]"""
    return values(pool, scales.transpose(0, 2, 1, 3))


def frequencies(rotary_dim, theta, scaling=None, factor=1.0, context=0, low=1.0, high=4.0, beta_fast=32.0, beta_slow=1.0, attention_factor=0.0):
    """(radians a position of each pair, factor on the rotated values)."""
    out, m = [], 1.0
    if scaling == "yarn":
        m = attention_factor if attention_factor > 0 else 0.1 * math.log(factor) + 1.0
        first, last = (rotary_dim * math.log(context / (2 * math.pi * b)) / (2 * math.log(theta)) for b in (beta_fast, beta_slow))
        first, last = max(math.floor(first), 0), min(math.ceil(last), rotary_dim - 1)
    for j in range(rotary_dim // 2):
        f = theta ** (-2.0 * j / rotary_dim)
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            turns = context * f / (2 * math.pi)
            if turns <= low:
                f = f / factor
            elif turns < high:
                t = (turns - low) / (high - low)
                f = (1 - t) * f / factor + t * f
        elif scaling == "yarn":
            t = min(max((j - first) / max(last - first, 1e-3), 0.0), 1.0)
            f = t * f / factor + (1 - t) * f
        out.append(f)
    return np.array(out), m


def turn(x: np.ndarray, pos: np.ndarray, freq: np.ndarray, m: float, layout: str) -> np.ndarray:
    """x float64 [T][H][d] -> the same, its first 2 * len(freq) values turned."""
    n = len(freq)
    a = np.asarray(pos, np.float64)[:, None, None] * freq
    c, s = m * np.cos(a), m * np.sin(a)
    i = np.arange(n) if layout == "half" else 2 * np.arange(n)
    j = i + n if layout == "half" else i + 1
    y = x.copy()
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y
