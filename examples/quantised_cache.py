#!/usr/bin/env python
"""Serving steps over a quantised cache: prompts come in, tokens are decoded, one sequence is interrupted by a span, and
at the end a sequence is read back.

Per step one plan, and per layer two calls: `asynclm_kv8_append` turns the new keys and queries by their positions (YaRN
scaled frequencies) and writes keys and values into the layer's cache in 8 bits, straight out of the fused projection's
output, and `asynclm_kv8_attn_mixed` attends over it.  At the end `asynclm_kv8_gather` reads a sequence's keys and values
back in bf16, as a program does that hands a context over to another cache, `asynclm_rope_apply` turns its last queries
again by themselves, and a plain softmax over what was read back has to give what the last step gave.

    python examples/quantised_cache.py [--layers 4] [--sequences 8] [--prompt 700] [--steps 16] [--dim 128]

Prints one JSON line; weights and inputs are random."""
from __future__ import annotations

import argparse
import json
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2412_07017_b200 import binding as B      # noqa: E402
from paper_2412_07017_b200 import workload as W      # noqa: E402

PAGE = 16


class Cache:
    """Per-layer quantised pools, and pages handed to sequences as they grow."""

    def __init__(self, layers: int, shape: W.Shape, sequences: int, most_tokens: int):
        per_seq = -(-most_tokens // PAGE)
        self.shape, self.num_pages = shape, sequences * per_seq + 1
        Hkv, d = shape.num_kv_heads, shape.head_dim
        self.pools = [torch.empty((self.num_pages, 2, Hkv, PAGE, d), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(layers)]
        self.scales = [torch.empty((self.num_pages, Hkv, 2, PAGE), dtype=torch.float8_e8m0fnu, device="cuda") for _ in range(layers)]
        self.free = list(np.random.default_rng(0).permutation(self.num_pages))
        self.pages = [[] for _ in range(sequences)]
        self.lengths = np.zeros(sequences, np.int32)

    def plan(self, new: np.ndarray) -> B.Plan:
        """The plan of a step that appends new[b] tokens to every sequence b."""
        for b, n in enumerate(self.lengths + new):
            while len(self.pages[b]) * PAGE < n:
                self.pages[b].append(self.free.pop())
        page_indptr = np.concatenate([[0], np.cumsum([len(p) for p in self.pages])]).astype(np.int32)
        q_indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        return B.asynclm_plan(self.shape, self.num_pages, q_indptr, self.lengths, page_indptr, np.concatenate(self.pages).astype(np.int32), kv8=True)


def run(layers=4, sequences=8, prompt=700, steps=16, dim=128, heads=(32, 8), seed=0) -> dict:
    """The steps, and the comparison at the end.  Returns what is printed."""
    Hq, Hkv = heads
    shape = W.Shape(Hq, Hkv, dim, PAGE)
    rng = np.random.default_rng(seed)
    span = 48
    cache = Cache(layers, shape, sequences, prompt + steps + span)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    table = B.asynclm_rope_table(dim, 500000.0, scaling="yarn", factor=4.0, context=8192)
    lengths = rng.integers(1, prompt + 1, sequences).astype(np.int32)

    def step(new):
        plan = cache.plan(new)
        total = int(new.sum())
        # what a layer's fused projection leaves: a row of Hq + 2 Hkv heads for every token
        fused = [torch.randn((total, Hq + 2 * Hkv, dim), dtype=torch.bfloat16, device="cuda", generator=gen) for _ in range(layers)]
        q = torch.empty((total, Hq, dim), dtype=torch.bfloat16, device="cuda")
        out = torch.empty_like(q)
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for x, pool, scales in zip(fused, cache.pools, cache.scales):
            B.asynclm_kv8_append(plan, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], pool, scales, table, x[:, :Hq], q)
            B.asynclm_kv8_attn_mixed(plan, q, pool, scales, out)
        end.record()
        end.synchronize()
        if B.last_device_status(plan) != 0:
            raise RuntimeError("a step reported a device status")
        cache.lengths = cache.lengths + new
        return plan, fused[-1], out, begin.elapsed_time(end) * 1e3

    times = {"prompts_us": step(lengths)[3], "decode_us": []}
    for k in range(steps):
        new = np.ones(sequences, np.int32)
        if k == steps // 2:
            new[0] = span      # a call has returned: its message goes in between
        plan, fused, out, us = step(new)
        (times["decode_us"].append(us) if k != steps // 2 else times.update(interrupted_us=us))
    times["decode_us"] = float(np.median(times["decode_us"])) if times["decode_us"] else None

    # sequence 0 of the last layer, read back
    n = int(cache.lengths[0])
    rows = np.zeros(sequences + 1, np.int64)
    rows[1:] = n
    k_back, v_back = (torch.empty((n, Hkv, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.asynclm_kv8_gather(plan, torch.from_numpy(rows).cuda(), torch.zeros(sequences, dtype=torch.int32, device="cuda"), cache.pools[-1], cache.scales[-1],
                         k_back, v_back)
    q_last = torch.empty((1, Hq, dim), dtype=torch.bfloat16, device="cuda")
    B.asynclm_rope_apply(table, torch.tensor([n - 1], dtype=torch.int32, device="cuda"), fused[:1, :Hq], q_last)
    if B.last_device_status(plan) != 0:
        raise RuntimeError("reading back reported a device status")
    k, v = (x.double().repeat_interleave(Hq // Hkv, 1) for x in (k_back, v_back))
    p = torch.softmax(torch.einsum("qhd,khd->qhk", q_last.double(), k) / dim ** 0.5, -1)
    want = torch.einsum("qhk,khd->qhd", p, v)
    # bf16 out, f16 weights: 1.1 * 2^-8 of sum p |v|
    bound = 1.1 * 2.0 ** -8 * torch.einsum("qhk,khd->qhd", p, v.abs()) + 1e-30
    times["error_of_bound"] = float(((out[:1].double() - want).abs() / bound).max())
    bytes_16, bytes_8 = 4 * Hkv * dim, 2 * Hkv * (dim + 1)
    return {"what": "steps over a quantised cache", "layers": layers, "sequences": sequences, "tokens": int(cache.lengths.sum()), "head_dim": dim,
            "cache_bytes_a_token_and_layer": bytes_8, "of_bf16": bytes_8 / bytes_16, **times}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("sequences", 8), ("prompt", 700), ("steps", 16), ("dim", 128)):
        ap.add_argument("--" + name, type=int, default=value)
    got = run(**vars(ap.parse_args()))
    print(json.dumps(got))
    sys.exit(0 if got["error_of_bound"] <= 1 else 1)
