"""The quantised cache's calls by both ways into the library, and the example that uses them together."""
import ctypes
import importlib.util
import os
import subprocess
import types

import numpy as np
import pytest
import torch

from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200 import build as lib_build
from paper_2412_07017_b200 import workload as W
from test_span_ring import ambiguous_waits, three_items

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def bits(t):
    return t.cpu().contiguous().view(torch.uint8).numpy().tobytes()


@pytest.mark.gpu
@pytest.mark.parametrize("strided", [False, True])
def test_the_extension_and_ctypes_lead_to_the_same_call(monkeypatch, strided):
    if lib_build.build_call_ext() is None:
        pytest.skip("no C compiler or Python header here: the calls go through ctypes")
    assert B._calls()
    shape = W.Shape(8, 2, 64, 16)
    wl = W.make_single_step("calls", shape, [0, 40, 333], [3, 1, 20], seed=11)
    st = wl.steps[0]
    gen = torch.Generator(device="cuda").manual_seed(3)
    total, n = st.total_q, [3, 41, 353]
    fused = torch.randn((total, 12, 64), dtype=torch.bfloat16, device="cuda", generator=gen)
    q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    table = B.asynclm_rope_table(64, 10000.0, rotary_dim=32, layout="interleaved")
    positions = torch.arange(total, dtype=torch.int32, device="cuda") * 7
    indptr = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int64, device="cuda")
    first = torch.zeros(3, dtype=torch.int32, device="cuda")

    def everything():
        pool = torch.zeros((wl.num_pages, 2, 2, 16, 64), dtype=torch.uint8, device="cuda")
        scales = torch.zeros((wl.num_pages, 2, 2, 16), dtype=torch.uint8, device="cuda")
        # (the contexts stand for themselves: codes of one byte, scales of 1)
        pool.fill_(0x38), scales.fill_(127)
        plan = B.asynclm_plan(shape, wl.num_pages, st.q_indptr, st.kv_len_before, st.page_indptr, st.page_indices, kv8=True)
        q_out, out, turned, k_turned = (torch.zeros((total, h, 64), dtype=torch.bfloat16, device="cuda") for h in (8, 8, 8, 2))
        lse = torch.zeros((total, 8), device="cuda")
        kb, vb = (torch.zeros((sum(n), 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        B.asynclm_kv8_append(plan, k, v, pool, scales, table, q, q_out)
        B.asynclm_kv8_attn_mixed(plan, q_out, pool, scales, out, lse)
        B.asynclm_kv8_gather(plan, indptr, first, pool, scales, kb, vb)
        B.asynclm_rope_apply(table, positions, q, turned, k, k_turned)
        torch.cuda.synchronize()
        assert B.last_device_status(plan) == 0
        return [bits(x) for x in (pool, scales, q_out, out, lse, kb, vb, turned, k_turned)]

    fast = everything()
    monkeypatch.setattr(B, "_calls", lambda: False)
    assert everything() == fast


def test_arguments_that_the_extension_leaves_to_ctypes_are_refused_there():
    """No GPU: tensors on the CPU, absent plans."""
    t = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    table = B.asynclm_rope_table(64)
    with pytest.raises((ValueError, B.AsynclmError)):
        B.asynclm_rope_apply(table, torch.zeros(4, dtype=torch.int32), t, t.clone(), k=t)
    pool, scales = torch.zeros((2, 2, 2, 16, 64), dtype=torch.uint8), torch.zeros((2, 2, 2, 16), dtype=torch.uint8)
    plan = types.SimpleNamespace(handle=None)
    for call in (lambda: B.asynclm_kv8_append(plan, t, t, pool, scales), lambda: B.asynclm_kv8_attn_mixed(plan, t, pool, scales, t),
                 lambda: B.asynclm_kv8_attn_mixed(plan, t, pool.float(), scales, t)):
        with pytest.raises((ValueError, B.AsynclmError)):
            call()


PROBE = """
#include "span_ring.h"
using namespace asynclm::tc;
extern "C" int slots_of(int which, int head_dim) { return ring_slots_kv8(which, head_dim); }
extern "C" int scales_of(int head_dim) { return scale_slots(ring_slots_kv8(0, head_dim)); }
"""


@pytest.fixture(scope="module")
def ring(tmp_path_factory):
    d = tmp_path_factory.mktemp("ring8")
    src, lib = os.path.join(d, "probe.cpp"), os.path.join(d, "probe.so")
    with open(src, "w") as f:
        f.write(PROBE)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", lib_build.CSRC, "-o", lib, src], check=True)
    return ctypes.CDLL(lib)


@pytest.mark.parametrize("head_dim", [128, 64])
def test_no_wait_on_the_8_bit_rings_can_pass_a_phase_early(ring, head_dim):
    """The model of the span body's hand-offs with this cache's rings, which differ in length.  (Here a K tile is released by both groups' warps,
    which is an order more, not one less.)"""
    slots = [ring.slots_of(which, head_dim) for which in (0, 1)]
    place = lambda which, t, first, tiles, dual: ((which, t % slots[which]), t // slots[which])      # noqa: E731
    for items in three_items():
        assert not ambiguous_waits(items, place), items
    assert not ambiguous_waits([(1, False)] * 30 + [(9, True), (2, False), (40, True)], place)


def reads_of_scales(items, slots):
    """For every tile t, the tiles whose scales a warp may still read when the producer writes t's: a group reads from its release of a tile to
    its release of the next one of its own (or its item's end, behind which nothing of that item is read)."""
    owner, first = [], 0      # of every tile: (item, groups)
    for i, (n, dual) in enumerate(items):
        owner += [(i, (0, 1) if dual else (j & 1,)) for j in range(n)]
        first += n
    for t in range(slots, first):
        live = set()
        for b in (0, 1):
            mine = [x for x in range(t - slots + 1) if b in owner[x][1]]      # released for certain
            if not mine:
                continue
            # both groups end an item together, so a tile of an item that ended before that of tile t - slots is through
            if owner[mine[-1]][0] == owner[t - slots][0]:
                live.add(mine[-1])
            later = [x for x in range(t - slots + 1, t) if b in owner[x][1]]
            live.update(later)
        yield t, live


@pytest.mark.parametrize("head_dim", [128, 64])
def test_scales_are_not_overwritten_while_they_are_read(ring, head_dim):
    slots, scales = ring.slots_of(0, head_dim), ring.scales_of(head_dim)
    for items in three_items():
        for t, live in reads_of_scales(items, slots):
            assert all(x % scales != t % scales for x in live), (items, t)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_the_example_holds_its_bound(dim):
    spec = importlib.util.spec_from_file_location("quantised_cache", os.path.join(ROOT, "examples", "quantised_cache.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    got = m.run(layers=2, sequences=5, prompt=300, steps=5, dim=dim)
    assert got["error_of_bound"] <= 1 and got["tokens"] > 5 * 5
