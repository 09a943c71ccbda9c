"""What the quantised cache's calls refuse before anything is launched: tensors that do not fit the plan, row strides that mean something else to the C
call, layouts that it cannot see.  No GPU: tensors are stand-ins, and a plan made on the host only, which the C call refuses, shows that the tensors
themselves were accepted."""
import types

import numpy as np
import pytest
import torch

from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200 import build as lib_build
from paper_2412_07017_b200 import workload as W

STREAM = types.SimpleNamespace(cuda_stream=0)
SHAPE, PAGES, TOKENS, BATCH = W.Shape(8, 2, 64, 16), 9, 5, 3
BF16, F32, U8, I32, I64 = torch.bfloat16, torch.float32, torch.uint8, torch.int32, torch.int64


class Fake:
    """A tensor on a GPU, as far as the binding looks at one."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, shape, dtype=BF16, strides=None):
        self.shape, self.dtype = tuple(shape), dtype
        dense = [int(np.prod(shape[k + 1:])) for k in range(len(shape))]
        self.strides = tuple(dense if strides is None else strides)
        self.whole = self.strides == tuple(dense)

    def dim(self):
        return len(self.shape)

    def stride(self, k=None):
        return self.strides if k is None else self.strides[k]

    def numel(self):
        return int(np.prod(self.shape))

    def is_contiguous(self):
        return self.whole

    def data_ptr(self):
        return 1 << 20


@pytest.fixture(params=["extension", "ctypes"])
def way(request, monkeypatch):
    if request.param == "ctypes":
        monkeypatch.setattr(B, "_calls", lambda: False)
    elif lib_build.build_call_ext() is None or not B._calls():
        pytest.skip("no C compiler or Python header here: the calls go through ctypes")


@pytest.fixture(scope="module")
def plan():
    return B.plan_host(SHAPE, PAGES, [0, 1, 4, 5], [20, 30, 0], [0, 2, 5, 6], [0, 1, 2, 3, 4, 5], kv8=True)


def accepted(call):
    """The tensors are: it is the C call that refuses the plan (or, of rows without one, a table that is none)."""
    with pytest.raises(B.AsynclmError) as e:
        call()
    assert e.value.status == -1


def refused(call, what):
    with pytest.raises(ValueError, match=what):
        call()


def rows(heads, n=TOKENS, d=64, **kw):
    return Fake((n, heads, d), **kw)


POOL, SCALES = Fake((PAGES, 2, 2, 16, 64), U8), Fake((PAGES, 2, 2, 16), U8)
FUSED = dict(strides=(12 * 64, 64, 1))


def test_append(way, plan):
    table = B.asynclm_rope_table(64)

    def call(k=rows(2), v=rows(2), pool=POOL, scales=SCALES, rope=table, q=rows(8), q_out=rows(8)):
        B.asynclm_kv8_append(plan, k, v, pool, scales, rope, q, q_out, stream=STREAM)
    accepted(call)
    accepted(lambda: call(k=rows(2, **FUSED), v=rows(2, **FUSED), q=rows(8, **FUSED)))
    for name in ("k", "v", "q"):
        match = name if name == "q" else name + "_new"
        heads = 8 if name == "q" else 2
        for bad in (rows(heads, TOKENS - 1), rows(heads, TOKENS + 1), rows(heads, 1), rows(heads - 1), rows(heads + 1), rows(heads, d=128), rows(heads, d=32),
                    rows(heads, strides=(0, 64, 1)), rows(heads, strides=(64, 64, 1)), rows(heads, strides=(heads * 64 - 8, 64, 1)),
                    rows(heads, strides=(-heads * 64, 64, 1)), rows(heads, strides=(heads * 64, 0, 1)), rows(heads, dtype=F32), Fake((TOKENS, heads * 64))):
            refused(lambda: call(**{name: bad} | ({"q_out": Fake(bad.shape)} if name == "q" else {})), match)      # noqa: B023
    refused(lambda: call(q_out=rows(8, TOKENS - 1)), "q_out")
    refused(lambda: call(q_out=rows(8, **FUSED)), "q_out")
    for bad in (Fake((PAGES - 1, 2, 2, 16, 64), U8), Fake((PAGES, 2, 2, 16, 32), U8)):
        refused(lambda: call(pool=bad), "kv8_pool")      # noqa: B023
    refused(lambda: call(scales=Fake((PAGES, 2, 1, 16), U8)), "kv8_scales")


def test_attention(way, plan):
    def call(q=rows(8), pool=POOL, scales=SCALES, out=rows(8), lse=Fake((TOKENS, 8), F32)):
        B.asynclm_kv8_attn_mixed(plan, q, pool, scales, out, lse, stream=STREAM)
    accepted(call)
    accepted(lambda: call(lse=None))
    for name in ("q", "out"):
        for bad in (rows(8, **FUSED), rows(8, strides=(0, 64, 1)), rows(8, TOKENS - 1), rows(8, TOKENS + 3), rows(2), rows(8, d=128), rows(8, dtype=F32),
                    rows(8, dtype=torch.float16)):
            refused(lambda: call(**{name: bad}), name)      # noqa: B023
    for bad in (Fake((TOKENS, 8), BF16), Fake((TOKENS, 7), F32), Fake((1, 8), F32), Fake((TOKENS, 8), F32, strides=(0, 1))):
        refused(lambda: call(lse=bad), "lse")      # noqa: B023
    refused(lambda: call(pool=Fake((PAGES, 1, 2, 16, 64), U8)), "kv8_pool")
    refused(lambda: call(scales=Fake((PAGES - 2, 2, 2, 16), U8)), "kv8_scales")


def test_read_back(way, plan):
    def call(out_indptr=Fake((BATCH + 1,), I64), first=Fake((BATCH,), I32), pool=POOL, scales=SCALES, k_out=rows(2, 40), v_out=rows(2, 40)):
        B.asynclm_kv8_gather(plan, out_indptr, first, pool, scales, k_out, v_out, stream=STREAM)
    accepted(call)
    refused(lambda: call(out_indptr=Fake((BATCH,), I64)), "out_indptr")
    refused(lambda: call(first=Fake((BATCH - 1,), I32)), "first")
    for bad in (rows(1, 40), rows(3, 40), rows(2, 40, 32), rows(2, 39), rows(2, 40, strides=(0, 64, 1)), rows(2, 40, **FUSED)):
        refused(lambda: call(k_out=bad), "k_out")      # noqa: B023
        refused(lambda: call(v_out=bad), "v_out")      # noqa: B023
        refused(lambda: call(k_out=bad, v_out=bad), "k_out") if bad.shape[0] == 40 else None      # noqa: B023
    refused(lambda: call(pool=Fake((PAGES, 2, 2, 16), U8)), "kv8_pool")


def test_rotary_rows(way):
    none = B.CRopeTable()      # (refused by the C call)

    def call(q=rows(8), q_out=rows(8), k=rows(2), k_out=rows(2), positions=Fake((TOKENS,), I32)):
        B.asynclm_rope_apply(none, positions, q, q_out, k, k_out, stream=STREAM)
    accepted(call)
    accepted(lambda: call(q=rows(8, **FUSED), q_out=rows(8, **FUSED), k=rows(2, **FUSED)))
    accepted(lambda: call(q=rows(8, 1, strides=(0, 64, 1)), q_out=rows(8, 1), k=None, k_out=None, positions=Fake((1,), I32)))      # (one row has no stride)
    for name, heads in (("q", 8), ("q_out", 8), ("k", 2), ("k_out", 2)):
        for strides in ((0, 64, 1), (64, 64, 1), (heads * 64 - 8, 64, 1), (-heads * 64, 64, 1)):
            refused(lambda: call(**{name: rows(heads, strides=strides)}), name)      # noqa: B023
