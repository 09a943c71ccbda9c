"""Paged caches for the GPU tests of shared prefixes and selected pages, and their attention in 64 bits."""
import numpy as np
import torch

from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200.workload import Shape

PAGE = 16
# A weight is rounded to bf16 (f16 for the 8-bit cache, fewer) and so is the output, half a step each, relative to A = sum p |V|; sums are fp32.
OUT_TOL = 2.1 * 2.0 ** -8
LSE_TOL = 4e-4


class Cache:
    """A pool with the pages of `ctx + new` tokens a sequence; the slots behind them and the spare pages hold NaN (8 bits: the largest code)."""

    def __init__(self, heads, ctx, new, groups=(), kv8=False, seed=0, spare=5, loud=1.0):
        r = np.random.RandomState(seed)
        self.hq, self.hkv, self.d = heads
        self.shape, self.kv8 = Shape(*heads, PAGE), kv8
        self.ctx, self.new = np.asarray(ctx, np.int32), np.asarray(new, np.int32)
        pages = -(-(self.ctx + self.new) // PAGE)
        self.indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
        self.num_pages = int(self.indptr[-1]) + spare
        self.ids = r.permutation(self.num_pages)[:int(self.indptr[-1])].astype(np.int32)
        for first, n, tokens in groups:
            for b in range(first + 1, first + n):
                self.ids[self.indptr[b]:self.indptr[b] + tokens // PAGE] = self.ids[self.indptr[first]:self.indptr[first] + tokens // PAGE]
        self.q_indptr = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1)
        self.total = int(self.new.sum())
        x = torch.randn((self.num_pages, 2, self.hkv, PAGE, self.d), generator=g, device="cuda")
        x[:, 0] = (0.6 * x[:, 0] + 0.8 * torch.randn((self.num_pages, self.hkv, 1, self.d), generator=g, device="cuda")) * loud
        self.q = torch.randn((self.total, self.hq, self.d), generator=g, device="cuda").bfloat16()
        used = torch.zeros((self.num_pages, PAGE), dtype=torch.bool)
        for b in range(len(self.ctx)):
            for j in range(int(pages[b])):
                used[self.ids[self.indptr[b] + j], :min(PAGE, int(self.ctx[b] + self.new[b]) - j * PAGE)] = True
        self.used = used.cuda()
        if kv8:
            e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448.0))
            self.pool = (x * torch.exp2(-e)).to(torch.float8_e4m3fn)
            self.pool.view(torch.uint8).masked_fill_(~self.used[:, None, None, :, None], 0x7e)
            byte = (e.squeeze(-1) + 127).to(torch.uint8).transpose(1, 2).contiguous()
            self.scales = byte.masked_fill_(~self.used[:, None, None], 254).view(torch.float8_e8m0fnu)
        else:
            self.pool = x.bfloat16().masked_fill_(~self.used[:, None, None, :, None], float("nan"))

    @property
    def args(self):
        return self.shape, self.num_pages, self.q_indptr, self.ctx, self.indptr, self.ids

    def values(self, b, which):
        """[kv heads][tokens][dim] of sequence b, in 64 bits."""
        pages = torch.as_tensor(self.ids[self.indptr[b]:self.indptr[b + 1]].astype(np.int64)).cuda()
        if self.kv8:
            x = self.pool.view(torch.uint8)[pages, which].view(torch.float8_e4m3fn).double()
            x = x * self.scales.view(torch.uint8)[pages, :, which].view(torch.float8_e8m0fnu).double()[..., None]
        else:
            x = self.pool[pages, which].double()
        return x.transpose(0, 1).flatten(1, 2)[:, :int(self.ctx[b] + self.new[b])]

    def exact(self, chosen=None):
        """(out, lse, A) of every row; chosen[row, kv head, keys]: the keys that it attends to, of those it sees."""
        out = torch.zeros((self.total, self.hq, self.d), dtype=torch.float64, device="cuda")
        lse, a_sum = torch.zeros((self.total, self.hq), dtype=torch.float64, device="cuda"), torch.zeros_like(out)
        row = 0
        for b in range(len(self.ctx)):
            k, v = self.values(b, 0), self.values(b, 1)
            for t in range(int(self.new[b])):
                n = int(self.ctx[b]) + t + 1
                s = torch.matmul(self.q[row].double().reshape(self.hkv, -1, self.d), k[:, :n].transpose(1, 2)) / self.d ** 0.5
                if chosen is not None:
                    s = s.masked_fill(~chosen[row][:, None, :n], -float("inf"))
                z = torch.logsumexp(s, -1)
                p = torch.exp(s - z[..., None])
                out[row] = torch.matmul(p, v[:, :n]).reshape(self.hq, self.d)
                a_sum[row] = torch.matmul(p, v[:, :n].abs()).reshape(self.hq, self.d)
                lse[row] = z.flatten()
                row += 1
        return out, lse, a_sum

    def attend(self, plan, out=None, lse=None, call=None):
        out = torch.full((self.total, self.hq, self.d), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
        lse = torch.full((self.total, self.hq), float("nan"), device="cuda") if lse is None else lse
        if call is not None:
            call(plan, self.q, self.pool, out, lse)
        elif self.kv8:
            B.asynclm_kv8_attn_mixed(plan, self.q, self.pool, self.scales, out, lse)
        else:
            B.asynclm_attn_mixed(plan, self.q, self.pool, out, lse)
        return out, lse

    def bounds(self):
        """[pages][kv heads][2][dim] of the used slots, in 64 bits; NaN for pages without any."""
        k = self.pool[:, 0].double()
        if self.kv8:
            k = k * self.scales.view(torch.uint8)[:, :, 0].view(torch.float8_e8m0fnu).double()[..., None]
        unused = ~self.used[:, None, :, None]
        b = torch.stack([k.masked_fill(unused, float("inf")).amin(-2), k.masked_fill(unused, -float("inf")).amax(-2)], -2)
        b[~self.used.any(-1)] = float("nan")
        return b


def check(got, want, what=""):
    out, lse = got
    ref, ref_lse, a_sum = want
    assert torch.isfinite(out).all() and torch.isfinite(lse).all(), what
    assert ((out.double() - ref).abs() <= OUT_TOL * a_sum + 1e-30).all(), f"{what}: {((out.double() - ref).abs() / a_sum).max() * 256} steps"
    assert (lse.double() - ref_lse).abs().max() <= LSE_TOL, what
