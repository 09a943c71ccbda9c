#!/usr/bin/env python
"""Serving steps with drafted tokens: all sequences begin with the same function descriptions, every step proposes a few tokens for each, and the target
accepts some of them.

Per step one plan and, for the one layer of this toy model, `asynclm_kv_append` of the last token and the drafts, `asynclm_kv_bounds` of their pages, the attention
and, on its outputs' probabilities, `asynclm_draft_verify`; a sequence then grows by what was accepted.  The first half of the steps reads the shared
descriptions once for all sequences (`asynclm_plan_prefix`), the second half attends to the pages that `asynclm_select_pages` chooses
(`asynclm_plan_sparse`).  Every step is held against the definitions in 64 bits.

    python examples/drafted_steps.py [--sequences 6] [--described 700] [--steps 8] [--drafts 4] [--budget 24] [--dim 128]

Prints one JSON line; the model is random."""
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


class Model:
    """A token's query, key and value rows are its own; the next token's logits are a projection of what attention gives."""

    def __init__(self, vocab, heads, dim, gen):
        def rows(n):
            return torch.randn((vocab, n, dim), device="cuda", generator=gen).bfloat16()
        self.q, self.k, self.v = rows(heads[0]), rows(heads[1]), rows(heads[1])
        self.project = torch.randn((heads[0] * dim, vocab), device="cuda", generator=gen) * 0.2
        self.bigrams = torch.randn((vocab, vocab), device="cuda", generator=gen)      # what the target and the cheap model share

    def target(self, tokens, out):
        return torch.softmax(2.0 * self.bigrams[tokens] + out.float().flatten(1) @ self.project, -1)

    def draft(self, token):
        return torch.softmax(2.0 * self.bigrams[token], -1)


def verified(indptr, target, draft, tokens, u, v):
    """The rule, a sequence at a time, on the host: tokens that are emitted."""
    out = []
    for b in range(len(indptr) - 1):
        i0, i1, a = indptr[b], indptr[b + 1], 0
        while i0 + a < i1 and u[i0 + a] * draft[i0 + a, tokens[i0 + a]] < target[i0 + a + b, tokens[i0 + a]]:
            a += 1
        w = target[i0 + a + b] if i0 + a == i1 else np.maximum(target[i0 + a + b] - draft[i0 + a], 0.0)
        sums = np.cumsum(w)
        out.append(list(tokens[i0:i0 + a]) + [int(np.argmax(sums > v[b] * sums[-1]))])
    return out


def run(sequences=6, described=700, steps=8, drafts=4, budget=24, dim=128, heads=(32, 8), vocab=500, seed=0) -> dict:
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    shape, model = W.Shape(heads[0], heads[1], dim, PAGE), Model(vocab, heads, dim, gen)
    shared = described // PAGE                                    # pages of the descriptions
    per_seq = -(-(described % PAGE + 40 + (steps + 1) * (drafts + 1)) // PAGE)
    num_pages = shared + sequences * per_seq
    ids = rng.permutation(num_pages).astype(np.int32)
    pages = [np.concatenate([ids[:shared], ids[shared + b * per_seq:shared + (b + 1) * per_seq]]) for b in range(sequences)]
    page_indptr, page_indices = np.arange(sequences + 1, dtype=np.int32) * (shared + per_seq), np.concatenate(pages)
    pool = torch.zeros((num_pages, 2, heads[1], PAGE, dim), dtype=torch.bfloat16, device="cuda")
    bounds = torch.zeros((num_pages, heads[1], 2, dim), dtype=torch.bfloat16, device="cuda")
    workspace = torch.zeros(B.draft_verify_workspace_bytes(sequences, vocab), dtype=torch.uint8, device="cuda")

    def plan_args(ctx, new):
        return shape, num_pages, np.concatenate([[0], np.cumsum(new)]).astype(np.int32), np.asarray(ctx, np.int32), page_indptr, page_indices

    # the descriptions, written once through the first sequence, then each sequence's own beginning
    text = [list(rng.integers(0, vocab, shared * PAGE))] * sequences
    text = [t + list(rng.integers(0, vocab, int(rng.integers(1, 40)))) for t in text]
    ctx = np.zeros(sequences, np.int32)
    for new in (np.array([shared * PAGE] + [0] * (sequences - 1)), np.array([len(t) - 1 - shared * PAGE for t in text])):
        plan = B.asynclm_plan(*plan_args(ctx, new))
        rows = torch.tensor([t for b in range(sequences) for t in text[b][ctx[b]:ctx[b] + new[b]]], device="cuda")
        if len(rows):
            B.asynclm_kv_append(plan, model.k[rows], model.v[rows], pool)
            B.asynclm_kv_bounds(plan, pool, bounds, from_start=True)
        ctx = ctx + new
        if new[0] == shared * PAGE:
            ctx[:] = shared * PAGE
    worst, accepted_all, emitted = 0.0, 0, 0
    for step in range(steps):
        count = rng.integers(0, drafts + 1, sequences)
        # the cheap model's proposals
        token = torch.tensor([t[-1] for t in text], device="cuda")
        fed, proposals, q_rows = [token], [], []
        for _ in range(drafts):
            q_rows.append(model.draft(token))
            token = torch.multinomial(q_rows[-1], 1, generator=gen)[:, 0]
            proposals.append(token)
            fed.append(token)
        at = [(b, i) for b in range(sequences) for i in range(count[b])]
        draft = torch.stack([q_rows[i][b] for b, i in at]) if at else torch.zeros((0, vocab), device="cuda")
        tokens = torch.tensor([int(proposals[i][b]) for b, i in at], dtype=torch.int32, device="cuda")
        new = count + 1
        rows = torch.tensor([int(fed[i][b]) for b in range(sequences) for i in range(new[b])], device="cuda")
        # the step
        selects = step >= steps // 2
        plan = B.asynclm_plan_sparse(*plan_args(ctx, new), budget, 1, 2) if selects else B.asynclm_plan_prefix(
            *plan_args(ctx, new), [(0, sequences, shared * PAGE)], flags=B.PLAN_SHARE_ALL)
        q, total = model.q[rows], len(rows)
        out = torch.empty_like(q)
        B.asynclm_kv_append(plan, model.k[rows], model.v[rows], pool)
        B.asynclm_kv_bounds(plan, pool, bounds)
        chosen = torch.empty((total, heads[1], budget), dtype=torch.int32, device="cuda")
        if selects:
            B.asynclm_select_pages(plan, q, bounds, chosen)
        B.asynclm_attn_mixed(plan, q, pool, out)
        target = model.target(rows, out)
        u, v = torch.rand(len(at), device="cuda", generator=gen), torch.rand(sequences, device="cuda", generator=gen)
        indptr = torch.tensor(np.concatenate([[0], np.cumsum(count)]), dtype=torch.int32, device="cuda")
        accepted = torch.empty(sequences, dtype=torch.int32, device="cuda")
        tokens_out = torch.empty(len(at) + sequences, dtype=torch.int32, device="cuda")
        B.asynclm_draft_verify(indptr, target, draft, tokens, u, v, accepted, tokens_out, workspace)
        if B.last_device_status(plan) != 0:
            raise RuntimeError("a step reported a device status")
        # held against the definitions
        row = 0
        for b in range(sequences):
            n = int(ctx[b] + new[b])
            where = torch.from_numpy(pages[b][:-(-n // PAGE)].astype(np.int64)).cuda()
            k, val = (pool[where, w].double().transpose(0, 1).flatten(1, 2)[:, :n] for w in (0, 1))
            for i in range(new[b]):
                sees = int(ctx[b]) + i + 1
                s = torch.matmul(q[row].double().reshape(heads[1], -1, dim), k[:, :sees].transpose(1, 2)) / dim ** 0.5
                if selects:
                    on = torch.zeros((heads[1], -(-sees // PAGE) + 1), dtype=torch.bool, device="cuda")
                    on.scatter_(1, torch.where(chosen[row] >= 0, chosen[row], on.shape[1] - 1).long(), True)
                    on[:, -1] = False
                    s = s.masked_fill(~on.repeat_interleave(PAGE, 1)[:, None, :sees], -float("inf"))
                p = torch.softmax(s, -1)
                want, a_sum = torch.matmul(p, val[:, :sees]).reshape(heads[0], dim), torch.matmul(p, val[:, :sees].abs()).reshape(heads[0], dim)
                worst = max(worst, float(((out[row].double() - want).abs() / (2.1 * 2.0 ** -8 * a_sum)).max()))
                row += 1
        host = [x.cpu().double().numpy() for x in (target, draft, u, v)]
        want = verified(indptr.cpu().numpy(), host[0], host[1], tokens.cpu().numpy(), host[2], host[3])
        for b in range(sequences):
            first = int(indptr[b]) + b
            got = tokens_out[first:first + int(accepted[b]) + 1].tolist()
            if got != want[b]:
                raise RuntimeError(f"step {step}, sequence {b}: {got} emitted, the rule gives {want[b]}")
            text[b] = text[b] + got
            ctx[b] += len(got)
            accepted_all += len(got) - 1
            emitted += len(got)
        if any(len(t) != ctx[b] + 1 for b, t in enumerate(text)):
            raise RuntimeError("the cache and the text have come apart")
    return {"what": "steps with drafted tokens behind shared descriptions", "sequences": sequences, "described": shared * PAGE, "steps": steps, "emitted": emitted,
            "accepted": accepted_all, "error_of_bound": worst}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("sequences", 6), ("described", 700), ("steps", 8), ("drafts", 4), ("budget", 24), ("dim", 128)):
        ap.add_argument("--" + name, type=int, default=value)
    got = run(**vars(ap.parse_args()))
    print(json.dumps(got))
    sys.exit(0 if got["error_of_bound"] <= 1 else 1)
