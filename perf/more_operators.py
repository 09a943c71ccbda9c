"""Measured cases of a decoding step with long and shared contexts: attention of sequences that begin with the same pages, attention over
the pages that a score selects, and verification of drafted tokens.

Shared prefix.  The sequences of a group have their first `prefix` tokens in the same pages.  Every new token attends to its whole sequence.

Selected pages.  key_bounds [num_pages][kv_heads][2 (least, largest)][head_dim] holds, for each page and channel, the least and largest value of the
keys in the page's used slots.  A page's score for a token and a kv head is
    max over the head's queries q of sum_c max(q_c * least_c, q_c * largest_c),
which no score of a key in the page exceeds.  Of the pages that hold the keys a token sees, the first `first_pages` and the last `last_pages` are taken, and
those of the others with the largest scores (the lowest page among equals), until there are `budget`.  The token attends to the keys in them.

Drafted tokens.  Draft i of a sequence, token x drawn from the distribution q_i, is accepted if u_i q_i(x) < p_i(x) and all before it are; p_i is the
target's distribution there.  Behind the accepted ones goes one token more: of the distribution max(p - q, 0) at the first rejected draft, or of the
target's behind the last draft.  It is the least t with sum_{t' <= t} w_t' > u * sum w.

Caches are those of bf16, pool [num_pages][2 (K, V)][kv_heads][16 slots][head_dim], or of 8 bits: e4m3 codes in that layout, a value is
code * 2^e, and e8m0 scales [num_pages][kv_heads][2 (K, V)][16 slots].

With `own` false, run() is the plain form in elementary torch operations; with `own` true it is the calls that a user of the package makes.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
INF = math.inf


# ---------------------------------------------------------------------------------------------------------------- cases

def _prefix(name, heads, groups, seqs, prefix, own_ctx, new=(1, 1), alone=0, spans=0, span=(1, 1), kv8=False, lens=1):
    return {"name": name, "op": "prefix", "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "groups": groups, "seqs": seqs, "prefix_lo": prefix[0],
            "prefix_hi": prefix[1], "own_lo": own_ctx[0], "own_hi": own_ctx[1], "new_lo": new[0], "new_hi": new[1], "alone": alone, "spans": spans,
            "span_lo": span[0], "span_hi": span[1], "kv8": kv8, "lens": lens}


def _sparse(name, heads, seqs, ctx, budget, first, last, new=(1, 1), kv8=False, lens=1, op="sparse"):
    return {"name": name, "op": op, "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "seqs": seqs, "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "budget": budget, "first_pages": first, "last_pages": last, "new_lo": new[0], "new_hi": new[1], "kv8": kv8, "lens": lens}


def _verify(name, seqs, vocab, drafts, apart, dtype, with_draft=True, lens=1):
    return {"name": name, "op": "verify", "seqs": seqs, "vocab": vocab, "drafts_lo": drafts[0], "drafts_hi": drafts[1], "apart": apart, "dtype": dtype,
            "with_draft": with_draft, "lens": lens}


def listed():
    wide, narrow = (32, 8, 128), (8, 2, 64)
    return [
        # four conversations that have just begun behind the same function descriptions: the smallest step, all latency
        _prefix("prefix 4 decode", wide, 1, 4, (2048, 2048), (20, 300)),
        # the ordinary batch: long descriptions for all, conversations of their own behind them
        _prefix("prefix 64 decode", wide, 1, 64, (4096, 4096), (100, 1500), lens=2),
        # two models' descriptions, some sequences without any, and interrupts: spans beside single tokens
        _prefix("prefix 40 in 2 groups, 8 with spans", wide, 2, 40, (1500, 6000), (64, 1000), alone=8, spans=8, span=(8, 64), lens=3),
        # drafted tokens of a large batch behind a very long document, 8-bit cache
        _prefix("prefix 96 drafts, 8 bits", wide, 1, 96, (16000, 24000), (17, 600), new=(1, 6), kv8=True, lens=4),
        # four long conversations: few rows, many pages
        _sparse("sparse 4 decode", wide, 4, (16000, 60000), 128, 1, 4, lens=5),
        # a batch of long contexts with drafted tokens
        _sparse("sparse 48 drafts", wide, 48, (3000, 12000), 64, 1, 4, new=(1, 4), lens=6),
        # the same of a small model, 8-bit cache, single tokens; some contexts fit the budget
        _sparse("sparse 150 decode, 8/2 of 64, 8 bits", narrow, 150, (300, 9000), 96, 2, 8, kv8=True, lens=7),
        # bounds of a cache that is there already: one short sequence, and a batch's
        _sparse("bounds 1 of 900, 8/2 of 64", narrow, 1, (900, 900), 8, 1, 1, lens=8, op="bounds"),
        _sparse("bounds 64", wide, 64, (1000, 4000), 64, 1, 4, lens=9, op="bounds"),
        # two sequences' drafts from a small vocabulary
        _verify("verify 2 x 4", 2, 32001, (4, 4), 0.7, "fp32", lens=10),
        # an ordinary batch
        _verify("verify 64 x 5", 64, 128256, (5, 5), 0.8, "fp32", lens=11),
        # many sequences, numbers of drafts that differ, none among them, proposed without a distribution (looked up in the text), bf16
        _verify("verify 300 looked up", 300, 100003, (0, 8), 0.5, "bf16", with_draft=False, lens=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice([(32, 8, 128), (8, 2, 64), (16, 16, 64), (8, 1, 128), (16, 8, 128), (32, 8, 64)])
    op = rng.choice(["prefix", "prefix", "sparse", "sparse", "verify", "bounds"])
    lens = rng.randrange(1, 1 << 30)
    kv8 = rng.random() < 0.35
    if op == "verify":
        vocab = _log(rng, 1000, 160000)
        seqs = _log(rng, 1, max(1, min(300, 38_000_000 // vocab)))
        hi = rng.randint(0, 8)
        case = _verify("", seqs, vocab, (rng.randint(0, hi), hi), rng.uniform(0.1, 1.5), rng.choice(["fp32", "bf16"]), rng.random() < 0.7, lens)
    elif op == "prefix":
        groups = rng.choice([1, 1, 2, 3])
        seqs = _log(rng, groups, 96)
        prefix_hi = _log(rng, 16, 24000)
        prefix = (rng.randint(16, prefix_hi), prefix_hi)
        own_hi = _log(rng, 1, max(1, min(4000, 90000 // seqs)))
        spans = rng.choice([0, 0, rng.randint(0, seqs // 4)])
        new_hi = rng.choice([1, 1, 5])
        rows = 250_000_000 // (prefix_hi * heads[0]) - seqs * new_hi      # the plain form's scores stay within a few GB
        span_hi = _log(rng, 2, max(2, min(200, rows // max(spans, 1))))
        case = _prefix("", heads, groups, seqs, prefix, (rng.randint(0, own_hi), own_hi), (1, new_hi), rng.choice([0, seqs // 5]), spans,
                       (rng.randint(1, span_hi), span_hi), kv8, lens)
    else:
        seqs = _log(rng, 1, 150)
        hi = _log(rng, 16, max(16, min(60000, 360000 // seqs)))
        budget = _log(rng, 4, 256)
        first = rng.randint(0, min(3, budget // 2))
        case = _sparse("", heads, seqs, (rng.randint(1, hi), hi), budget, first, rng.randint(1, max(1, min(8, budget - first))), (1, rng.choice([1, 1, 4])), kv8,
                       lens, op)
    return {k: v for k, v in case.items() if k != "name"}


# ---------------------------------------------------------------------------------------------------------------- inputs

def _lengths(case):
    """Tokens of each sequence in the cache (ctx) and new ones, the groups (first sequence, sequences, tokens), and the page table."""
    r = np.random.RandomState(case["lens"] % (1 << 31))
    n = case["seqs"]
    new = r.randint(case["new_lo"], case["new_hi"] + 1, n)
    if case["op"] != "prefix":
        ctx, groups = r.randint(case["ctx_lo"], case["ctx_hi"] + 1, n), []
    else:
        at = r.permutation(n)[:case["spans"]]
        new[at] = r.randint(case["span_lo"], case["span_hi"] + 1, len(at))
        grouped = n - case["alone"]
        edges = np.linspace(0, grouped, case["groups"] + 1).astype(int)
        groups = [(int(a), int(b - a), int(r.randint(case["prefix_lo"], case["prefix_hi"] + 1)) // PAGE * PAGE) for a, b in zip(edges[:-1], edges[1:]) if b > a]
        ctx = r.randint(case["own_lo"], case["own_hi"] + 1, n)
        for first, count, tokens in groups:
            ctx[first:first + count] += tokens
    pages = -(-(ctx + new) // PAGE)
    indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    fresh = np.ones(int(indptr[-1]), bool)           # entries that have a page of their own
    source = np.arange(int(indptr[-1]))              # of the others, the entry whose page they have
    for first, count, tokens in groups:
        for b in range(first + 1, first + count):
            fresh[indptr[b]:indptr[b] + tokens // PAGE] = False
            source[indptr[b]:indptr[b] + tokens // PAGE] = indptr[first] + np.arange(tokens // PAGE)
    num_pages = int(fresh.sum()) + 3
    ids = np.zeros(int(indptr[-1]), np.int32)
    ids[fresh] = r.permutation(num_pages)[:int(fresh.sum())]
    return ctx, new, groups, indptr, ids[source].astype(np.int32), num_pages


def _cuda(a, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype).cuda()


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _codes(x):
    """Rows of fp32 values in 8 bits: codes, and the bytes e + 127 of their scales, e the least integer with max|x| <= 448 * 2^e."""
    most = x.abs().amax(-1, keepdim=True).clamp(min=1e-20)
    e = torch.ceil(torch.log2(most.double() / 448.0))
    return (x.double() * torch.exp2(-e)).float().to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).squeeze(-1)


def _values(s, pages, which):
    """The cached K (0) or V (1) of pages, [..., kv_heads][16][head_dim] in fp32."""
    if not s["case"]["kv8"]:
        return s["pool"][:, which][pages].float()
    codes = s["pool"].view(torch.uint8)[:, which][pages].view(torch.float8_e4m3fn).float()
    return codes * s["scales"].view(torch.uint8)[:, :, which][pages].view(torch.float8_e8m0fnu).float()[..., None]


def _prepare_verify(case, seed):
    r = np.random.RandomState(case["lens"] % (1 << 31))
    n, vocab = case["seqs"], case["vocab"]
    drafts = r.randint(case["drafts_lo"], case["drafts_hi"] + 1, n)
    indptr = np.concatenate([[0], np.cumsum(drafts)]).astype(np.int32)
    total = int(indptr[-1])
    dtype = {"fp32": torch.float32, "bf16": torch.bfloat16}[case["dtype"]]
    g = _generator(seed)
    s = {"case": case, "indptr": _cuda(indptr), "drafts": drafts}
    target = torch.empty((total + n, vocab), dtype=dtype, device="cuda")
    draft = torch.empty((total, vocab), dtype=dtype, device="cuda") if case["with_draft"] else None
    tokens = torch.empty(total, dtype=torch.int32, device="cuda")
    for b in range(n):      # the draft model's logits are the target's with noise
        i0, k = int(indptr[b]), int(drafts[b])
        logits = 3.0 * torch.randn((k + 1, vocab), generator=g, device="cuda")
        target[i0 + b:i0 + b + k + 1] = torch.softmax(logits, -1)
        if k == 0:
            continue
        q = torch.softmax(logits[:k] + case["apart"] * torch.randn((k, vocab), generator=g, device="cuda"), -1)
        if draft is not None:
            draft[i0:i0 + k] = q
            race = q / torch.empty_like(q).exponential_(generator=g)      # the largest is a draw from q
        else:                                                             # a guess that is often the likeliest token
            race = q
        tokens[i0:i0 + k] = race.argmax(-1).int()
    s["target"], s["draft"], s["tokens"] = target, draft, tokens
    s["accept_u"] = torch.rand(total, generator=g, device="cuda")
    s["sample_u"] = torch.rand(n, generator=g, device="cuda")
    s["accepted"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["tokens_out"] = torch.empty(total + n, dtype=torch.int32, device="cuda")
    if own:
        from paper_2412_07017_b200 import binding
        s["binding"] = binding
        s["workspace"] = torch.zeros(binding.draft_verify_workspace_bytes(n, vocab), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    if case["op"] == "verify":
        return _prepare_verify(case, seed)
    ctx, new, groups, indptr, ids, num_pages = _lengths(case)
    hq, hkv, d, n = case["q_heads"], case["kv_heads"], case["dim"], case["seqs"]
    g = _generator(seed)
    total = int(new.sum())
    q_indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    seq = np.repeat(np.arange(n), new)
    pos = np.arange(total) - q_indptr[seq] + ctx[seq]
    s = {"case": case, "groups": groups, "q_indptr": q_indptr, "ctx": _cuda(ctx, torch.int64), "indptr": indptr, "ids": ids}
    s["pool"] = torch.empty((num_pages, 2, hkv, PAGE, d), dtype=torch.float8_e4m3fn if case["kv8"] else torch.bfloat16, device="cuda")
    if case["kv8"]:
        s["scales"] = torch.empty((num_pages, hkv, 2, PAGE), dtype=torch.float8_e8m0fnu, device="cuda")
    s["bounds"] = torch.empty((num_pages, hkv, 2, d), dtype=torch.bfloat16, device="cuda")
    loud = 1.0 + 3.0 * (torch.rand(d, generator=g, device="cuda") < 0.04)      # a few channels of keys are larger than the rest
    for p in range(0, num_pages, 4096):      # the cache as earlier steps left it; the keys of a page resemble one another
        m = min(4096, num_pages - p)
        x = torch.randn((m, 2, hkv, PAGE, d), generator=g, device="cuda")
        x[:, 0] = (0.6 * x[:, 0] + 0.8 * torch.randn((m, hkv, 1, d), generator=g, device="cuda")) * loud
        if case["kv8"]:
            codes, byte = _codes(x)
            s["pool"][p:p + m] = codes
            s["scales"][p:p + m].view(torch.uint8).copy_(byte.transpose(1, 2))
        else:
            s["pool"][p:p + m] = x
        k = _values(s, slice(p, p + m), 0)
        s["bounds"][p:p + m] = torch.stack([k.amin(-2), k.amax(-2)], -2)
    s["q"] = torch.randn((total, hq, d), generator=g, device="cuda").bfloat16()
    s["out"] = torch.empty((total, hq, d), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.empty((total, hq), device="cuda")
    s["pos"], s["seq"], s["in_seq"] = _cuda(pos, torch.int64), _cuda(seq, torch.int64), _cuda(pos - ctx[seq], torch.int64)
    s["rows"] = _cuda(np.minimum(q_indptr[:-1, None] + np.arange(new.max())[None], total - 1), torch.int64)
    most = int(np.diff(indptr).max())
    logical = np.minimum(np.arange(most)[None], np.diff(indptr)[:, None] - 1) + indptr[:-1, None]
    s["table"] = _cuda(ids[logical], torch.int64)                                  # [seqs][pages], the last page again behind the end
    s["chosen"] = torch.empty((total, hkv, case.get("budget", 0)), dtype=torch.int32, device="cuda")
    if case["op"] == "prefix":
        shared = np.zeros(n, np.int64)
        for first, count, tokens in groups:
            shared[first:first + count] = tokens
        s["shared"] = _cuda(shared)
        lengths = np.diff(indptr) - shared // PAGE      # pages of their own
        at = np.minimum(np.arange(int(lengths.max()))[None], lengths[:, None] - 1) + (indptr[:-1] + shared // PAGE)[:, None]
        s["own_table"] = _cuda(ids[at], torch.int64)
        s["prefix_pages"] = [_cuda(ids[indptr[first]:indptr[first] + tokens // PAGE], torch.int64) for first, _, tokens in groups]
    else:
        # the pages whose bounds a call brings up to date, and their slots in use: those of the new tokens, or all
        first = np.zeros(n, np.int64) if case["op"] == "bounds" else ctx // PAGE
        last = (ctx + new - 1) // PAGE
        which = np.repeat(np.arange(n), last - first + 1)
        page = np.concatenate([np.arange(a, b + 1) for a, b in zip(first, last)])
        s["bound_pages"], s["bound_used"] = _cuda(ids[indptr[which] + page], torch.int64), _cuda(np.minimum((ctx + new)[which] - page * PAGE, PAGE), torch.int64)
    if own:      # the handles that a program keeps: the step's plan (one for all layers)
        from paper_2412_07017_b200 import binding
        from paper_2412_07017_b200.workload import Shape
        s["binding"] = binding
        args = (Shape(hq, hkv, d, PAGE), num_pages, q_indptr, ctx.astype(np.int32), indptr, ids)
        if case["op"] == "prefix":
            s["plan"] = binding.asynclm_plan_prefix(*args, groups, kv8=case["kv8"])
        elif case["op"] == "sparse":
            s["plan"] = binding.asynclm_plan_sparse(*args, budget_pages=case["budget"], first_pages=case["first_pages"], last_pages=case["last_pages"],
                                                    kv8=case["kv8"])
        else:
            s["plan"] = binding.asynclm_plan(*args, kv8=case["kv8"])
    return s


# ---------------------------------------------------------------------------------------------------------------- one pass, in plain operations

def _plain_prefix(s):
    case = s["case"]
    hq, hkv, d, n = case["q_heads"], case["kv_heads"], case["dim"], case["seqs"]
    gq, scale = hq // hkv, 1.0 / math.sqrt(d)
    q = s["q"].float().unflatten(1, (hkv, gq))                                     # [rows][kv heads][heads][dim]
    total = q.shape[0]
    # each sequence's own keys
    k = _values(s, s["own_table"], 0).transpose(1, 2).reshape(n, hkv, -1, d)
    score = torch.einsum("ntkgd,nkcd->nktgc", q[s["rows"]], k).mul_(scale)
    del k
    sees = (s["ctx"] - s["shared"])[:, None] + torch.arange(s["rows"].shape[1], device="cuda") + 1
    hidden = torch.arange(score.shape[-1], device="cuda") >= sees[..., None]
    score.masked_fill_(hidden[:, None, :, None], -INF)
    most = score.amax(-1, keepdim=True)
    p = score.sub_(most).exp_()
    v = _values(s, s["own_table"], 1).transpose(1, 2).reshape(n, hkv, -1, d)
    o = torch.einsum("nktgc,nkcd->nktgd", p, v)
    del v

    def rows(x):      # [seqs][kv heads][tokens].. -> [rows][kv heads]..
        return x.transpose(1, 2)[s["seq"], s["in_seq"]]
    out, weight, most = rows(o), rows(p.sum(-1, keepdim=True)), rows(most)
    # the shared ones, joined to them
    for (first, count, tokens), pages in zip(s["groups"], s["prefix_pages"]):
        r0, r1 = int(s["q_indptr"][first]), int(s["q_indptr"][first + count])
        if tokens == 0:
            continue
        k, v = (_values(s, pages, which).transpose(0, 1).reshape(hkv, -1, d) for which in (0, 1))
        a = torch.einsum("tkgd,kcd->tkgc", q[r0:r1], k).mul_(scale)
        m = torch.maximum(a.amax(-1, keepdim=True), most[r0:r1])
        a = a.sub_(m).exp_()
        old = (most[r0:r1] - m).exp()
        out[r0:r1] = out[r0:r1] * old + torch.einsum("tkgc,kcd->tkgd", a, v)
        weight[r0:r1] = weight[r0:r1] * old + a.sum(-1, keepdim=True)
        most[r0:r1] = m
    return {"out": (out / weight).reshape(total, hq, d).bfloat16(), "lse": (most + weight.log()).reshape(total, hq)}


def _plain_bounds(s):
    k = _values(s, s["bound_pages"], 0)
    unused = (torch.arange(PAGE, device="cuda") >= s["bound_used"][:, None])[:, None, :, None]
    s["bounds"][s["bound_pages"]] = torch.stack([k.masked_fill(unused, INF).amin(-2), k.masked_fill(unused, -INF).amax(-2)], -2).bfloat16()
    return s["bounds"]


def _plain_select(s):
    """The chosen pages [rows][kv heads][budget], rising, -1 behind the last."""
    case = s["case"]
    hkv, gq, budget = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["budget"]
    score = torch.empty((s["q"].shape[0], hkv, s["table"].shape[1]), dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        r0, r1 = int(s["q_indptr"][b]), int(s["q_indptr"][b + 1])
        q = s["q"][r0:r1].double().unflatten(1, (hkv, gq))
        lo, hi = s["bounds"][s["table"][b]].double().unbind(2)                     # [pages][kv heads][dim]
        up = torch.einsum("tkgd,pkd->tkgp", q.clamp(min=0), hi) + torch.einsum("tkgd,pkd->tkgp", q.clamp(max=0), lo)
        score[r0:r1] = up.amax(2)
    pages = (s["pos"] // PAGE + 1)[:, None, None]                                  # that hold the keys a token sees
    at = torch.arange(score.shape[-1], device="cuda")
    always = (at < case["first_pages"]) | (at >= pages - case["last_pages"])
    score.masked_fill_(always, INF).masked_fill_(at >= pages, -INF)
    k = min(budget, score.shape[-1])
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :k]
    order = torch.where(torch.arange(k, device="cuda") < pages, order, 1 << 30).sort(-1)[0]
    chosen = torch.full((*score.shape[:2], budget), -1, dtype=torch.int32, device="cuda")
    chosen[..., :k] = torch.where(order < (1 << 30), order, -1).int()
    return chosen


def _plain_sparse(s):
    case = s["case"]
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    gq = hq // hkv
    _plain_bounds(s)
    chosen = _plain_select(s)
    out, lse = [], []
    for r0 in range(0, chosen.shape[0], 64):
        at = chosen[r0:r0 + 64].long()                                             # [rows][kv heads][budget]
        physical = s["table"][s["seq"][r0:r0 + 64, None, None], at.clamp(min=0)]
        heads = torch.arange(hkv, device="cuda")[None, :, None]

        def cached(which):
            if not case["kv8"]:
                x = s["pool"][physical, which, heads].float()
            else:
                x = s["pool"].view(torch.uint8)[physical, which, heads].view(torch.float8_e4m3fn).float()
                x = x * s["scales"].view(torch.uint8)[physical, heads, which].view(torch.float8_e8m0fnu).float()[..., None]
            return x.flatten(2, 3)                                                 # [rows][kv heads][keys][dim]
        q = s["q"][r0:r0 + 64].float().unflatten(1, (hkv, gq))
        a = torch.matmul(q, cached(0).transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
        key = (at[..., None] * PAGE + torch.arange(PAGE, device="cuda")).flatten(2)
        hidden = (key > s["pos"][r0:r0 + 64, None, None]) | (at < 0).repeat_interleave(PAGE, -1)
        a.masked_fill_(hidden[:, :, None], -INF)
        most = a.amax(-1, keepdim=True)
        a = a.sub_(most).exp_()
        weight = a.sum(-1, keepdim=True)
        out.append((torch.matmul(a, cached(1)) / weight).flatten(1, 2).bfloat16())
        lse.append((most + weight.log()).flatten(1))
    return {"bounds": s["bounds"], "pages": chosen, "out": torch.cat(out), "lse": torch.cat(lse)}


def _plain_verify(s):
    drafts = (s["indptr"][1:] - s["indptr"][:-1]).long()
    n, total, vocab = drafts.shape[0], s["tokens"].shape[0], s["target"].shape[1]
    b = torch.arange(n, device="cuda")
    seq = torch.repeat_interleave(b, drafts, output_size=total)
    i = torch.arange(total, device="cuda")
    x = s["tokens"].long()
    p = s["target"][i + seq, x].double()
    q = torch.ones_like(p) if s["draft"] is None else s["draft"][i, x].double()
    bad = ~(s["accept_u"].double() * q < p)
    place = i - s["indptr"][:-1].long()[seq]
    accepted = torch.scatter_reduce(drafts.clone(), 0, seq, torch.where(bad, place, vocab + total), "amin")
    row = s["indptr"][:-1].long() + accepted
    weight = s["target"][row + b].double()
    rejected = accepted < drafts
    at = row.clamp(max=max(total - 1, 0))
    if total:
        if s["draft"] is None:
            weight[b[rejected], x[at[rejected]]] = 0.0
        else:
            weight = torch.where(rejected[:, None], (weight - s["draft"][at].double()).clamp(min=0), weight)
    sums = weight.cumsum(-1)
    token = (sums > s["sample_u"].double()[:, None] * sums[:, -1:]).int().argmax(-1)
    out = torch.full((total + n,), -1, dtype=torch.int32, device="cuda")
    out[i + seq] = torch.where(place < accepted[seq], s["tokens"], -1)
    out[row + b] = token.int()
    return {"accepted": accepted.int(), "tokens": out}


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "bounds":
            return {"bounds": _plain_bounds(s)}
        return {"prefix": _plain_prefix, "sparse": _plain_sparse, "verify": _plain_verify}[op](s)
    b, kv8 = s["binding"], s["case"].get("kv8")
    if op == "verify":
        b.asynclm_draft_verify(s["indptr"], s["target"], s["draft"], s["tokens"], s["accept_u"], s["sample_u"], s["accepted"], s["tokens_out"], s["workspace"])
        return {"accepted": s["accepted"], "tokens": s["tokens_out"]}
    if op != "prefix":
        if kv8:
            b.asynclm_kv8_bounds(s["plan"], s["pool"], s["scales"], s["bounds"], from_start=op == "bounds")
        else:
            b.asynclm_kv_bounds(s["plan"], s["pool"], s["bounds"], from_start=op == "bounds")
        if op == "bounds":
            return {"bounds": s["bounds"]}
        b.asynclm_select_pages(s["plan"], s["q"], s["bounds"], s["chosen"])
    if kv8:
        b.asynclm_kv8_attn_mixed(s["plan"], s["q"], s["pool"], s["scales"], s["out"], s["lse"])
    else:
        b.asynclm_attn_mixed(s["plan"], s["q"], s["pool"], s["out"], s["lse"])
    if op == "prefix":
        return {"out": s["out"], "lse": s["lse"]}
    return {"bounds": s["bounds"], "pages": s["chosen"], "out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------------------------------------------------------- what a pass needs, and its result

def work(case):
    if case["op"] == "verify":
        r = np.random.RandomState(case["lens"] % (1 << 31))
        drafts = r.randint(case["drafts_lo"], case["drafts_hi"] + 1, case["seqs"])
        size = {"fp32": 4, "bf16": 2}[case["dtype"]]
        rows = float(case["seqs"])                   # one of the target's for every sequence; one of the draft's where a token was rejected
        if case["with_draft"]:
            accept = math.erfc(case["apart"] / (2 * math.sqrt(2)))      # of one token: log p/q is about normal
            rows += float((1 - accept ** drafts).sum())
        return {"bytes": rows * case["vocab"] * size + float(drafts.sum()) * (12 + 2 * size) + 12.0 * case["seqs"], "flops": 2.0 * rows * case["vocab"]}
    ctx, new, groups, _, _, _ = _lengths(case)
    hq, hkv, d, total = case["q_heads"], case["kv_heads"], case["dim"], int(new.sum())
    row = hkv * (d + 1) if case["kv8"] else hkv * 2 * d              # bytes of a token's keys
    rows = total * hq * (4 * d + 4)                                  # queries, outputs, log-sum-exps
    if case["op"] == "prefix":
        keys = float((ctx + new).sum() - sum((count - 1) * tokens for _, count, tokens in groups))
        pairs = float((new * ctx + new * (new + 1) // 2).sum())
        return {"bytes": keys * 2 * row + rows, "flops": 4.0 * d * hq * pairs}
    if case["op"] == "bounds":
        return {"bytes": float((ctx + new).sum()) * row + float((-(-(ctx + new) // PAGE)).sum()) * hkv * 4 * d, "flops": 2.0 * hkv * d * float((ctx + new).sum())}
    seq = np.repeat(np.arange(case["seqs"]), new)
    pos = np.arange(total) - (np.cumsum(new) - new)[seq] + ctx[seq]
    pages = pos // PAGE + 1
    keys = float(((np.minimum(pages, case["budget"]) - 1) * PAGE + pos % PAGE + 1).sum())
    scored = float(pages[pages > case["budget"]].sum())
    distinct = float(((ctx + new - 1) // PAGE + 1).sum())
    return {"bytes": keys * 2 * row + min(scored, distinct) * hkv * 4 * d + float(((ctx % PAGE) + new).sum()) * row + rows + total * hkv * case["budget"] * 4.0,
            "flops": 4.0 * d * hq * keys + 2.0 * d * hq * scored}


def _exact_verify(case, seed):
    s = _prepare_verify(case, seed)
    target, tokens, u, v = s["target"], s["tokens"].cpu().numpy(), s["accept_u"].double().cpu().numpy(), s["sample_u"].double().cpu().numpy()
    accepted, out, i0 = [], [], 0
    for b, k in enumerate(s["drafts"]):
        k, a = int(k), 0
        while a < k:
            x = int(tokens[i0 + a])
            qx = 1.0 if s["draft"] is None else float(s["draft"][i0 + a, x])
            if not u[i0 + a] * qx < float(target[i0 + b + a, x]):
                break
            a += 1
        w = target[i0 + b + a].double().cpu().numpy()
        if a < k and s["draft"] is None:
            w[tokens[i0 + a]] = 0.0
        elif a < k:
            w = np.maximum(w - s["draft"][i0 + a].double().cpu().numpy(), 0.0)
        sums = np.cumsum(w)
        token = int(np.searchsorted(sums, v[b] * sums[-1], side="right"))
        accepted.append(a)
        out += list(tokens[i0:i0 + a]) + [token] + [-1] * (k - a)
        i0 += k
    return {"accepted": _cuda(np.array(accepted), torch.int32), "tokens": _cuda(np.array(out), torch.int32)}


def exact(case, seed):
    """What run() returns, in 64 bits, from the definitions at the top, a token or a sequence at a time."""
    global own
    keep, own = own, False
    try:
        if case["op"] == "verify":
            return _exact_verify(case, seed)
        s = prepare(case, seed)
    finally:
        own = keep
    ctx, new, _, indptr, ids, _ = _lengths(case)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    gq = hq // hkv
    pool = s["pool"]

    def sequence(b, which):      # [kv heads][tokens][dim]
        pages = _cuda(ids[indptr[b]:indptr[b + 1]], torch.int64)
        if case["kv8"]:
            x = pool.view(torch.uint8)[pages, which].view(torch.float8_e4m3fn).double()
            x = x * s["scales"].view(torch.uint8)[pages, :, which].view(torch.float8_e8m0fnu).double()[..., None]
        else:
            x = pool[pages, which].double()
        return x.transpose(0, 1).flatten(1, 2)[:, :int(ctx[b] + new[b])]
    bounds = s["bounds"].double()
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    chosen = torch.full(s["chosen"].shape, -1, dtype=torch.int32, device="cuda")
    row = 0
    for b in range(case["seqs"]):
        k = sequence(b, 0)
        pages = _cuda(ids[indptr[b]:indptr[b + 1]], torch.int64)
        if case["op"] != "prefix":
            for j in range(0 if case["op"] == "bounds" else int(ctx[b]) // PAGE, (int(ctx[b] + new[b]) - 1) // PAGE + 1):
                x = k[:, j * PAGE:(j + 1) * PAGE]
                bounds[pages[j], :, 0], bounds[pages[j], :, 1] = x.min(1)[0], x.max(1)[0]
            if case["op"] == "bounds":
                continue
        v = sequence(b, 1)
        edges = bounds[pages] if case["op"] == "sparse" else None
        for t in range(int(new[b])):
            upto = int(ctx[b]) + t + 1
            q = s["q"][row].double().reshape(hkv, gq, d)
            a = torch.matmul(q, k[:, :upto].transpose(1, 2)) / math.sqrt(d)
            if edges is not None:
                n = (upto + PAGE - 1) // PAGE
                seen = torch.zeros((hkv, n), dtype=torch.bool, device="cuda")
                if n <= case["budget"]:
                    seen[:] = True
                else:
                    seen[:, :case["first_pages"]] = True
                    seen[:, n - case["last_pages"]:] = True
                    rest = case["budget"] - int(seen[0].sum())
                    lo, hi = edges[:n, :, 0].transpose(0, 1)[:, None], edges[:n, :, 1].transpose(0, 1)[:, None]      # [kv heads][1][pages][dim]
                    best = torch.maximum(q[:, :, None] * lo, q[:, :, None] * hi).sum(-1).amax(1)
                    best[seen] = -INF
                    if rest > 0:
                        least = best.sort(-1, descending=True)[0][:, rest - 1:rest]
                        take = best > least
                        tied = best == least
                        take |= tied & (tied.cumsum(-1) <= rest - take.sum(-1, keepdim=True))
                        seen |= take
                for h in range(hkv):
                    at = seen[h].nonzero().flatten()
                    chosen[row, h, :len(at)] = at.int()
                a.masked_fill_(~seen.repeat_interleave(PAGE, -1)[:, None, :upto], -INF)
            z = torch.logsumexp(a, -1)
            out[row] = torch.matmul(torch.exp(a - z[..., None]), v[:, :upto]).reshape(hq, d)
            lse[row] = z.reshape(hq)
            row += 1
    if case["op"] == "bounds":
        return {"bounds": bounds}
    if case["op"] == "sparse":
        return {"bounds": bounds, "pages": chosen, "out": out, "lse": lse}
    return {"out": out, "lse": lse}
