"""Measured cases of the quantised paged cache: rotary positions, the quantising append, the read-back and the attention over it.

The cache.  A row is the head_dim values of one (token, kv head, K or V).  It is held as e4m3 codes and one scale 2^e: e is the smallest
integer, at least -100, with max|x| <= 448 * 2^e, a code is x * 2^-e rounded to nearest even, and stands for code * 2^e.  A row with a value that is
not finite has the scale NaN and codes 0.
    pool    float8_e4m3fn  [num_pages][2 (K, V)][kv_heads][16 slots][head_dim]
    scales  float8_e8m0fnu [num_pages][kv_heads][2 (K, V)][16 slots]

Rotary positions turn pair j of a head's first `rotary` values by position * f_j radians; pairs are (j, j + rotary / 2) ("half") or
(2j, 2j + 1) ("interleaved").

With `own` false, run() is the plain form in elementary torch operations; with `own` true it is the calls that a user of the package makes.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
CODE_MAX = 448.0
LEAST_EXPONENT = -100
CONTEXT = 8192          # positions a model was trained for, where its positions are scaled
THETA = 500000.0


# ---------------------------------------------------------------------------------------------------------------- cases

def _attn(name, heads, seqs, ctx, spans=0, span=(1, 1), lens=1):
    return {"name": name, "op": "attn", "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "seqs": seqs, "ctx_lo": ctx[0],
            "ctx_hi": ctx[1], "spans": spans, "span_lo": span[0], "span_hi": span[1], "lens": lens}


def _rows(name, op, heads, seqs, ctx, spans, span, rotary, layout, scaling, fused, lens=1):
    return {**_attn(name, heads, seqs, ctx, spans, span, lens), "op": op, "rotary": rotary, "layout": layout, "scaling": scaling, "fused": fused}


def listed():
    wide, narrow = (32, 8, 128), (8, 2, 64)
    return [
        # four sequences that decode beside nothing else: the smallest step that a server makes, all latency
        _attn("attn 4 decode", wide, 4, (500, 4000)),
        # a batch of decoding sequences: the ordinary step
        _attn("attn 64 decode", wide, 64, (1000, 3000), lens=2),
        # many short sequences of a small model
        _attn("attn 201 decode, 8/2 of 64", narrow, 201, (17, 1500), lens=3),
        # a few sequences with very long contexts, cut over their length and joined
        _attn("attn 5 decode, long", wide, 5, (32000, 110000), lens=4),
        # decoding sequences, some of which get an interrupt: spans beside single tokens
        _attn("attn 32, 8 with spans", wide, 32, (512, 4096), 8, (8, 64), lens=5),
        # a context that is computed anew, or a long prompt: all of it at once, bound by the products
        _attn("attn 7777 prompt", wide, 1, (0, 0), 1, (7777, 7777), lens=6),
        # the append of a decode step: rows out of the fused projection's output, keys and queries rotated, angles scaled by bands
        _rows("append 5 decode", "append", wide, 5, (300, 20000), 0, (1, 1), 128, "half", "bands", True, lens=7),
        # the append of a long prompt, interleaved pairs of half of the head, scaled for four times the context
        _rows("append 8192 prompt", "append", wide, 2, (0, 3000), 2, (4096, 4096), 64, "interleaved", "yarn", True, lens=8),
        # rotary positions alone, for a cache that stays in 16 bits: a decode step, and a long prompt of odd length
        _rows("rope 3 decode", "rope", wide, 3, (100, 9000), 0, (1, 1), 128, "half", "none", False, lens=9),
        _rows("rope 4097 prompt", "rope", wide, 1, (0, 0), 1, (4097, 4097), 128, "half", "linear", True, lens=10),
        # one sequence's cache read back, and a batch's, as for a hand-over to another server
        _attn("gather 1 of 700, 8/2 of 64", narrow, 1, (700, 700), lens=11) | {"op": "gather"},
        _attn("gather 64", wide, 64, (1000, 3000), lens=12) | {"op": "gather"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice([(32, 8, 128), (8, 2, 64), (16, 16, 64), (8, 1, 128), (16, 8, 128), (32, 8, 64)])
    op = rng.choice(["attn", "attn", "attn", "append", "rope", "gather"])
    lens = rng.randrange(1, 1 << 30)
    if op == "attn":
        kind = rng.choice(["decode", "mixed", "prompt"])
        if kind == "prompt":
            span = _log(rng, 2, 6000)
            ctx = rng.choice([0, _log(rng, 1, 2000)])
            return {k: v for k, v in _attn("", heads, 1, (ctx, ctx), 1, (span, span), lens).items() if k != "name"}
        seqs = _log(rng, 1, 256)
        hi = _log(rng, 16, min(110000, 350000 // seqs))
        lo = rng.randint(1, hi)
        spans, span = 0, (1, 1)
        if kind == "mixed":
            spans = rng.randint(1, seqs)
            most = max(2, min(300, 600_000_000 // (seqs * heads[0] * (hi + 300))))      # the plain form's scores stay within a few GB
            span_hi = _log(rng, 2, most)
            span = (rng.randint(1, span_hi), span_hi)
        return {k: v for k, v in _attn("", heads, seqs, (lo, hi), spans, span, lens).items() if k != "name"}
    if op == "gather":
        seqs = _log(rng, 1, 128)
        hi = _log(rng, 1, 120000 // seqs)
        return {k: v for k, v in (_attn("", heads, seqs, (rng.randint(1, hi), hi), lens=lens) | {"op": "gather"}).items() if k != "name"}
    spans = rng.choice([0, 1])
    seqs = _log(rng, 1, 256) if not spans else _log(rng, 1, 16)
    span_hi = _log(rng, 2, 8192 // seqs) if spans else 1
    rotary = rng.choice([heads[2], heads[2] // 2, heads[2] // 4, 24])
    if op == "append" and rng.random() < 0.25:
        rotary = 0
    return {k: v for k, v in _rows("", op, heads, seqs, (0, _log(rng, 10, 30000)), seqs if spans else 0, (rng.randint(1, span_hi), span_hi), rotary,
                                   rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "bands", "yarn"]),
                                   rng.random() < 0.5, lens).items() if k != "name"}


# ---------------------------------------------------------------------------------------------------------------- inputs

def _lengths(case):
    """Context and new tokens of each sequence, pages of each, and the physical page of each logical one."""
    r = np.random.RandomState(case["lens"] % (1 << 31))
    n = case["seqs"]
    ctx = r.randint(case["ctx_lo"], case["ctx_hi"] + 1, n)
    new = np.ones(n, np.int64) if case["op"] != "gather" else np.zeros(n, np.int64)
    at = r.permutation(n)[:case["spans"]]
    new[at] = r.randint(case["span_lo"], case["span_hi"] + 1, len(at))
    pages = -(-(ctx + new) // PAGE)
    pages_indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    ids = r.permutation(int(pages_indptr[-1]) + 3)[:int(pages_indptr[-1])].astype(np.int32)
    first = np.minimum(r.randint(0, 40, n), ctx // 2)      # where a read-back starts
    return ctx, new, pages_indptr, ids, first


def frequencies(case):
    """Radians a position of each pair, and the factor on the rotated values."""
    rd, f, m = case["rotary"], THETA ** (-np.arange(0, case["rotary"], 2, dtype=np.float64) / case["rotary"]), 1.0
    if case["scaling"] == "linear":
        f = f / 8.0
    elif case["scaling"] == "bands":
        wave = 2 * np.pi / f
        mix = np.clip((CONTEXT / wave - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = (1 - mix) * f / 8.0 + mix * f
    elif case["scaling"] == "yarn":
        pair = lambda turns: rd * math.log(CONTEXT / (2 * math.pi * turns)) / (2 * math.log(THETA))  # noqa: E731
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rd - 1)
        ramp = np.clip((np.arange(rd // 2) - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        f = f / 4.0 * ramp + f * (1 - ramp)
        m = 0.1 * math.log(4.0) + 1.0
    return f, m


def _two_to(e):
    """2^e in fp32 for whole e in -126 .. 127, by its bits."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes of rows of fp32 values, and the scales' bytes (e + 127, or 255), by the definition at the top."""
    most = x.abs().amax(-1, keepdim=True)
    _, e = torch.frexp(most / CODE_MAX)              # most / 448 = m * 2^e, 1/2 <= m < 1
    fine = torch.isfinite(most)
    e = torch.where(fine & (most > 0), e, LEAST_EXPONENT + 1).clamp(min=LEAST_EXPONENT + 1)
    e = torch.where(most <= CODE_MAX * _two_to(e - 1), e - 1, e)
    codes = torch.where(fine, x * _two_to(-e), 0.0).to(torch.float8_e4m3fn)
    byte = torch.where(fine, e + 127, 255).to(torch.uint8)
    return codes, byte.squeeze(-1)


def _cuda(a, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype).cuda()


def prepare(case, seed):
    ctx, new, pages_indptr, ids, first = _lengths(case)
    hq, hkv, d, n = case["q_heads"], case["kv_heads"], case["dim"], case["seqs"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    num_pages = int(pages_indptr[-1]) + 3
    total = int(new.sum())
    q_indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    seq = np.repeat(np.arange(n), new)
    pos = np.arange(total) - q_indptr[seq] + ctx[seq]
    s = {"case": case, "ctx": _cuda(ctx, torch.int64), "new": _cuda(new, torch.int64), "positions": _cuda(pos, torch.int32)}

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    loud = 1.0 + 4.0 * (torch.rand(d, generator=g, device="cuda") < 0.04)      # a few channels of keys are larger than the rest
    if case["op"] != "rope":
        s["pool"] = torch.empty((num_pages, 2, hkv, PAGE, d), dtype=torch.float8_e4m3fn, device="cuda")
        s["scales"] = torch.empty((num_pages, hkv, 2, PAGE), dtype=torch.float8_e8m0fnu, device="cuda")
        for p in range(0, num_pages, 4096):      # the cache as earlier steps left it
            x = normal(min(4096, num_pages - p), 2, hkv, PAGE, d)
            x[:, 0] *= loud
            codes, byte = _quantise(x)
            s["pool"][p:p + 4096] = codes
            s["scales"][p:p + 4096].view(torch.uint8).copy_(byte.transpose(1, 2))
    if case["op"] in ("append", "rope"):
        # rows of the projections: of one fused product's output, or of three
        if case["fused"]:
            qkv = normal(total, hq + 2 * hkv, d)
            qkv[:, hq:hq + hkv] *= loud
            qkv = qkv.bfloat16()
            s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        else:
            s["q"], s["k"], s["v"] = normal(total, hq, d).bfloat16(), (normal(total, hkv, d) * loud).bfloat16(), normal(total, hkv, d).bfloat16()
        s["q_out"] = torch.empty((total, hq, d), dtype=torch.bfloat16, device="cuda")
        s["k_out"] = torch.empty((total, hkv, d), dtype=torch.bfloat16, device="cuda")
        if case["rotary"]:
            f, s["factor"] = frequencies(case)
            s["f"] = _cuda(f)
        s["row_page"] = _cuda(ids[pages_indptr[seq] + pos // PAGE], torch.int64)
        s["row_slot"] = _cuda(pos % PAGE, torch.int64)
    if case["op"] == "attn":
        s["q"] = normal(total, hq, d).bfloat16()
        s["out"] = torch.empty((total, hq, d), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty((total, hq), device="cuda")
        most = int(np.diff(pages_indptr).max())
        logical = np.minimum(np.arange(most)[None], np.diff(pages_indptr)[:, None] - 1) + pages_indptr[:-1, None]
        s["table"] = _cuda(ids[logical], torch.int64)                                  # [seqs][pages], the last page again behind the end
        s["rows"] = _cuda(np.minimum(q_indptr[:-1, None] + np.arange(new.max())[None], total - 1), torch.int64)
        s["seq"], s["in_seq"] = _cuda(seq, torch.int64), _cuda(pos - ctx[seq], torch.int64)
    if case["op"] == "gather":
        length = ctx - first
        s["out_indptr"] = _cuda(np.concatenate([[0], np.cumsum(length)]), torch.int64)
        s["first"] = _cuda(first, torch.int32)
        which = np.repeat(np.arange(n), length)
        at = np.arange(int(length.sum())) - (np.cumsum(length) - length)[which] + first[which]
        s["row_page"], s["row_slot"] = _cuda(ids[pages_indptr[which] + at // PAGE], torch.int64), _cuda(at % PAGE, torch.int64)
        s["k_out"] = torch.empty((len(at), hkv, d), dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    if own:      # the handles that a program keeps: the step's plan (one for all layers) and the table of angles
        from paper_2412_07017_b200 import binding
        from paper_2412_07017_b200.workload import Shape
        s["binding"] = binding
        if case["op"] != "rope":
            s["plan"] = binding.asynclm_plan(Shape(hq, hkv, d, PAGE), num_pages, q_indptr, ctx.astype(np.int32), pages_indptr, ids,
                                             kv8=True)
        s["turn"] = None
        if case.get("rotary"):
            more = {"none": {}, "linear": {"factor": 8.0}, "bands": {"factor": 8.0, "low_freq_factor": 1.0, "high_freq_factor": 4.0, "context": CONTEXT},
                    "yarn": {"factor": 4.0, "beta_fast": 32.0, "beta_slow": 1.0, "context": CONTEXT}}[case["scaling"]]
            s["turn"] = binding.asynclm_rope_table(d, theta=THETA, rotary_dim=case["rotary"], layout=case["layout"], scaling=case["scaling"], **more)
    return s


# ---------------------------------------------------------------------------------------------------------------- one pass

def _rotated(s, x):
    """Rows x [tokens][heads][dim] turned by their positions, in 32 bits (the angle, which passes 10^5 radians, in 64)."""
    x = x.float()
    if not s["case"]["rotary"]:
        return x
    rd = s["case"]["rotary"]
    a = s["positions"].double()[:, None] * s["f"]
    c, n = (torch.cos(a).float() * s["factor"])[:, None], (torch.sin(a).float() * s["factor"])[:, None]
    if s["case"]["layout"] == "half":
        u, v = x[..., :rd // 2], x[..., rd // 2:rd]
        turned = torch.cat([u * c - v * n, v * c + u * n], -1)
    else:
        u, v = x[..., 0:rd:2], x[..., 1:rd:2]
        turned = torch.stack([u * c - v * n, v * c + u * n], -1).flatten(-2)
    return torch.cat([turned, x[..., rd:]], -1)


def _plain_append(s):
    for which, rows in ((0, _rotated(s, s["k"])), (1, s["v"].float())):
        codes, byte = _quantise(rows)
        s["pool"].view(torch.uint8)[s["row_page"], which, :, s["row_slot"]] = codes.view(torch.uint8)
        s["scales"].view(torch.uint8)[s["row_page"], :, which, s["row_slot"]] = byte
    out = {"pool": s["pool"], "scales": s["scales"]}
    if s["case"]["rotary"]:
        out["q"] = _rotated(s, s["q"]).bfloat16()
    return out


def _plain_rope(s):
    return {"q": _rotated(s, s["q"]).bfloat16(), "k": _rotated(s, s["k"]).bfloat16()}


def _plain_gather(s):
    def rows(which):
        codes = s["pool"].view(torch.uint8)[s["row_page"], which, :, s["row_slot"]].view(torch.float8_e4m3fn).float()
        scale = s["scales"].view(torch.uint8)[s["row_page"], :, which, s["row_slot"]].view(torch.float8_e8m0fnu).float()
        return (codes * scale[..., None]).bfloat16()
    return {"k": rows(0), "v": rows(1)}


def _plain_attn(s):
    case = s["case"]
    hq, hkv, d, n = case["q_heads"], case["kv_heads"], case["dim"], case["seqs"]

    def cached(which):      # [seqs][kv heads][keys][dim]
        codes = s["pool"].view(torch.uint8)[:, which][s["table"]].view(torch.float8_e4m3fn).float()
        scale = s["scales"].view(torch.uint8)[:, :, which][s["table"]].view(torch.float8_e8m0fnu).float()
        return (codes * scale[..., None]).transpose(1, 2).reshape(n, hkv, -1, d)
    k = cached(0)
    q = s["q"][s["rows"]].float().reshape(n, -1, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).flatten(2, 3)      # [seqs][kv heads][tokens x heads][dim]
    score = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).unflatten(2, (-1, hq // hkv))
    del k
    sees = s["ctx"][:, None] + torch.arange(s["rows"].shape[1], device="cuda") + 1                         # keys that a token sees
    hidden = torch.arange(score.shape[-1], device="cuda") >= sees[..., None]
    score.masked_fill_(hidden[:, None, :, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    p = score.sub_(most).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), cached(1)).unflatten(2, (-1, hq // hkv)) / total
    lse = (most + total.log()).squeeze(-1)
    out = out.permute(0, 2, 1, 3, 4).reshape(n, -1, hq, d)[s["seq"], s["in_seq"]]
    return {"out": out.bfloat16(), "lse": lse.permute(0, 2, 1, 3).reshape(n, -1, hq)[s["seq"], s["in_seq"]]}


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"append": _plain_append, "rope": _plain_rope, "gather": _plain_gather, "attn": _plain_attn}[op](s)
    b = s["binding"]
    if op == "append":
        if s["turn"] is None:
            b.asynclm_kv8_append(s["plan"], s["k"], s["v"], s["pool"], s["scales"])
            return {"pool": s["pool"], "scales": s["scales"]}
        b.asynclm_kv8_append(s["plan"], s["k"], s["v"], s["pool"], s["scales"], s["turn"], s["q"], s["q_out"])
        return {"pool": s["pool"], "scales": s["scales"], "q": s["q_out"]}
    if op == "rope":
        b.asynclm_rope_apply(s["turn"], s["positions"], s["q"], s["q_out"], s["k"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "gather":
        b.asynclm_kv8_gather(s["plan"], s["out_indptr"], s["first"], s["pool"], s["scales"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    b.asynclm_kv8_attn_mixed(s["plan"], s["q"], s["pool"], s["scales"], s["out"], s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------------------------------------------------------- what a pass needs, and its result

def work(case):
    ctx, new, _, _, first = _lengths(case)
    hq, hkv, d, total = case["q_heads"], case["kv_heads"], case["dim"], int(new.sum())
    if case["op"] == "attn":
        pairs = float((new * ctx + new * (new + 1) // 2).sum())
        return {"bytes": float((ctx + new).sum()) * hkv * 2 * (d + 1) + total * hq * (4 * d + 4), "flops": 4.0 * d * hq * pairs}
    if case["op"] == "gather":
        return {"bytes": float((ctx - first).sum()) * hkv * 2 * (d + 1 + 2 * d), "flops": 0.0}
    turned = 3.0 * case["rotary"]
    if case["op"] == "rope":
        return {"bytes": 4.0 * total * (hq + hkv) * d, "flops": turned * total * (hq + hkv)}
    q_bytes = 4.0 * total * hq * d if case["rotary"] else 0.0
    return {"bytes": total * hkv * 2.0 * (2 * d + d + 1) + q_bytes, "flops": turned * total * (hq + hkv) + 4.0 * total * hkv * d}


def _exact_turned(case, pos, x):
    x = x.double()
    rd = case["rotary"]
    if not rd:
        return x
    f, m = frequencies(case)
    a = pos.double()[:, None, None] * _cuda(f)
    e = torch.polar(torch.full_like(a, m), a)
    y = x.clone()
    first, second = (slice(0, rd // 2), slice(rd // 2, rd)) if case["layout"] == "half" else (slice(0, rd, 2), slice(1, rd, 2))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * e
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rows(x):
    """(values of the codes, scales) of rows in 64 bits, from the definition: the exponent by counting, the code by its step."""
    most = x.abs().amax(-1, keepdim=True)
    scale = torch.full_like(most, 2.0 ** LEAST_EXPONENT)
    for k in range(LEAST_EXPONENT, 121):
        scale = torch.where(most > CODE_MAX * 2.0 ** k, 2.0 ** (k + 1), scale)
    y = x / scale
    power = torch.tensor([2.0 ** k for k in range(-9, 10)], dtype=torch.float64, device="cuda")
    step = power[(torch.frexp(y)[1] - 4).clamp(min=-9).long() + 9]      # three bits behind the leading one; below 2^-6 the least step, 2^-9
    return torch.round(y / step) * step, scale.squeeze(-1)


def exact(case, seed):
    """What run() returns, in 64 bits: the outputs' definitions, a sequence or a tensor at a time."""
    ctx, new, pages_indptr, ids, first = _lengths(case)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    if case["op"] == "rope":
        return {"q": _exact_turned(case, s["positions"], s["q"]), "k": _exact_turned(case, s["positions"], s["k"])}
    pool, scales = s["pool"].double(), s["scales"].double()
    if case["op"] == "append":
        at, slot = s["row_page"], s["row_slot"]
        for which, rows in ((0, _exact_turned(case, s["positions"], s["k"])), (1, s["v"].double())):
            values, scale = _exact_rows(rows)
            pool[at, which, :, slot] = values
            scales[at, :, which, slot] = scale
        out = {"pool": pool, "scales": scales}
        if case["rotary"]:
            out["q"] = _exact_turned(case, s["positions"], s["q"])
        return out
    del pool, scales

    def sequence(b, which, upto):      # [tokens][kv heads][dim]
        pages = _cuda(ids[pages_indptr[b]:pages_indptr[b + 1]], torch.int64)
        codes = s["pool"].view(torch.uint8)[pages, which].view(torch.float8_e4m3fn).double()      # [pages][heads][16][dim]
        scale = s["scales"].view(torch.uint8)[pages, :, which].view(torch.float8_e8m0fnu).double()
        return (codes * scale[..., None]).permute(0, 2, 1, 3).reshape(-1, hkv, d)[:upto]
    if case["op"] == "gather":
        return {name: torch.cat([sequence(b, which, int(ctx[b]))[int(first[b]):] for b in range(case["seqs"])]) for name, which in (("k", 0), ("v", 1))}
    out, lse, row = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda"), 0
    for b in range(case["seqs"]):
        k, v = sequence(b, 0, int(ctx[b] + new[b])), sequence(b, 1, int(ctx[b] + new[b]))
        for t0 in range(0, int(new[b]), 512):
            t1 = min(t0 + 512, int(new[b]))
            upto = int(ctx[b]) + t1
            q = s["q"][row + t0:row + t1].double().reshape(t1 - t0, hkv, hq // hkv, d)
            a = torch.einsum("thgd,khd->htgk", q, k[:upto]) / math.sqrt(d)
            visible = torch.arange(upto, device="cuda")[None] <= int(ctx[b]) + torch.arange(t0, t1, device="cuda")[:, None]
            a = torch.where(visible[None, :, None], a, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
            z = torch.logsumexp(a, -1)
            o = torch.einsum("htgk,khd->thgd", torch.exp(a - z[..., None]), v[:upto])
            out[row + t0:row + t1] = o.reshape(t1 - t0, hq, d)
            lse[row + t0:row + t1] = z.permute(1, 0, 2).reshape(t1 - t0, hq)
        row += int(new[b])
    return {"out": out, "lse": lse}
