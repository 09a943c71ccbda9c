"""Verification of drafted tokens where the numbers are no probabilities, against the rule in 64 bits (GPU)."""
import numpy as np
import pytest
import torch

from test_draft_verify import Case

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]
# (vocabulary, distance of rows, values in front of the first): q's rows lie as p's do, or not
PLACES = [(1000, 1000, 0), (1003, 1003, 3), (70001, 70001, 1)]


def none_if_negative(x):
    return np.where(x < 0, 0.0, x)      # (NaN stays)


def rule(indptr, target, draft, tokens, u, v):
    """Negative probabilities count as none; NaN accepts nothing and weighs nothing."""
    accepted, out = [], []
    for b in range(len(indptr) - 1):
        i0, i1, a = indptr[b], indptr[b + 1], 0
        p_of = lambda k: none_if_negative(target[i0 + k + b])      # noqa: E731
        q_of = lambda k: none_if_negative(draft[i0 + k])      # noqa: E731
        while i0 + a < i1 and u[i0 + a] * q_of(a)[tokens[i0 + a]] < p_of(a)[tokens[i0 + a]]:
            a += 1
        p = np.nan_to_num(p_of(a), nan=0.0)
        w = np.nan_to_num(np.maximum(p_of(a) - q_of(a), 0.0), nan=0.0) if i0 + a < i1 else p
        token = -1
        for w in (w, p):
            if w.sum() > 0:
                over = np.cumsum(w) > v[b] * np.cumsum(w)[-1]
                token = int(over.argmax()) if over.any() else int(np.nonzero(w)[0][-1])
                break
        accepted.append(a)
        out += list(tokens[i0:i0 + a]) + [token] + [-1] * (i1 - i0 - a)
    return accepted, out


def check(c):
    c.call()
    host = [t.cpu().double().numpy() for t in (c.target, c.draft, c.u, c.v)]
    assert (c.accepted.cpu().tolist(), c.out.cpu().tolist()) == rule(c.indptr.cpu().numpy(), host[0], host[1], c.tokens.cpu().numpy(), host[2], host[3])


def put(rows, where, bits, dtype):
    """Sets places of rows to the number with these (fp32) bits."""
    if dtype == torch.float32:
        rows.view(torch.int32)[where] = int(np.uint32(bits).view(np.int32))
    else:
        rows.view(torch.int16)[where] = int(np.uint16(bits >> 16).view(np.int16))


def set_numbers(c, k):
    """Other random numbers for the samples, and a first draft that is rejected."""
    c.v.copy_(torch.linspace(0.01 + 0.02 * k, 0.93 + 0.02 * k, c.n))
    c.u.fill_(0.999)


@pytest.mark.parametrize("bits", [0x7fc00000, 0xffc00000, 0xffff0000], ids=["positive", "negative", "negative, all bits"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab,stride,offset", PLACES)
def test_nan_in_the_draft_weighs_nothing(vocab, stride, offset, dtype, bits):
    """A third of q is NaN, of either sign (0/0 is the negative one on x86): those tokens are not sampled."""
    c = Case([1] * 9, vocab, dtype, True, 1, stride, offset=offset)
    put(c.draft, (slice(None), slice(1, None, 3)), bits, dtype)
    x = c.tokens.long() // 3 * 3      # (a token whose q is a number)
    c.tokens.copy_(x)
    c.target[torch.arange(0, 18, 2, device="cuda"), x] = 0      # rejected
    for k in range(3):
        set_numbers(c, k)
        check(c)
        assert c.accepted.sum() == 0 and (c.out[0::2] % 3 != 1).all()


# p, q, u of a draft and whether it is accepted: u * q < p, negative probabilities being none
ACCEPTED = [(0.0, -0.25, 0.5, False), (-0.125, -0.5, 0.5, False), (-0.125, 0.25, 0.0, False), (0.0, 0.25, 0.0, False), (0.25, -0.5, 0.9, True), (0.25, -0.0, 0.9, True),
            (-0.0, -0.5, 0.25, False), (0.25, float("nan"), 0.0, False), (float("nan"), 0.25, 0.0, False), (0.25, -float("inf"), 0.5, True), (-float("inf"), 0.25, 0.5, False)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab,stride,offset", PLACES)
def test_negative_numbers_accept_nothing(vocab, stride, offset, dtype):
    n = len(ACCEPTED)
    c = Case([1] * n, vocab, dtype, True, 2, stride, offset=offset)
    for b, (p, q, u, _) in enumerate(ACCEPTED):
        c.target[2 * b, c.tokens[b].long()], c.draft[b, c.tokens[b].long()], c.u[b] = p, q, u
    check(c)
    assert c.accepted.tolist() == [int(x[3]) for x in ACCEPTED]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab,stride,offset", PLACES)
def test_negative_numbers_weigh_nothing(vocab, stride, offset, dtype):
    """Negative numbers among p and q: no weight, and nothing that a weight is lessened by."""
    c = Case([1] * 9, vocab, dtype, True, 4, stride, offset=offset)
    c.target[:, ::3] *= -1
    c.draft[:, ::5] *= -1
    c.draft[:, 3:20:4] = -0.0
    for k in range(3):
        set_numbers(c, k)
        check(c)


def subnormal(shape, dtype, seed):
    """Random subnormal numbers, a quarter of them zero."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    most = 2 ** 23 if dtype == torch.float32 else 2 ** 7
    x = torch.randint(1, most, shape, generator=g, device="cuda") * (torch.rand(shape, generator=g, device="cuda") > 0.25)
    return x.to(torch.int32).view(torch.float32) if dtype == torch.float32 else x.to(torch.int16).view(torch.bfloat16)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab,stride,offset", PLACES)
def test_subnormal_weights(vocab, stride, offset, dtype):
    """Rows that begin with subnormal numbers, or have no others; with a draft and behind the last one."""
    c = Case([0, 1] * 6, vocab, dtype, True, 6, stride, offset=offset)
    c.u.fill_(0.999)
    front = vocab // 2
    c.target[:, :front] = subnormal((c.total + c.n, front), dtype, 1)
    c.target[6:] = subnormal((c.total + c.n - 6, vocab), dtype, 2)      # the later sequences have no others
    c.draft[:, :front] = subnormal((c.total, front), dtype, 3)
    c.draft[4:] = subnormal((c.total - 4, vocab), dtype, 4)
    c.draft[2] = c.target[7]
    c.draft[2, 5] = c.target[7, 5] = 0
    x = c.tokens.long()
    c.target[torch.arange(1, 18, 3, device="cuda"), x] = 0      # rejected
    for v in (0.0, 2.0 ** -149, 2.0 ** -24, 0.25, 0.6171875, 1.0 - 2.0 ** -24):
        c.v.fill_(v)
        check(c)
    assert c.accepted.sum() == 0 and (c.out[torch.arange(0, 18, 3, device="cuda")] >= 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_subnormal_numbers_in_the_test_of_acceptance(dtype):
    small, tiny = (2.0 ** -140, 2.0 ** -149) if dtype == torch.float32 else (2.0 ** -130, 2.0 ** -133)
    rows = [(small, small, 0.5, 1), (small, small, 1.0 - 2.0 ** -24, 1), (small, small * 2, 0.5, 0), (tiny, 0.0, 0.5, 1), (0.0, tiny, 0.0, 0), (tiny, tiny, 0.25, 1),
            (small, 1.0, 2.0 ** -149, 1), (tiny, 1.0, 2.0 ** -133, 0), (2.0 ** -126, small, 0.5, 1), (small, 2.0 ** -126, 0.5, 0)]
    c = Case([1] * len(rows), 600, dtype, True, 7)
    for b, (p, q, u, _) in enumerate(rows):
        c.target[2 * b, c.tokens[b].long()], c.draft[b, c.tokens[b].long()], c.u[b] = p, q, u
    check(c)
    assert c.accepted.tolist() == [x[3] for x in rows]
