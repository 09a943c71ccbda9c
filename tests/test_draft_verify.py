"""Verification of drafted tokens: accepted numbers and tokens are equal to the definition's in 64 bits (GPU)."""
import numpy as np
import pytest
import torch

from paper_2412_07017_b200 import binding as B

pytestmark = pytest.mark.gpu


def reference(indptr, target, draft, tokens, u, v):
    """numpy, a sequence at a time; the arrays on the host in 64 bits."""
    accepted, out = [], []
    for b in range(len(indptr) - 1):
        i0, i1 = indptr[b], indptr[b + 1]
        a = 0
        while i0 + a < i1:
            x = tokens[i0 + a]
            inside = 0 <= x < target.shape[1]
            if not (inside and u[i0 + a] * (1.0 if draft is None else draft[i0 + a, x]) < target[i0 + a + b, x]):
                break
            a += 1
        p = np.maximum(np.nan_to_num(target[i0 + a + b], nan=0.0), 0.0)
        w = p.copy()
        if i0 + a < i1:
            if draft is not None:
                w = np.nan_to_num(np.maximum(target[i0 + a + b] - draft[i0 + a], 0.0), nan=0.0)
            elif 0 <= tokens[i0 + a] < len(w):
                w[tokens[i0 + a]] = 0.0
        token = -1
        for w in (w, p):
            if w.sum() > 0:
                over = np.cumsum(w) > v[b] * np.cumsum(w)[-1]
                token = int(over.argmax()) if over.any() else int(np.nonzero(w)[0][-1])
                break
        accepted.append(a)
        out += list(tokens[i0:i0 + a]) + [token] + [-1] * (i1 - i0 - a)
    return accepted, out


class Case:
    def __init__(self, drafts, vocab, dtype=torch.float32, with_draft=True, seed=0, stride=None, apart=0.7, offset=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.total, self.vocab = len(drafts), int(sum(drafts)), vocab
        self.indptr = torch.tensor(np.concatenate([[0], np.cumsum(drafts)]), dtype=torch.int32, device="cuda")

        def rows(n, values):
            base = torch.full((n * (stride or vocab) + offset + vocab,), float("nan"), dtype=dtype, device="cuda")
            t = base[offset:offset + n * (stride or vocab)].view(n, stride or vocab)[:, :vocab]
            t.copy_(values)
            return t
        logits = 2 * torch.randn((self.total + self.n, vocab), generator=g, device="cuda")
        at = torch.tensor([i + b for b in range(self.n) for i in range(int(self.indptr[b]), int(self.indptr[b + 1]))], dtype=torch.long, device="cuda")
        q = torch.softmax(logits[at] + apart * torch.randn((self.total, vocab), generator=g, device="cuda"), -1)
        self.target = rows(self.total + self.n, torch.softmax(logits, -1))
        self.draft = rows(self.total, q) if with_draft else None
        self.tokens = (q / torch.empty_like(q).exponential_(generator=g)).argmax(-1).int() if self.total else torch.zeros(0, dtype=torch.int32, device="cuda")
        self.u, self.v = torch.rand(self.total, generator=g, device="cuda"), torch.rand(self.n, generator=g, device="cuda")
        self.workspace = torch.zeros(B.draft_verify_workspace_bytes(self.n, vocab), dtype=torch.uint8, device="cuda")
        self.accepted = torch.full((self.n,), 99, dtype=torch.int32, device="cuda")
        self.out = torch.full((self.total + self.n,), 99, dtype=torch.int32, device="cuda")

    def call(self):
        B.asynclm_draft_verify(self.indptr, self.target, self.draft, self.tokens, self.u, self.v, self.accepted, self.out, self.workspace)

    def want(self):
        host = lambda t: None if t is None else t.cpu().double().numpy()      # noqa: E731
        return reference(self.indptr.cpu().numpy(), host(self.target), host(self.draft), self.tokens.cpu().numpy(), host(self.u), host(self.v))

    def check(self):
        self.call()
        assert (self.accepted.cpu().tolist(), self.out.cpu().tolist()) == self.want()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("drafts,vocab", [([1], 1), ([0], 5), ([4, 0, 2], 511), ([1, 2, 3], 512), ([5] * 3, 513), ([3, 0, 8, 1], 32001), ([40, 0, 33], 700), ([2] * 7, 128256),
                                          ([1] * 700, 1030), ([0] * 5, 4096), ([1, 0, 2], 600001)])
def test_exact(drafts, vocab, with_draft, dtype):
    for seed in range(3):
        c = Case(drafts, vocab, dtype, with_draft, seed, apart=(0.05, 0.7, 2.0)[seed])
        c.check()
        c.check()      # the workspace is fit for the next call


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,stride,offset", [(1000, 1003, 0), (1000, 1000, 1), (1001, 1008, 0), (1003, 1003, 3), (4096, 8192, 8)])
def test_strides(vocab, stride, offset, dtype):
    Case([3, 1, 0, 5], vocab, dtype, True, 3, stride, offset=offset).check()


def test_rows_beyond_32_bits():
    """Rows that lie more than 2^31 values behind the first."""
    c = Case([7, 8, 4], 5000, torch.bfloat16, seed=8)
    for name in ("target", "draft"):
        t = getattr(c, name)
        base = torch.empty(t.shape[0] * (2 ** 27 + 3), dtype=t.dtype, device="cuda").view(t.shape[0], -1)[:, :5000]
        base.copy_(t)
        setattr(c, name, base)
    assert 21 * (2 ** 27 + 3) > 2 ** 31
    c.check()


def test_random_numbers_at_the_ends():
    c = Case([2, 2, 2], 5000, seed=4)
    for x in (0.0, 1.0 - 2.0 ** -24):
        c.u.fill_(x), c.v.fill_(x)
        c.check()
    c.target[:, :100] = 0      # u = 0 takes the first token with a weight
    c.v.fill_(0.0), c.u.fill_(1.0)
    c.check()
    for x in (1.0, 7.0, float("nan"), -1.0):      # outside [0, 1): a token all the same
        c.u.fill_(0.999), c.v.fill_(x)
        c.call()
        assert ((c.out >= -1) & (c.out < 5000)).all() and (c.out[c.indptr[:-1].long() + torch.arange(3, device="cuda") + c.accepted.long()] >= 0).all()


def test_weights_that_are_nothing():
    c = Case([2, 2, 1, 0], 1000, seed=5)
    c.u.fill_(0.999999)
    c.target[0] = c.draft[0] * 0.5      # p < q everywhere: the target's own
    c.target[3] = 0                     # no probability at all
    c.target[6] = float("nan")
    c.target[8] = 0                     # the last sequence has no draft: row drafts + batch - 1
    c.check()
    assert c.out[8] == -1
    one = Case([1], 1000, with_draft=False)
    one.target[0] = 0
    one.target[0, 77], one.tokens[0], one.u[0] = 0.5, 77, 0.9
    one.check()
    assert one.accepted[0] == 0 and one.out[0] == 77


def test_tokens_outside_the_vocabulary():
    for with_draft in (True, False):
        c = Case([3, 3], 600, with_draft=with_draft)
        c.u.fill_(0.0)
        c.tokens[1], c.tokens[3] = 600, -5
        c.check()
        assert c.accepted.tolist() == [1, 0]


def test_all_accepted_and_equal_distributions():
    c = Case([6, 6], 3001, seed=7, apart=0.0)
    c.draft.copy_(c.target[torch.tensor([0, 1, 2, 3, 4, 5, 7, 8, 9, 10, 11, 12], device="cuda")])
    c.check()
    assert c.accepted.tolist() == [6, 6]


def test_one_workspace_for_calls_of_different_sizes():
    big = Case([3] * 50, 20000)
    small = Case([1, 2], 70000, seed=2)
    small.workspace = big.workspace
    for c in (big, small, big, Case([0] * 33, 777)):
        c.workspace = big.workspace
        c.check()


def test_graph_and_stream():
    c = Case([5, 2, 0, 7], 40000, seed=9)
    c.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call()
        c.call()
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        c.u.copy_(torch.rand(c.total, generator=g, device="cuda"))
        c.v.copy_(torch.rand(c.n, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert (c.accepted.cpu().tolist(), c.out.cpu().tolist()) == c.want()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.check()


def test_distribution():
    """What is emitted is distributed as the target: 40 000 sequences of one draft each over a vocabulary of 6, within 5 standard deviations."""
    n, vocab = 40000, 6
    g = torch.Generator(device="cuda").manual_seed(1)
    p = torch.softmax(torch.randn((1, vocab), generator=g, device="cuda"), -1)
    q = torch.softmax(torch.randn((1, vocab), generator=g, device="cuda"), -1)
    c = Case([1] * n, vocab)
    c.target.copy_(p.expand(2 * n, vocab))
    c.draft.copy_(q.expand(n, vocab))
    c.tokens.copy_(torch.multinomial(q[0], n, replacement=True, generator=g))
    c.u.copy_(torch.rand(n, generator=g, device="cuda"))
    c.v.copy_(torch.rand(n, generator=g, device="cuda"))
    c.call()
    first = c.out[0::2].long()
    share = torch.bincount(first, minlength=vocab).double() / n
    assert ((share - p[0].double()).abs() <= 5 * (p[0] * (1 - p[0]) / n).double().sqrt()).all()


def test_refusals():
    c = Case([2, 1], 100)
    args = lambda: [c.indptr, c.target, c.draft, c.tokens, c.u, c.v, c.accepted, c.out, c.workspace]      # noqa: E731

    def refused(at, bad):
        a = args()
        a[at] = bad
        with pytest.raises(ValueError):
            B.asynclm_draft_verify(*a)
    for at, bad in ((0, c.indptr.long()), (1, c.target[:-1]), (1, c.target.half()), (1, c.target.t()), (1, c.target.cpu()), (2, c.draft.bfloat16()), (2, c.draft[:, :99]),
                    (2, c.draft[:1].expand(3, 100)), (3, c.tokens.float()), (4, c.u[:2]), (5, c.v.double()), (6, c.accepted[:1]), (7, c.out[:-1]),
                    (8, c.workspace[:100])):
        refused(at, bad)
    a = args()
    a[8] = c.workspace[1:]      # misaligned (and too small)
    with pytest.raises(ValueError):
        B.asynclm_draft_verify(*a)
    c.check()
