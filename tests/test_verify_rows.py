"""Verification of drafted tokens: rows of many pieces, summed twice, and batches of any size (GPU)."""
import pytest
import torch

from test_draft_verify import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1000, 128256, 300001, 600001])
def test_nothing_left_of_the_difference(vocab, dtype, offset):
    """p < q everywhere: the row is summed again, by the last of its CTAs; with more pieces than shared memory has sums for, too."""
    c = Case([1, 0, 2], vocab, dtype, True, 3, offset=offset)
    c.u.fill_(0.99)
    c.target[0].copy_(c.draft[0].float() * 0.5)
    c.target[3].copy_(c.draft[1].float() * 0.25)
    for k in range(4):
        c.v.copy_(torch.tensor([0.2, 0.5, 0.7]) + 0.07 * k)
        c.check()
        assert c.accepted.tolist() == [0, 0, 0]


@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch", [236, 237, 300, 355, 356, 700, 888, 889, 1702, 1777])
def test_large_batches(batch, dtype, with_draft):
    """Around the sizes at which a row is divided among fewer CTAs."""
    c = Case([b % 3 for b in range(batch)], 5003, dtype, with_draft, batch)
    c.check()
    c.check()
