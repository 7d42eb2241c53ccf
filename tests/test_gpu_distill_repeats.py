"""An index that a row of the top names several times: its gradient has the same bits whichever entry writes it."""
import pytest
import torch

import paper_2412_21124_b200 as absnt
from tests.test_gpu_distill import F32, gen

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


# a cluster of one block and of several, and the kernel of a block a row; entries of one warp and of four
@pytest.mark.parametrize("vocab", (1000, 50257, 300_000))
@pytest.mark.parametrize("entries", ((0, 100, 200, 300), (3, 9, 20, 31), (5, 6, 399)))
def test_probabilities_of_one_index_are_added_in_the_order_of_the_entries(vocab, entries):
    """The index's logit is so low that its gradient is the probability alone, -p with the factor 1; what each entry's p
    is comes from the same row with four indices, and their sum in fp32 is exact to the bit in one order."""
    rows, top = 200, 400
    g = gen(vocab)
    places = torch.arange(top, device=DEV) * 2 + 1
    ids = places.expand(rows, top).clone()
    t = torch.full((rows, top), -30.0, device=DEV)
    t[:, list(entries)] = torch.randn(rows, len(entries), device=DEV, generator=g) - 3.0
    z = torch.zeros(rows, vocab, device=DEV)
    z[:, places[list(entries)]] = -300.0
    lse = torch.zeros(rows, device=DEV)
    losses, dz = torch.empty(rows, device=DEV), torch.empty_like(z)
    absnt.abs_distill_loss(z, ids, t, losses, teacher_lse=lse, dlogits=dz)
    want = torch.zeros(rows, device=DEV, dtype=F32)
    for j in entries:
        want = want + -dz[:, places[j]]
    ids[:, list(entries)] = places[entries[0]]
    for _ in range(5):
        absnt.abs_distill_loss(z, ids, t, losses, teacher_lse=lse, dlogits=dz)
        assert torch.equal(-dz[:, places[entries[0]]], want)
