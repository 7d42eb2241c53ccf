"""abs_distill_loss on logits that are masked with large finite values, against fp64.

The tolerances are those derived in test_gpu_distill.py.  Every comparison here is one that a NaN fails: a difference
has to be at most its tolerance."""
import pytest
import torch

import paper_2412_21124_b200 as absnt
from tests.test_gpu_distill import BF16, F16, F32, ROUND, STEP, gen, make, plain

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def close(z, ids, t, dz, losses, **more):
    ref, tol, grad, err = plain(z, ids, t, **more)
    ok = (losses.double() - ref).abs() <= tol
    assert ok.all(), (losses[~ok][:4], ref[~ok][:4], tol[~ok][:4], (~ok).nonzero()[:4])
    ok = (dz.double() - grad).abs() <= err + grad.abs() * ROUND[dz.dtype] + STEP[dz.dtype]
    assert ok.all(), (dz[~ok][:4], grad[~ok][:4], err[~ok][:4], (~ok).nonzero()[:4])


@pytest.mark.parametrize("vocab", (200, 50257, 300_000))
@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("tau", (2.0, 20.0))
def test_losses_near_the_largest_float(vocab, dtype, tau):
    """A tenth or so of a row's mass at masking values whose distance times the temperature is no float any more, in the
    rest and in the top: the loss is still one."""
    g = gen(vocab)
    low = -3e38
    z, ids, t = make(4, vocab, 6, dtype, g)
    keep = torch.zeros(4, vocab, dtype=torch.bool, device=DEV).scatter_(1, ids, True)
    z[0] = z[0].masked_fill(~keep[0], low)
    z[1, ids[1, 2]] = low
    t[1, 2] = t[1].amax() - 3 * tau
    z[2] = z[2].masked_fill(~keep[2], low)
    z[2, ids[2, 4]] = low
    t[2, 4] = t[2].amax() - 3 * tau
    lse = torch.logsumexp(t.double() / tau, -1).float() + 0.05 / tau
    losses, dz = torch.empty(4, device=DEV), torch.empty_like(z)
    absnt.abs_distill_loss(z, ids, t, losses, tau, teacher_lse=lse, dlogits=dz)
    assert (losses[:3] > 1e36).all()
    close(z, ids, t, dz, losses, tau=tau, lse=lse)
