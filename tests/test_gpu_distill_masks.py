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


# one warp of a row's block up to eight blocks a row; both sides of the products at which a value's distance from the
# reference is formed another way, and where the product leaves the range of a float
MASKS = (-1e4, -1e6, -1.2e7, -1e9, -1e10, -1e20, -1e30, -5e35, -3e38)


@pytest.mark.parametrize("vocab", (200, 1000, 4096, 50257, 128256))
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("tau", (1.0, 2.0, 0.1, 1e-3))
def test_masks_of_large_finite_values(vocab, dtype, tau):
    g = gen(vocab)
    masks = [m for m in MASKS if m >= torch.finfo(dtype).min]
    rows = 5 * len(masks)
    z, ids, t = make(rows, vocab, 12, dtype, g)
    keep = torch.zeros(rows, vocab, dtype=torch.bool, device=DEV).scatter_(1, ids, True)
    at = torch.arange(vocab, device=DEV)
    for k, mask in enumerate(masks):
        # the whole rest; half of the vocabulary; its last quarter; all but the first 256 places (one warp's); all but
        # one place far from the top
        for j, hidden in enumerate((at >= 0, at < vocab // 2, at >= vocab - vocab // 4, at >= 256, at != vocab // 3)):
            row = 5 * k + j
            z[row] = z[row].masked_fill(hidden & ~keep[row], mask)
    for lse in (None, torch.logsumexp(t.double() / tau, -1).float() + 0.5):
        for scale in (1.0, 1e30) if dtype == F32 else (1.0,):
            losses, dz = torch.empty(rows, device=DEV), torch.empty_like(z)
            absnt.abs_distill_loss(z, ids, t, losses, tau, teacher_lse=lse, dlogits=dz, grad_scale=scale)
            close(z, ids, t, dz, losses, tau=tau, lse=lse, scale=scale)
            alone = torch.empty(rows, device=DEV)
            absnt.abs_distill_loss(z, ids, t, alone, tau, teacher_lse=lse)
            assert torch.equal(alone, losses)


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_large_logits_that_differ_a_little(dtype):
    """Values next to one another at 1e6 to 1e9, as the type holds them: their distances are what counts."""
    g = gen(1)
    for vocab in (1000, 50257):
        for k, high in enumerate((1e6, 3e7, -3e7, 1e9)):
            z, ids, t = make(6, vocab, 12, dtype, g)
            z = (z.float() + high).to(dtype)
            step = torch.finfo(dtype).eps * abs(high)
            tau = max(1.0, min(step / 4, 1e3))
            losses, dz = torch.empty(6, device=DEV), torch.empty_like(z)
            absnt.abs_distill_loss(z, ids, t, losses, tau, dlogits=dz)
            close(z, ids, t, dz, losses, tau=tau)
