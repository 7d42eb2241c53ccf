"""A wait of the distillation kernel that runs out: rows become NaN, never another number, and the call ends.

The self-test makes the part that loads rows give up as soon as it needs a place a second time.  Nothing is broken on the
way: the rows it has loaded before are worked on, the others' waits end after their limit of about a second.
Tolerances: test_gpu_distill.py."""
import ctypes

import pytest
import torch

import paper_2412_21124_b200 as absnt
from paper_2412_21124_b200 import binding
from tests.test_gpu_distill import BF16, F16, F32, ROUND, STEP, gen, make, plain, table

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("vocab,rows,dtype", ((1000, 6000, BF16), (50257, 2000, BF16), (32000, 2000, F16), (128256, 600, F32)))
def test_a_loader_that_gives_up(vocab, rows, dtype, monkeypatch):
    g = gen(vocab)
    z, ids, t = make(rows, vocab, 9, dtype, g)
    weights = torch.rand(rows, device=DEV, generator=g) + 0.5
    weights[::11] = 0
    offsets = table([rows - 4], 2)
    lse = torch.logsumexp(t, -1) + 0.3
    losses, dz = torch.full((rows,), 3.0, device=DEV), torch.full_like(z, 3.0)
    whole = binding.lib().abs_distill_loss
    short = binding.lib().abs_selftest_distill_wait

    def call():
        absnt.abs_distill_loss(z, ids, t, losses, teacher_lse=lse, weights=weights, offsets=offsets, dlogits=dz)
        torch.cuda.synchronize()

    monkeypatch.setattr(binding.lib(), "abs_distill_loss",
                        lambda args, stream: short(args, 0, ctypes.c_void_p(stream)))
    call()
    got, got_dz = losses.clone(), dz.clone()
    monkeypatch.setattr(binding.lib(), "abs_distill_loss", whole)
    call()  # the context is as usable as before
    ref, tol, grad, err = plain(z, ids, t, lse=lse, weights=weights)
    err = err + grad.abs() * ROUND[dtype] + STEP[dtype]
    own = torch.zeros(rows, dtype=torch.bool, device=DEV)
    own[2:-2] = True
    for x, dx in ((losses, dz), (got, got_dz)):
        assert (x[~own] == 3).all() and (dx[~own] == 3).all()
        assert (x[own & (weights == 0)] == 0).all() and (dx[own & (weights == 0)] == 0).all()
    work = own & (weights != 0)
    assert ((losses.double() - ref).abs() <= tol)[work].all() and ((dz.double() - grad).abs() <= err)[work].all()
    lost = torch.isnan(got)
    assert rows // 10 < int(lost.sum()) < rows and not lost[~work].any()
    right = work & ~lost
    assert ((got.double() - ref).abs() <= tol)[right].all()
    assert torch.isnan(got_dz[lost]).all()
    assert ((got_dz.double() - grad).abs() <= err)[right].logical_or(torch.isnan(got_dz[right])).all()
