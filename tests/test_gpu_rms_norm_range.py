"""abs_rms_norm and its gradient where the numbers are large or small.

Tolerances: those derived in test_gpu_rms_norm.py, in a form that a NaN fails."""
import pytest
import torch

import paper_2412_21124_b200 as absnt
from tests.test_gpu_rms_norm import (E, E4M3, E8M0, F32, ROUND, STEP, check_weight, gen, near_scaled, plain, plain_grad,
                                     rand)

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def within(got, ref, tol):
    got = got.double()
    ok = (got - ref).abs() <= tol
    assert ok.all(), (got[~ok][:4], ref[~ok][:4], tol[~ok][:4], (~ok).nonzero()[:4])


@pytest.mark.parametrize("width", (60, 64, 512, 1000, 1001, 2048, 4096, 16384))
@pytest.mark.parametrize("eps", (1e30, 1e26))
def test_eps_counts_on_both_sides_of_the_largest_sum(width, eps):
    """Rows just below and above a sum of squares of 1e36, for whole rows and for the part of a warp."""
    g = gen(width)
    sizes = [f * (1e36 / n) ** 0.5 for n in (width, 128, 256, 512) for f in (0.9, 1.1)] + [1e15, 3e18, 1e25]
    x = rand((len(sizes), width), F32, g) * torch.tensor(sizes, device=DEV)[:, None]
    out = torch.empty_like(x)
    absnt.abs_rms_norm(x, None, out, eps)
    y = plain(x, None, None, eps)[1]
    within(out, y, y.abs() * (32 * E + ROUND[F32]) + STEP[F32])
    dy, dx, dw = rand(x.shape, F32, g), torch.empty_like(x), torch.empty(width, device=DEV)
    absnt.abs_rms_norm_grad(dy, x, None, dx, dw, eps, work=absnt.alloc_rms_norm_work(x))
    ref, size, part = plain_grad(dy, x, None, None, eps)
    within(dx, ref, size + ref.abs() * (ROUND[F32] + E) + STEP[F32])
    check_weight(dw, part)


@pytest.mark.parametrize("width", (60, 64, 99, 512, 1001, 4096, 16384))
@pytest.mark.parametrize("group", (0, 32, 128))
@pytest.mark.parametrize("size,weight,eps", ((1e17, 1e25, 1e-6), (1e30, 1e36, 1e-6), (1e-14, 1e-28, 1e-30)))
def test_eight_bits_where_the_row_times_its_weight_is_no_float(width, group, size, weight, eps):
    """y is one: the row is normalised before the weight's turn."""
    g = gen(width)
    for kind in (F32, E8M0):
        x = rand((5, width), F32, g, size)
        w = weight * (1 + 0.2 * torch.randn(width, device=DEV, generator=g))
        q = torch.empty(5, width, device=DEV, dtype=E4M3)
        scales = torch.empty(5, -(-width // group) if group else 1, device=DEV, dtype=kind)
        absnt.abs_rms_norm(x, w, q, eps, scales_out=scales, group=group)
        near_scaled(q, scales, plain(x, w, None, eps)[1], group)
