"""CPU-side checks of the calls on rows of matrices: every refusal comes before the first CUDA call.  As in
test_abi_cpu.py, no device is visible while fabricated addresses are handed over: a call that its checks
let through answers ABS_ERR_CUDA."""
import itertools
import os
import random

import pytest

import __graft_entry__ as entry
from paper_2412_21124_b200 import binding as B

FAKE = 0x1000000
LET_THROUGH = B.ABS_ERR_CUDA


@pytest.fixture(scope="module", autouse=True)
def _no_visible_device():
    old = os.environ.get("CUDA_VISIBLE_DEVICES")
    os.environ["CUDA_VISIBLE_DEVICES"] = ""
    yield
    if old is None:
        os.environ.pop("CUDA_VISIBLE_DEVICES", None)
    else:
        os.environ["CUDA_VISIBLE_DEVICES"] = old


@pytest.fixture(scope="module")
def L():
    entry.build()
    return B.lib()


def far(i):
    return FAKE + i * 0x10000000


def rows(data=FAKE, s0=64, s1=0, dtype=B.ABS_F32, reserved=0):
    return (data, s0, s1, dtype, reserved)


NONE = (0, 0, 0, 0, 0)


def norm(L, n0=10, n1=1, h=64, x=rows(far(1)), residual=NONE, sum=NONE, out=rows(far(2)), scales=NONE, stride2=0, weight=0,
         w_dtype=0, group=0, eps=1e-6):
    return L.abs_rms_norm(B._NORM_ARGS.pack(n0, n1, h, *x, *residual, *sum, *out, *scales, stride2, weight, w_dtype, group, eps),
                          None)


def grad(L, n0=10, n1=1, h=64, dy=rows(far(1)), s=rows(far(2)), add=NONE, dx=rows(far(3)), weight=0, offsets=0, dw=0, apart=0,
         work=0, n_samples=0, ld=64, work_bytes=0, eps=1e-6, scale=1.0, w_dtype=0):
    return L.abs_rms_norm_grad(B._NORM_GRAD_ARGS.pack(n0, n1, h, *dy, *s, *add, *dx, weight, offsets, dw, apart, work, n_samples,
                                                      ld, work_bytes, eps, scale, w_dtype, 0), None)


def test_argument_blocks_are_those_of_the_header():
    assert (B._NORM_ARGS.size, B._NORM_GRAD_ARGS.size) == (216, 240)


E4 = rows(far(2), dtype=B.ABS_E4M3)
SC = rows(far(5), s0=1)
MX = rows(far(5), s0=2, dtype=B.ABS_E8M0)


@pytest.mark.parametrize("change,status", [
    ({}, LET_THROUGH),
    (dict(n0=0), B.ABS_OK), (dict(n1=0, x=NONE, out=NONE), B.ABS_OK),
    (dict(n0=-1), B.ABS_ERR_RANGE), (dict(h=0), B.ABS_ERR_RANGE), (dict(n0=1 << 31), B.ABS_ERR_RANGE),
    (dict(n0=1 << 20, n1=1 << 20), B.ABS_ERR_RANGE),
    (dict(h=16385, x=rows(far(1), s0=16385), out=rows(far(2), s0=16385)), B.ABS_ERR_TOO_LARGE),
    (dict(x=NONE), B.ABS_ERR_NULL), (dict(out=NONE), B.ABS_ERR_NULL), (dict(sum=rows(far(3))), B.ABS_ERR_NULL),
    (dict(x=rows(far(1), dtype=6)), B.ABS_ERR_DTYPE), (dict(x=rows(far(1), dtype=B.ABS_E4M3)), B.ABS_ERR_DTYPE),
    (dict(out=rows(far(2), dtype=B.ABS_E8M0)), B.ABS_ERR_DTYPE),
    (dict(residual=rows(far(3), dtype=B.ABS_BF16)), B.ABS_ERR_DTYPE),
    (dict(x=rows(far(1), dtype=B.ABS_BF16), residual=rows(far(3))), LET_THROUGH),
    (dict(residual=rows(far(3)), sum=rows(far(4), dtype=B.ABS_BF16)), B.ABS_ERR_DTYPE),
    (dict(x=rows(far(1) + 2)), B.ABS_ERR_ALIGN), (dict(x=rows(far(1) + 2, dtype=B.ABS_BF16)), LET_THROUGH),
    (dict(x=rows(far(1), s0=-64)), B.ABS_ERR_RANGE), (dict(x=rows(far(1), reserved=1)), B.ABS_ERR_RANGE),
    (dict(x=rows(far(1), s0=1 << 45)), B.ABS_ERR_RANGE), (dict(x=rows(far(1), s0=0)), LET_THROUGH),
    (dict(out=rows(far(2), s0=0)), B.ABS_ERR_ALIAS), (dict(out=rows(far(2), s0=63)), B.ABS_ERR_ALIAS),
    (dict(n0=1, out=rows(far(2), s0=0)), LET_THROUGH),
    (dict(eps=0.0), B.ABS_ERR_RANGE), (dict(eps=float("nan")), B.ABS_ERR_RANGE), (dict(eps=float("inf")), B.ABS_ERR_RANGE),
    (dict(weight=far(6)), LET_THROUGH), (dict(weight=far(6), w_dtype=B.ABS_E4M3), B.ABS_ERR_DTYPE),
    (dict(weight=far(6) + 2), B.ABS_ERR_ALIGN), (dict(weight=far(2) + 640), B.ABS_ERR_ALIAS),
    # in place, and not quite
    (dict(out=rows(far(1))), LET_THROUGH), (dict(out=rows(far(1) + 4)), B.ABS_ERR_ALIAS),
    (dict(out=rows(far(1), s0=65)), B.ABS_ERR_ALIAS), (dict(out=rows(far(1), dtype=B.ABS_BF16)), B.ABS_ERR_ALIAS),
    (dict(x=rows(far(1), s0=128), out=rows(far(1) + 256, s0=128)), LET_THROUGH),  # other columns
    (dict(x=rows(far(1), s0=128), out=rows(far(1) + 252, s0=128)), B.ABS_ERR_ALIAS),
    (dict(residual=rows(far(3)), sum=rows(far(3)), out=rows(far(1))), LET_THROUGH),
    (dict(residual=rows(far(3)), sum=rows(far(2))), B.ABS_ERR_ALIAS),
    # 8 bits
    (dict(out=E4), B.ABS_ERR_NULL), (dict(out=E4, scales=SC), LET_THROUGH), (dict(scales=SC), B.ABS_ERR_RANGE),
    (dict(group=32), B.ABS_ERR_RANGE), (dict(out=E4, scales=MX, group=32, stride2=1), LET_THROUGH),
    (dict(out=E4, scales=MX, group=16, stride2=1), B.ABS_ERR_RANGE), (dict(out=E4, scales=MX, group=-1), B.ABS_ERR_RANGE),
    (dict(out=E4, scales=rows(far(5), s0=1, dtype=B.ABS_BF16)), B.ABS_ERR_DTYPE),
    (dict(out=E4, scales=MX, group=32, stride2=0), B.ABS_ERR_ALIAS),
    (dict(out=E4, scales=rows(far(5), s0=1, dtype=B.ABS_E8M0), group=32, stride2=1), B.ABS_ERR_ALIAS),
    (dict(out=E4, scales=rows(far(5), s0=1, dtype=B.ABS_E8M0), group=32, stride2=10), LET_THROUGH),
    (dict(out=E4, scales=rows(far(5), s0=1, dtype=B.ABS_E8M0), group=32, stride2=9), B.ABS_ERR_ALIAS),
    (dict(out=E4, scales=rows(far(2) + 64, s0=1)), B.ABS_ERR_ALIAS),
])
def test_norm_checks(L, change, status):
    assert norm(L, **change) == status


WORK = dict(work=far(7), work_bytes=1 << 20)


@pytest.mark.parametrize("change,status", [
    ({}, LET_THROUGH), (dict(n0=0, dy=NONE, s=NONE, dx=NONE), B.ABS_OK),
    (dict(dy=NONE), B.ABS_ERR_NULL), (dict(s=NONE), B.ABS_ERR_NULL), (dict(dx=NONE), B.ABS_ERR_NULL),
    (dict(dw=far(6)), B.ABS_ERR_NULL), (dict(dw=far(6), **WORK), LET_THROUGH),
    (dict(dw=far(6), work=far(7), work_bytes=11 * 64 * 4 - 1), B.ABS_ERR_TOO_LARGE),
    (dict(dw=far(6), work=far(7), work_bytes=11 * 64 * 4), LET_THROUGH),
    (dict(dw=far(6), work=far(7) + 16, work_bytes=1 << 20), B.ABS_ERR_ALIGN),
    (dict(dw=far(6) + 1, **WORK), B.ABS_ERR_ALIGN), (dict(dw=far(3), **WORK), B.ABS_ERR_ALIAS),
    (dict(dw=far(1), **WORK), B.ABS_ERR_ALIAS), (dict(dw=far(7), **WORK), B.ABS_ERR_ALIAS),
    (dict(dw=far(6), work=far(2), work_bytes=1 << 20), B.ABS_ERR_ALIAS),
    (dict(offsets=far(8)), B.ABS_ERR_NULL), (dict(n_samples=3), B.ABS_ERR_NULL),
    (dict(offsets=far(8), n_samples=3), LET_THROUGH), (dict(offsets=far(8) + 2, n_samples=3), B.ABS_ERR_ALIGN),
    (dict(offsets=far(8), n_samples=(1 << 20) + 1), B.ABS_ERR_RANGE), (dict(n_samples=-1), B.ABS_ERR_RANGE),
    (dict(apart=far(9), **WORK), B.ABS_ERR_NULL),
    (dict(offsets=far(8), n_samples=3, apart=far(9), **WORK), LET_THROUGH),
    (dict(offsets=far(8), n_samples=3, apart=far(9), ld=63, **WORK), B.ABS_ERR_RANGE),
    (dict(offsets=far(8), n_samples=3, apart=far(9), ld=1 << 46, **WORK), B.ABS_ERR_RANGE),
    (dict(offsets=far(8), n_samples=1, apart=far(9), ld=0, **WORK), LET_THROUGH),
    (dict(offsets=far(8), n_samples=3, apart=far(9), dw=far(9) + 256, **WORK), B.ABS_ERR_ALIAS),
    (dict(offsets=far(9), n_samples=3, apart=far(9), **WORK), B.ABS_ERR_ALIAS),
    (dict(weight=far(3)), B.ABS_ERR_ALIAS), (dict(weight=far(6), w_dtype=9), B.ABS_ERR_DTYPE),
    (dict(dx=rows(far(1))), LET_THROUGH), (dict(dx=rows(far(2))), LET_THROUGH), (dict(dx=rows(far(1) + 4)), B.ABS_ERR_ALIAS),
    (dict(dx=rows(far(3), s0=32)), B.ABS_ERR_ALIAS), (dict(dx=rows(far(3), dtype=B.ABS_E4M3)), B.ABS_ERR_DTYPE),
    (dict(dy=rows(far(1), dtype=B.ABS_F16)), LET_THROUGH), (dict(s=rows(far(2), dtype=B.ABS_F16)), B.ABS_ERR_DTYPE),
    (dict(add=rows(far(4), dtype=B.ABS_F16)), B.ABS_ERR_DTYPE),
    (dict(eps=-1.0), B.ABS_ERR_RANGE), (dict(scale=float("nan")), B.ABS_ERR_RANGE), (dict(scale=float("inf")), B.ABS_ERR_RANGE),
])
def test_gradient_checks(L, change, status):
    assert grad(L, **change) == status


def test_work_bytes(L):
    f = L.abs_rms_norm_grad_bytes
    assert f(10, 1, 64, 0) == 11 * 64 * 4 and f(10, 1, 61, 0) == 11 * 64 * 4
    assert f(10, 1, 64, 3) == (10 + 13 + 1) * 64 * 4
    for bad in ((-1, 1, 64, 0), (1, 1, 0, 0), (1, 1, 16385, 0), (1 << 31, 1, 64, 0), (1, 1, 64, -1), (1, 1, 64, (1 << 20) + 1)):
        assert f(*bad) == 0


def test_overlaps_of_views_against_a_search(L):
    """Tensors of the same strides: the answer is exact.  Compared with the sets of bytes that the rows cover."""
    rng = random.Random(1)
    seen = {True: 0, False: 0}
    for _ in range(1500):
        n0, n1, h = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 5)
        s1 = h + rng.randint(0, 4)
        s0 = n1 * s1 + rng.randint(0, 6)
        if rng.random() < 0.3:  # the outer dimension lies inside
            s0, s1 = h + rng.randint(0, 4), 0
            s1 = n0 * s0 + rng.randint(0, 6)
        d = rng.randint(-3 * (s0 + s1), 3 * (s0 + s1))

        def cover(at):
            return {at + i * s0 + j * s1 + c for i, j, c in itertools.product(range(n0), range(n1), range(h))}
        touch = bool(cover(0) & cover(d)) and d != 0
        rc = norm(L, n0, n1, h, x=rows(far(3), s0, s1), out=rows(far(3) + 4 * d, s0, s1))
        assert rc == (B.ABS_ERR_ALIAS if touch else LET_THROUGH), (n0, n1, h, s0, s1, d)
        seen[touch] += 1
    assert min(seen.values()) > 100


# ------------------------------------------------------------------------------------- distillation
def distill(L, rows_=10, vocab=100, top=8, z=rows(far(1), s0=100), dz=NONE, t=rows(far(3), s0=8), ids=far(4), lse=0, weights=0,
            offsets=0, losses=far(5), samples=0, ids_stride=8, n_samples=0, tau=1.0, scale=1.0, id_bytes=8):
    return L.abs_distill_loss(B._DISTILL_ARGS.pack(rows_, vocab, top, *z, *dz, *t, ids, lse, weights, offsets, losses, samples,
                                                   ids_stride, n_samples, tau, scale, id_bytes, 0), None)


def test_distillation_argument_block():
    assert B._DISTILL_ARGS.size == 24 + 3 * 32 + 6 * 8 + 2 * 8 + 2 * 8 + 8


DZ = rows(far(2), s0=100)


@pytest.mark.parametrize("change,status", [
    ({}, LET_THROUGH), (dict(dz=DZ), LET_THROUGH), (dict(rows_=0, z=NONE, t=NONE, ids=0, losses=0), B.ABS_OK),
    (dict(rows_=-1), B.ABS_ERR_RANGE), (dict(rows_=1 << 31), B.ABS_ERR_RANGE), (dict(vocab=0), B.ABS_ERR_RANGE),
    (dict(vocab=(1 << 20) + 1), B.ABS_ERR_TOO_LARGE), (dict(vocab=1 << 20, z=rows(far(1), s0=1 << 20)), LET_THROUGH),
    (dict(top=0), B.ABS_ERR_RANGE), (dict(top=513), B.ABS_ERR_RANGE),
    (dict(tau=0.0), B.ABS_ERR_RANGE), (dict(tau=float("nan")), B.ABS_ERR_RANGE), (dict(tau=1e4), B.ABS_ERR_RANGE),
    (dict(scale=float("nan")), B.ABS_ERR_RANGE), (dict(id_bytes=2), B.ABS_ERR_DTYPE), (dict(id_bytes=4), LET_THROUGH),
    (dict(z=NONE), B.ABS_ERR_NULL), (dict(t=NONE), B.ABS_ERR_NULL), (dict(ids=0), B.ABS_ERR_NULL), (dict(losses=0), B.ABS_ERR_NULL),
    (dict(z=rows(far(1), s0=100, dtype=B.ABS_E4M3)), B.ABS_ERR_DTYPE), (dict(dz=rows(far(2), s0=100, dtype=B.ABS_BF16)), B.ABS_ERR_DTYPE),
    (dict(t=rows(far(3), s0=8, dtype=B.ABS_F16)), LET_THROUGH), (dict(t=rows(far(3), s0=8, dtype=7)), B.ABS_ERR_DTYPE),
    (dict(ids=far(4) + 4), B.ABS_ERR_ALIGN), (dict(ids=far(4) + 4, id_bytes=4), LET_THROUGH), (dict(ids=far(4) + 2, id_bytes=4), B.ABS_ERR_ALIGN),
    (dict(ids_stride=-1), B.ABS_ERR_RANGE), (dict(ids_stride=0, t=rows(far(3), s0=0)), LET_THROUGH),
    (dict(losses=far(5) + 2), B.ABS_ERR_ALIGN), (dict(weights=far(6) + 1), B.ABS_ERR_ALIGN), (dict(lse=far(6) + 1), B.ABS_ERR_ALIGN),
    (dict(offsets=far(7)), B.ABS_ERR_NULL), (dict(n_samples=2), B.ABS_ERR_NULL), (dict(offsets=far(7), n_samples=2), LET_THROUGH),
    (dict(offsets=far(7), n_samples=(1 << 20) + 1), B.ABS_ERR_RANGE),
    (dict(dz=rows(far(1), s0=100)), LET_THROUGH), (dict(dz=rows(far(1) + 4, s0=100)), B.ABS_ERR_ALIAS),
    (dict(z=rows(far(1), s0=200), dz=rows(far(1) + 400, s0=200)), LET_THROUGH),
    (dict(dz=rows(far(2), s0=99)), B.ABS_ERR_ALIAS), (dict(dz=rows(far(3), s0=100)), B.ABS_ERR_ALIAS),
    (dict(dz=rows(far(4) + 64, s0=100)), B.ABS_ERR_ALIAS), (dict(dz=DZ, weights=far(2)), B.ABS_ERR_ALIAS),
    (dict(losses=far(1)), B.ABS_ERR_ALIAS), (dict(losses=far(3)), B.ABS_ERR_ALIAS), (dict(losses=far(4) + 320), B.ABS_ERR_ALIAS),
    (dict(losses=far(4) + 640), LET_THROUGH), (dict(losses=far(4) + 320, id_bytes=4), LET_THROUGH),
    (dict(weights=far(5)), B.ABS_ERR_ALIAS), (dict(samples=far(5) + 36), B.ABS_ERR_ALIAS), (dict(samples=far(5) + 40), LET_THROUGH),
    (dict(lse=far(8), samples=far(8)), B.ABS_ERR_ALIAS), (dict(dz=DZ, samples=far(2)), B.ABS_ERR_ALIAS),
])
def test_distillation_checks(L, change, status):
    assert distill(L, **change) == status


def test_the_self_test_of_its_waits_takes_the_same_arguments(L):
    args = B._DISTILL_ARGS.pack(10, 100, 8, *rows(far(1), s0=100), *NONE, *rows(far(3), s0=8), far(4), 0, 0, 0, far(5), 0, 8, 0, 1.0,
                                1.0, 8, 0)
    for polls, status in ((-1, B.ABS_ERR_RANGE), (0, LET_THROUGH), (2 ** 18, LET_THROUGH), (2 ** 18 + 1, B.ABS_ERR_RANGE)):
        assert L.abs_selftest_distill_wait(args, polls, None) == status
    assert L.abs_selftest_distill_wait(None, 0, None) == B.ABS_ERR_NULL
