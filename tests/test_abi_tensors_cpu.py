"""CPU-side checks of the calls over a list of tensors: the plan is host code and is checked here in
full; every refusal of the launching calls comes before the first CUDA call.  As in
test_abi_cpu.py, no device is visible while fabricated addresses are handed over."""
import ctypes
import os
import random

import pytest

import __graft_entry__ as entry
from paper_2412_21124_b200 import binding as B

FAKE = 0x10000


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


def T(data=FAKE, numel=100, row_len=0, row_stride=0, col_stride=0, dtype=B.ABS_F32, group=0):
    return B.abs_tensor(data, numel, row_len, row_stride, col_stride, dtype, group)


def arr(*ts):
    return (B.abs_tensor * max(len(ts), 1))(*ts)


def plan(L, grads, outs=None, p=None, m=None, v=None, p16=None, short=0):
    g = arr(*grads)
    roles = [arr(*x) if x is not None else None for x in (outs, p, m, v, p16)]
    nbytes = L.abs_tensors_plan_bytes(g, len(grads))
    buf = (ctypes.c_uint64 * (nbytes // 8 + 1))()
    rc = L.abs_tensors_plan(g, *roles, len(grads), buf, nbytes - short)
    return rc, buf


def far(i):
    return FAKE + i * 0x100000


def state(n=1, numel=100, **over):
    x = dict(p=[T(far(10 + i), numel) for i in range(n)], m=[T(far(40 + i), numel) for i in range(n)],
             v=[T(far(70 + i), numel) for i in range(n)])
    x.update(over)
    return x


@pytest.mark.parametrize("grad,status", [
    (T(), B.ABS_OK), (T(numel=0, data=None), B.ABS_OK), (T(numel=1), B.ABS_OK),
    (T(row_len=10, row_stride=12, col_stride=1), B.ABS_OK),
    (T(row_len=10, row_stride=1, col_stride=10), B.ABS_OK),      # transposed
    (T(data=None), B.ABS_ERR_NULL),
    (T(numel=-1), B.ABS_ERR_RANGE), (T(numel=1 << 50), B.ABS_ERR_RANGE),
    (T(dtype=3), B.ABS_ERR_DTYPE), (T(dtype=-1), B.ABS_ERR_DTYPE),
    (T(data=FAKE + 2), B.ABS_ERR_ALIGN), (T(data=FAKE + 1, dtype=B.ABS_BF16), B.ABS_ERR_ALIGN),
    (T(data=FAKE + 2, dtype=B.ABS_F16), B.ABS_OK),
    (T(row_len=7, row_stride=10, col_stride=1), B.ABS_ERR_RANGE),    # 100 is no multiple of 7
    (T(row_len=10, row_stride=9, col_stride=1), B.ABS_ERR_RANGE),    # rows overlap
    (T(row_len=10, row_stride=0, col_stride=1), B.ABS_ERR_RANGE),    # broadcast
    (T(row_len=10, row_stride=10, col_stride=0), B.ABS_ERR_RANGE),
    (T(row_len=-5, row_stride=10, col_stride=1), B.ABS_ERR_RANGE),
    (T(row_len=10, row_stride=1 << 60, col_stride=1), B.ABS_ERR_RANGE),
    (T(numel=1 << 33, row_len=1 << 32, row_stride=1 << 40, col_stride=1), B.ABS_ERR_RANGE),
    (T(numel=1 << 33, row_len=1 << 32, row_stride=1 << 32, col_stride=1), B.ABS_OK),  # no gap
    (T(group=-1), B.ABS_ERR_RANGE), (T(group=16), B.ABS_ERR_RANGE), (T(group=15), B.ABS_OK),
])
def test_plan_of_one_tensor(L, grad, status):
    rc, buf = plan(L, [grad])
    assert rc == status
    assert bool(L.abs_tensors_work_bytes(buf)) == (status == B.ABS_OK)


def test_plan_of_roles(L):
    g = [T(far(1))]
    assert plan(L, g, **state())[0] == B.ABS_OK
    assert plan(L, g, **state(m=None))[0] == B.ABS_ERR_NULL
    assert plan(L, g, p16=[T(far(5), dtype=B.ABS_BF16)])[0] == B.ABS_ERR_NULL
    assert plan(L, g, p16=[T(far(5), dtype=B.ABS_BF16)], **state())[0] == B.ABS_OK
    assert plan(L, g, p16=[T(far(5), dtype=B.ABS_F16)], **state())[0] == B.ABS_ERR_DTYPE
    assert plan(L, g, **state(p=[T(far(10), dtype=B.ABS_BF16)]))[0] == B.ABS_ERR_DTYPE
    assert plan(L, g, **state(v=[T(far(70), 99)]))[0] == B.ABS_ERR_RANGE
    assert plan(L, g, **state(v=[T(far(70), 100, 10, 12, 1)]))[0] == B.ABS_ERR_RANGE
    assert plan(L, g, **state(v=[T(None)]))[0] == B.ABS_ERR_NULL
    assert plan(L, g, outs=[T(far(3), 99)])[0] == B.ABS_ERR_RANGE
    assert plan(L, g, outs=[T(far(3), dtype=B.ABS_F16)])[0] == B.ABS_OK
    assert plan(L, g, outs=[T(far(3), dtype=9)])[0] == B.ABS_ERR_DTYPE


def test_plan_of_overlaps(L):
    alias = B.ABS_ERR_ALIAS
    assert plan(L, [T(far(1))], outs=[T(far(1))])[0] == alias
    assert plan(L, [T(far(1))], outs=[T(far(1) + 396)])[0] == alias      # the last element
    assert plan(L, [T(far(1))], outs=[T(far(1) + 400)])[0] == B.ABS_OK
    assert plan(L, [T(far(1))], **state(m=[T(far(10) + 8)]))[0] == alias
    assert plan(L, [T(far(10) + 8)], **state())[0] == alias
    # an output over another tensor's gradient, far apart in the list
    many = [T(far(1) + 400 * i) for i in range(50)]
    outs = [T(far(2) + 400 * i) for i in range(50)]
    assert plan(L, many, outs=outs)[0] == B.ABS_OK
    outs[3] = T(far(1) + 400 * 40 + 4)
    assert plan(L, many, outs=outs)[0] == alias
    # columns of one matrix: apart, and with a column in common
    col = lambda c, w: T(far(1) + 4 * c, 10 * w, w, 32, 1)  # noqa: E731
    assert plan(L, [T(far(9), 80)], outs=[col(0, 8)])[0] == B.ABS_OK
    assert plan(L, [col(8, 8)], outs=[col(0, 8)])[0] == B.ABS_OK
    assert plan(L, [col(24, 8)], outs=[col(0, 8)])[0] == B.ABS_OK
    assert plan(L, [col(7, 8)], outs=[col(0, 8)])[0] == alias
    assert plan(L, [col(28, 8)], outs=[col(0, 8)])[0] == alias             # wraps into the next row
    # gradients may overlap each other, but not be scaled in place then
    rc, buf = plan(L, [T(far(1)), T(far(1) + 40)])
    assert rc == B.ABS_OK
    assert L.abs_grad_clip(buf, FAKE, B.ABS_NORM_2, 1.0, 1.0, None, far(3), None) == alias
    rc, buf = plan(L, [T(far(1)), T(far(1) + 40)], outs=[T(far(5)), T(far(6))])
    assert rc == B.ABS_OK


def test_plan_arguments(L):
    g = arr(T())
    assert L.abs_tensors_plan_bytes(None, 1) == 0 and L.abs_tensors_plan_bytes(g, -1) == 0
    assert L.abs_tensors_plan_bytes(arr(T(numel=-3)), 1) == 0
    buf = (ctypes.c_uint64 * 1000)()
    assert L.abs_tensors_plan(g, None, None, None, None, None, 1, None, 8000) == B.ABS_ERR_NULL
    assert L.abs_tensors_plan(None, None, None, None, None, None, 1, buf, 8000) == B.ABS_ERR_NULL
    assert L.abs_tensors_plan(g, None, None, None, None, None, -1, buf, 8000) == B.ABS_ERR_RANGE
    assert L.abs_tensors_plan(g, None, None, None, None, None, B.ABS_MAX_TENSORS + 1, buf, 8000) == B.ABS_ERR_RANGE
    at = ctypes.addressof(buf)
    assert L.abs_tensors_plan(g, None, None, None, None, None, 1, at + 4, 7000) == B.ABS_ERR_ALIGN
    for have in (0, 8, 100):
        assert L.abs_tensors_plan(g, None, None, None, None, None, 1, buf, have) == B.ABS_ERR_TOO_LARGE
    assert plan(L, [])[0] == B.ABS_OK
    assert L.abs_tensors_work_bytes(None) == 0
    assert L.abs_tensors_work_bytes((ctypes.c_uint64 * 8)()) == 0
    big = [T(far(i), 1 << 45) for i in range(3)]
    assert L.abs_tensors_plan_bytes(arr(*big), 3) == 0


def test_launching_calls_refuse(L):
    rc, buf = plan(L, [T(far(1), group=2)], **state())
    none = (ctypes.c_uint64 * 8)()
    hp = (B.abs_adamw_hparams * 16)(*[B.abs_adamw_hparams(1e-3, 0.9, 0.999, 1e-8, 0.1)] * 16)
    work, norms = far(100), far(101)
    nan, inf = float("nan"), float("inf")
    assert L.abs_tensors_upload(None, work, None) == B.ABS_ERR_NULL
    assert L.abs_tensors_upload(buf, None, None) == B.ABS_ERR_NULL
    assert L.abs_tensors_upload(none, work, None) == B.ABS_ERR_RANGE
    assert L.abs_tensors_upload(buf, work + 8, None) == B.ABS_ERR_ALIGN

    def norm(plan=buf, work=work, kind=2, scale=1.0, max_norm=0.0, norms=norms):
        return L.abs_grad_norm(plan, work, kind, scale, max_norm, norms, None)

    def clip(plan=buf, work=work, kind=2, scale=1.0, max_norm=1.0, sum_in=None, norms=norms):
        return L.abs_grad_clip(plan, work, kind, scale, max_norm, sum_in, norms, None)

    def adamw(plan=buf, work=work, kind=2, scale=1.0, max_norm=1.0, sum_in=None, norms=norms, hp=hp,
              groups=3, step=1):
        return L.abs_grad_adamw(plan, work, hp, groups, step, kind, scale, max_norm, sum_in, norms, None)

    for call in (norm, clip, adamw):
        assert call(plan=None) == B.ABS_ERR_NULL
        assert call(work=None) == B.ABS_ERR_NULL
        assert call(norms=None) == B.ABS_ERR_NULL
        assert call(plan=none) == B.ABS_ERR_RANGE
        assert call(work=work + 8) == B.ABS_ERR_ALIGN
        assert call(norms=norms + 2) == B.ABS_ERR_ALIGN
        assert call(norms=work + 16) == B.ABS_ERR_ALIAS
        for kind in (-1, 3):
            assert call(kind=kind) == B.ABS_ERR_RANGE
        for scale in (0.0, nan, inf, 1e39, -1e300):
            assert call(scale=scale) == B.ABS_ERR_RANGE
        for max_norm in (-1.0, nan, inf):
            assert call(max_norm=max_norm) == B.ABS_ERR_RANGE
    for call in (clip, adamw):
        assert call(sum_in=FAKE + 4) == B.ABS_ERR_ALIGN
    assert clip(max_norm=0.0) == B.ABS_ERR_RANGE
    assert adamw(hp=None) == B.ABS_ERR_NULL
    assert adamw(step=0) == B.ABS_ERR_RANGE
    for groups in (0, 2, 17):  # the list uses group 2
        assert adamw(groups=groups) == B.ABS_ERR_RANGE
    hp[1].eps = -1.0
    assert adamw() == B.ABS_ERR_RANGE
    rc, bare = plan(L, [T(far(1))])
    hp[1].eps = 1e-8
    assert adamw(plan=bare) == B.ABS_ERR_NULL



def shared(L, a, b):
    """Whether the plan of a list in which `a` is a gradient and `b` an output of another tensor finds
    an element that both hold."""
    rc, _ = plan(L, [a, T(far(200), b.numel)], outs=[T(far(220), a.numel), b])
    assert rc in (B.ABS_OK, B.ABS_ERR_ALIAS)
    return rc == B.ABS_ERR_ALIAS


def test_views_that_interleave(L):
    at = far(1)
    # even and odd columns of a matrix of 10 x 20
    even, odd = T(at, 100, 10, 20, 2), T(at + 4, 100, 10, 20, 2)
    assert not shared(L, even, odd) and not shared(L, odd, even)
    assert shared(L, even, T(at + 8, 90, 9, 20, 2))
    # column slices of a transposed matrix, the columns walked first
    left, right = T(at, 80, 10, 1, 20), T(at + 4 * 8, 120, 10, 1, 20)
    assert not shared(L, left, right)
    assert shared(L, left, T(at + 4 * 7, 120, 10, 1, 20))
    # a contiguous tensor between two rows, and one that reaches into the second
    rows = T(at, 40, 8, 20, 1)
    assert not shared(L, rows, T(at + 32, 12)) and not shared(L, T(at + 32, 12), rows)
    assert shared(L, rows, T(at + 32, 13)) and shared(L, rows, T(at + 28, 12))
    # rows of different strides: every fourth, every third, every fourth of them in the gaps
    assert not shared(L, T(at, 50, 1, 4, 1), T(at + 4, 25, 1, 8, 1))
    assert shared(L, T(at, 50, 1, 4, 1), T(at + 4, 50, 1, 3, 1))
    # 16-bit views between fp32 ones
    assert not shared(L, T(at, 100, 10, 20, 2), T(at + 4, 100, 10, 40, 4, B.ABS_BF16))
    assert not shared(L, T(at, 100, 10, 20, 2), T(at + 6, 100, 10, 40, 4, B.ABS_F16))
    assert shared(L, T(at, 100, 10, 20, 2), T(at + 2, 100, 10, 40, 4, B.ABS_F16))
    # a whole embedding's columns dealt out to two, far apart in a long matrix
    assert not shared(L, T(at, 50_000 * 96, 96, 192, 2), T(at + 4, 50_000 * 96, 96, 192, 2))
    assert shared(L, T(at, 50_000, 1, 1001, 1), T(at + 4 * 1001 * 40_000, 7000, 1, 997, 1))


def test_views_share_an_element_or_not(L):
    """Against the elements themselves, random pairs of views."""
    rng = random.Random(7)

    def view():
        esz, dtype = rng.choice(((4, B.ABS_F32), (2, B.ABS_BF16)))
        inner, outer = rng.choice((1, 1, 2, 3, 8)), rng.choice((1, 2, 5, 12))
        step = rng.choice((1, 1, 2, 3, 5))
        stride = (inner - 1) * step + 1 + rng.choice((0, 0, 1, 2, 7, 40))
        if rng.random() < 0.3:  # the columns walked first
            inner, outer, step, stride = outer, inner, stride, step
        at = FAKE + esz * rng.randrange(0, 160)
        held = {at + esz * (i * stride + j * step) + k for i in range(outer) for j in range(inner)
                for k in range(esz)}
        return T(at, inner * outer, inner, stride, step, dtype), held

    found = [0, 0]
    for _ in range(20_000):
        (a, x), (b, y) = view(), view()
        assert shared(L, a, b) == bool(x & y), (
            [(t.data - FAKE, t.numel, t.row_len, t.row_stride, t.col_stride, t.dtype) for t in (a, b)])
        found[bool(x & y)] += 1
    assert min(found) > 2000


def test_results_and_work_area_over_the_lists_tensors(L):
    """norms_out (n + 2 floats) and the work area share no byte with a tensor of the list.  (Clipping with
    max_norm 0 is refused too, but after that.)"""
    rows = T(far(1), 200, 20, 64, 1)  # ten rows of 20 floats, 64 apart
    rc, buf = plan(L, [rows, T(far(2), 10, dtype=B.ABS_BF16)], outs=[T(far(3), 200), T(far(4), 10)],
                   p16=[T(far(5), 200, dtype=B.ABS_BF16), T(far(6), 10, dtype=B.ABS_BF16)],
                   **{k: [T(far(i), 200), T(far(i + 1), 10)] for k, i in (("p", 10), ("m", 40), ("v", 70))})
    assert rc == B.ABS_OK
    hp = (B.abs_adamw_hparams * 1)(B.abs_adamw_hparams(1e-3, 0.9, 0.999, 1e-8, 0.1))
    size = L.abs_tensors_work_bytes(buf)
    work, apart = far(100), far(101)
    taken = [far(i) + 4 for i in (1, 3, 4, 5, 10, 11, 40, 41, 70, 71)]
    taken += [far(2) + 16, far(6) + 16, far(3) + 796]       # the last elements
    taken += [far(1) + 64 * 4 * 9 + 76, far(3) - 12]        # of the rows; norms_out reaches into it
    free = [far(2) + 20, far(3) + 800, far(3) - 16, far(1) + 64 * 4 * 9 + 80]
    free += [far(1) + 80, far(1) + 64 * 4 - 16]              # between two rows
    for at in taken:
        assert L.abs_grad_norm(buf, work, 2, 1.0, 0.0, at, None) == B.ABS_ERR_ALIAS
        assert L.abs_grad_clip(buf, work, 2, 1.0, 0.0, None, at, None) == B.ABS_ERR_ALIAS
        assert L.abs_grad_adamw(buf, work, hp, 1, 1, 2, 1.0, 1.0, None, at, None) == B.ABS_ERR_ALIAS
    for at in free:
        assert L.abs_grad_clip(buf, work, 2, 1.0, 0.0, None, at, None) == B.ABS_ERR_RANGE
    for at in (far(1), far(2) - 16, (far(4) - size + 16) & ~15, (far(11) - size + 16) & ~15, far(70) + 32):
        assert L.abs_tensors_upload(buf, at, None) == B.ABS_ERR_ALIAS
        assert L.abs_grad_norm(buf, at, 2, 1.0, 0.0, apart, None) == B.ABS_ERR_ALIAS
    assert L.abs_grad_clip(buf, far(4) - ((size + 15) & ~15), 2, 1.0, 0.0, None, apart, None) == B.ABS_ERR_RANGE
    # none of it for an empty list
    rc, buf = plan(L, [T(None, 0)])
    assert rc == B.ABS_OK and L.abs_grad_clip(buf, work, 2, 1.0, 0.0, None, apart, None) == B.ABS_ERR_RANGE


def test_a_scale_that_is_zero_as_a_float(L):
    """grad_scale is a float: below its range the norm would be scaled and the gradients be zeroed."""
    rc, buf = plan(L, [T(far(1))], **state())
    hp = (B.abs_adamw_hparams * 1)(B.abs_adamw_hparams(1e-3, 0.9, 0.999, 1e-8, 0.1))
    for scale in (1e-60, -1e-60, 5e-324, 7e-46):
        assert L.abs_grad_norm(buf, far(100), 2, scale, 0.0, far(101), None) == B.ABS_ERR_RANGE
        assert L.abs_grad_clip(buf, far(100), 2, scale, 1.0, None, far(101), None) == B.ABS_ERR_RANGE
        assert L.abs_grad_adamw(buf, far(100), hp, 1, 1, 2, scale, 1.0, None, far(101), None) == B.ABS_ERR_RANGE
