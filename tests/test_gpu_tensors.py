"""The calls over a list of tensors (abs_grad_norm, abs_grad_clip, abs_grad_adamw) against plain
implementations in fp64.

Tolerances, from the arithmetic: at most eight values are added in fp32 before a sum goes on in fp64,
so a power sum is off by at most 8 * 2^-24 of itself (all terms are positive), a norm by as much
(p = 1; half of it for p = 2), and its fp32 copy by 2^-24 more: NORM_REL = 9 * 2^-24.  A clipped
value carries the factor's error (NORM_REL and a rounding) and one rounding to its own type.
A moment is two products and a sum; the update carries the errors of both moments, and the
approximate square root and reciprocal (2^-22 each)."""
import math

import pytest
import torch

import paper_2412_21124_b200 as absnt
from paper_2412_21124_b200 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NORM_REL = 9 * 2.0 ** -24
# one rounding to the type, and its smallest step
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
STEP = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
ORDERS = (2, 1, math.inf)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def make(shape, dtype, layout, g, std=1.0):
    """A tensor of random values: dense, a view at an odd offset, columns of a wider matrix (of an
    even or an odd width), a single column, or dense with its dimensions swapped."""
    x = torch.randn(shape, device=DEV, generator=g) * std
    if layout == "odd":
        t = torch.empty(x.numel() + 3, device=DEV, dtype=dtype)[3:].view(shape)
    elif layout in ("columns", "columns_odd") and x.dim() == 2:
        width, at = (2 * shape[1], 0) if layout == "columns" else (2 * shape[1] + 1, shape[1])
        t = torch.empty(shape[0], width, device=DEV, dtype=dtype)[:, at:at + shape[1]]
    elif layout == "swapped" and x.dim() == 2:
        t = torch.empty(shape[1], shape[0], device=DEV, dtype=dtype).t()
    else:
        t = torch.empty(shape, device=DEV, dtype=dtype)
    t.copy_(x)
    return t


def ref_norms(grads, order, scale):
    each = torch.stack([torch.linalg.vector_norm(g.double().reshape(-1), order) if g.numel()
                        else torch.zeros((), dtype=torch.float64, device=DEV) for g in grads]) * abs(scale)
    return torch.linalg.vector_norm(each, order), each


def check_norms(ts, grads, order, scale=1.0):
    total, each = ref_norms(grads, order, scale)
    assert abs(float(ts.norm) - float(total)) <= NORM_REL * float(total)
    assert ((ts.norms.double() - each).abs() <= NORM_REL * each).all()
    assert float(ts.header[absnt.ABS_GRAD_FLAGS]) == 0.0
    return float(total)


def check_scaled(got, x, factor, dtype):
    ref = x.double() * factor
    tol = ref.abs() * (NORM_REL + 2.0 ** -23 + ROUND[dtype]) + STEP[dtype]
    assert ((got.double() - ref).abs() <= tol).all()


SHAPES = [(1,), (0,), (7,), (64, 50), (33, 129), (1000,), (300, 257), (5, 1), (1, 4096), (40_009,)]
# beside them: nothing (the list fits one cluster), or a tensor that makes it one for all SMs
MORE = ([], [(1500, 1100)])
LAYOUTS = ("dense", "odd", "columns", "columns_odd", "swapped")


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("more", MORE)
def test_norm(more, order, dtype, layout):
    g = gen(1)
    grads = [make(s, dtype, layout, g, 0.01 * (i + 1)) for i, s in enumerate(SHAPES + more)]
    ts = absnt.GradTensors(grads)
    for scale in (1.0, 0.125, -3.0):  # the same object, called again
        absnt.abs_grad_norm(ts, norm_type=order, grad_scale=scale)
        check_norms(ts, grads, order, scale)
    assert float(ts.coef) == 1.0


@pytest.mark.parametrize("sizes", [(1,), (2,), (8,), (31, 33), (255, 256, 257), (1023, 1024, 1025),
                                   (2047, 2048, 2049, 4097), (65_537,), (3_000_001,),
                                   (1,) * 700, (10_000_001, 3, 4_000_000)])
@pytest.mark.parametrize("dtype", (F32, BF16))
def test_norm_sizes(sizes, dtype):
    g = gen(len(sizes) + sum(sizes))
    grads = [make((n,), dtype, ("dense", "odd")[i % 2], g) for i, n in enumerate(sizes)]
    ts = absnt.GradTensors(grads)
    absnt.abs_grad_norm(ts)
    check_norms(ts, grads, 2)


def test_types_mixed_in_one_list():
    g = gen(3)
    grads = [make((300, 77 + i), (F32, BF16, F16)[i % 3], LAYOUTS[i % 5], g, 10.0 ** (i % 4 - 2))
             for i in range(30)]
    outs = [torch.empty(x.shape, device=DEV, dtype=(BF16, F32, F16, F32)[i % 4])
            for i, x in enumerate(grads)]
    before = [x.clone() for x in grads]
    ts = absnt.GradTensors(grads, out=outs)
    absnt.abs_grad_clip(ts, 2.5, grad_scale=0.5)
    total = check_norms(ts, grads, 2, 0.5)
    coef = 2.5 / (total + 1e-6)
    assert abs(float(ts.coef) - coef) <= (NORM_REL + 2.0 ** -23) * coef
    for x, b, y in zip(grads, before, outs):
        assert torch.equal(x, b)
        check_scaled(y, x, 0.5 * coef, y.dtype)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("more", MORE)
def test_clip_in_place(more, order, dtype, layout):
    g = gen(5)
    grads = [make(s, dtype, layout, g, 0.1) for s in SHAPES + more]
    before = [x.clone() for x in grads]
    total, _ = ref_norms(grads, order, 1.0)
    total = float(total)
    ts = absnt.GradTensors(grads)
    # above the norm: nothing changes, bit for bit
    assert absnt.abs_grad_clip(ts, 2 * total, norm_type=order) is ts.norm
    assert float(ts.coef) == 1.0
    assert all(torch.equal(x, b) for x, b in zip(grads, before))
    absnt.abs_grad_clip(ts, 0.3 * total, norm_type=order)
    check_norms(ts, before, order)
    factor = 0.3 * total / (total + 1e-6)
    for x, b in zip(grads, before):
        check_scaled(x, b, factor, dtype)


@pytest.mark.parametrize("out_dtype", (F32, BF16, F16))
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("layouts", [("dense", "dense"), ("dense", "odd"), ("odd", "odd"),
                                     ("columns", "dense"), ("dense", "columns"),
                                     ("columns_odd", "columns"), ("swapped", "swapped"),
                                     ("dense", "swapped"), ("swapped", "columns")])
@pytest.mark.parametrize("more", MORE)
def test_clip_into(more, layouts, dtype, out_dtype):
    g = gen(6)
    shapes = SHAPES + [(600, 520)] + more
    grads = [make(s, dtype, layouts[0], g, 0.1) for s in shapes]
    outs = [make(s, out_dtype, layouts[1], g) for s in shapes]
    before = [x.clone() for x in grads]
    ts = absnt.GradTensors(grads, out=outs)
    for max_norm in (1.0, 1e9):
        absnt.abs_grad_clip(ts, max_norm, grad_scale=0.25)
        total = check_norms(ts, grads, 2, 0.25)
        factor = 0.25 * min(1.0, max_norm / (total + 1e-6))
        for x, b, y in zip(grads, before, outs):
            assert torch.equal(x, b)
            check_scaled(y, x, factor, out_dtype)


def test_every_other_column():
    g = gen(16)
    parent = torch.randn(70, 90, device=DEV, generator=g)
    before = parent.clone()
    ts = absnt.GradTensors([parent[:, ::2], parent[3, 1::2]])  # the second one: a column of 45
    absnt.abs_grad_norm(ts)
    check_norms(ts, [parent[:, ::2], parent[3, 1::2]], 2)
    ts = absnt.GradTensors([parent[:, ::2]])
    absnt.abs_grad_clip(ts, 1.0)
    total = check_norms(ts, [before[:, ::2]], 2)
    check_scaled(parent[:, ::2], before[:, ::2], 1.0 / (total + 1e-6), F32)
    assert torch.equal(parent[:, 1::2], before[:, 1::2])


def test_interleaved_slices_in_place():
    """Three gradients that are the columns of one matrix do not overlap and leave the gap alone."""
    g = gen(7)
    parent = torch.randn(129, 100, device=DEV, generator=g)
    before = parent.clone()
    views = lambda t: [t[:, 0:32], t[:, 32:65], t[:, 70:97]]  # noqa: E731
    ts = absnt.GradTensors(views(parent))
    absnt.abs_grad_clip(ts, 1.0)
    total = check_norms(ts, views(before), 2)
    for x, b in zip(views(parent), views(before)):
        check_scaled(x, b, 1.0 / (total + 1e-6), F32)
    assert torch.equal(parent[:, 65:70], before[:, 65:70])
    assert torch.equal(parent[:, 97:], before[:, 97:])


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("rows", (70, 9000))
def test_interleaved_views_in_place(rows, dtype):
    """Gradients in each other's gaps, in one list, scaled in place: even and odd columns, a contiguous
    one between two rows of another, columns of a transposed matrix."""
    g = gen(22)
    parents = [make((rows, 90), dtype, "dense", g), make((rows, 64), dtype, "dense", g),
               make((rows, 50), dtype, "swapped", g)]
    views = lambda a, b, c: [a[:, ::2], a[:, 1::2], b[:, :20], b[3, 20:], c[:, 8:31], c[:, :8]]  # noqa: E731
    before = [x.clone() for x in parents]
    ts = absnt.GradTensors(views(*parents))
    absnt.abs_grad_clip(ts, 1.0)
    total = check_norms(ts, views(*before), 2)
    for x, b in zip(views(*parents), views(*before)):
        check_scaled(x, b, 1.0 / (total + 1e-6), dtype)
    assert torch.equal(parents[1][4:, 20:], before[1][4:, 20:])
    assert torch.equal(parents[2][:, 31:], before[2][:, 31:])


@pytest.mark.parametrize("n", (127, 128, 129, 130, 257))
@pytest.mark.parametrize("many", (40, 700))
def test_short_last_rows(n, many):
    """Tensors whose last 512-byte row is short or taken by the head before the first 16-byte
    boundary, as many as a small list's warps and several to a warp."""
    g = gen(17)
    grads = [make((n,), F32, "odd", g, 1.0 + i) for i in range(many)]
    outs = [torch.empty(n, device=DEV) for _ in grads]
    st = state_like([(n,)] * many, g)
    before = [[x.clone() for x in t] for t in st]
    ts = absnt.GradTensors(grads, out=outs, params=st[0], m=st[1], v=st[2])
    absnt.abs_grad_clip(ts, 1.0)
    total = check_norms(ts, grads, 2)
    for x, y in zip(grads, outs):
        check_scaled(y, x, 1.0 / (total + 1e-6), F32)
    absnt.abs_grad_adamw(ts, HP, 3, 1.0)
    check_norms(ts, grads, 2)
    for i in range(0, many, 13):
        w, m1, v1, e_p, e_m, e_v = adamw_ref(*(b[i].double() for b in before),
                                             grads[i].double() / (total + 1e-6), HP, 3)
        for got, ref, tol in zip((t[i] for t in st), (w, m1, v1), (e_p, e_m, e_v)):
            assert ((got.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("out_dtype", (F32, BF16))
def test_every_alignment(dtype, out_dtype):
    """Gradient, output and state at every distance from a boundary, runs of every length up to a few
    vectors and one beyond a unit; nothing beside the output is touched."""
    g = gen(18)
    room = 32
    sizes = list(range(1, 40)) + [63, 64, 65, 4095, 4097, 40_000]
    for shift in range(8):
        grads, outs, guards, ps = [], [], [], []
        for k, n in enumerate(sizes):
            a, b = (shift + k) % 8, (3 * shift + 5 * k) % 8
            grads.append(make((n + a,), dtype, "dense", g)[a:])
            whole = torch.full((n + b + room,), 7.0, device=DEV, dtype=out_dtype)
            guards.append((whole, b))
            outs.append(whole[b:b + n])
            ps.append([make((n + b,), F32, "dense", g, 0.02)[b:] for _ in range(3)])
        p, m, v = (list(x) for x in zip(*ps))
        for x in v:
            x.copy_(x.square() + 1e-6)
        before = [[x.clone() for x in t] for t in (p, m, v)]
        ts = absnt.GradTensors(grads, out=outs, params=p, m=m, v=v)
        # with a sum given the second pass runs as a kernel of its own, whatever the list's size
        absnt.abs_grad_norm(ts)
        total = check_norms(ts, grads, 2)
        absnt.abs_grad_clip(ts, 1.0, sum_in=ts.header)
        absnt.abs_grad_adamw(ts, HP, 3, 1.0, sum_in=ts.header)
        for i, n in enumerate(sizes):
            check_scaled(outs[i], grads[i], 1.0 / (total + 1e-6), out_dtype)
            whole, b = guards[i]
            assert (whole[:b] == 7).all() and (whole[b + n:] == 7).all()
            w, m1, v1, e_p, e_m, e_v = adamw_ref(*(t[i].double() for t in before),
                                                 grads[i].double() / (total + 1e-6), HP, 3)
            for got, ref, tol in zip((p[i], m[i], v[i]), (w, m1, v1), (e_p, e_m, e_v)):
                assert ((got.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("width", (1, 3, 63, 64, 65, 200, 4099))
@pytest.mark.parametrize("dtype", (F32, BF16))
def test_rows_of_every_width(width, dtype):
    """Column slices whose rows begin at changing distances from a boundary, in place and into a
    dense and a sliced output."""
    g = gen(19)
    rows = max(3, 30_000 // width)
    parent = make((rows, 2 * width + 5), dtype, "dense", g)
    keep = parent.clone()
    grad, ref = parent[:, 3:3 + width], keep[:, 3:3 + width]
    for out in (torch.empty(rows, width, device=DEV),
                torch.empty(rows, width + 3, device=DEV)[:, 1:1 + width], None):
        ts = absnt.GradTensors([grad], out=None if out is None else [out])
        absnt.abs_grad_norm(ts)
        total = check_norms(ts, [ref], 2)
        absnt.abs_grad_clip(ts, 1.0, sum_in=ts.header)
        check_scaled(grad if out is None else out, ref, 1.0 / (total + 1e-6),
                     dtype if out is None else F32)
    assert torch.equal(parent[:, :3], keep[:, :3])
    assert torch.equal(parent[:, 3 + width:], keep[:, 3 + width:])


def adamw_ref(p, m, v, g, hp, step):
    hp = {k: float(torch.tensor(x, dtype=F32)) for k, x in hp.items()}  # the C struct holds floats
    b1, b2 = hp["beta1"], hp["beta2"]
    m1 = b1 * m + (1 - b1) * g
    v1 = b2 * v + (1 - b2) * g * g
    den = (v1 / (1 - b2 ** step)).sqrt() + hp["eps"]
    upd = hp["lr"] / (1 - b1 ** step) * m1 / den
    e_m = 2.0 ** -22 * (m.abs() + g.abs()) + NORM_REL * g.abs()
    e_v = 2.0 ** -21 * (v + g * g) + 2 * NORM_REL * g * g
    e_p = (2.0 ** -22 * (p.abs() + upd.abs()) + 2.0 ** -20 * upd.abs()
           + hp["lr"] / (1 - b1 ** step) * e_m / den)
    return (1 - hp["lr"] * hp["weight_decay"]) * p - upd, m1, v1, e_p, e_m, e_v


def state_like(shapes, g, layout="dense"):
    p = [make(s, F32, layout, g, 0.02) for s in shapes]
    m = [make(s, F32, layout, g, 0.01) for s in shapes]
    v = [make(s, F32, layout, g, 0.01) for s in shapes]
    for x in v:
        x.copy_(x.square() + 1e-6)
    return p, m, v


@pytest.mark.parametrize("layouts", [("dense", "dense"), ("odd", "odd"), ("dense", "odd"),
                                     ("columns", "dense"), ("columns_odd", "odd"),
                                     ("swapped", "swapped"), ("swapped", "dense"),
                                     ("columns", "swapped")])
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("clip", (True, False))
@pytest.mark.parametrize("shapes", (SHAPES[:6] + SHAPES[7:9], SHAPES, SHAPES + [(1500, 1100)]))
def test_adamw(shapes, clip, dtype, layouts):
    """Lists whose update is part of the cluster kernel, whose norm is, and for all SMs."""
    g = gen(8)
    grads = [make(s, dtype, layouts[0], g, 0.1) for s in shapes]
    p, m, v = state_like(shapes, g, layouts[1])
    p16 = [make(s, BF16, layouts[1], g) for s in shapes]
    groups = [i % 3 for i in range(len(shapes))]
    hps = [HP, dict(HP, weight_decay=0.0), dict(HP, lr=3e-4, beta1=0.8)]
    before = [[x.clone() for x in t] for t in (p, m, v, grads)]
    ts = absnt.GradTensors(grads, params=p, m=m, v=v, params_bf16=p16, groups=groups)
    step = 7
    absnt.abs_grad_adamw(ts, hps, step, 1.0 if clip else 0.0, grad_scale=0.5)
    factor = 0.5
    if clip:
        total = check_norms(ts, grads, 2, 0.5)
        factor *= 1.0 / (total + 1e-6)
        assert total > 2.0
    for i, k in enumerate(groups):
        p0, m0, v0, g0 = (b[i].double() for b in before)
        w, m1, v1, e_p, e_m, e_v = adamw_ref(p0, m0, v0, g0 * factor, hps[k], step)
        assert ((m[i].double() - m1).abs() <= e_m).all()
        assert ((v[i].double() - v1).abs() <= e_v).all()
        assert ((p[i].double() - w).abs() <= e_p).all()
        assert torch.equal(p16[i], p[i].to(BF16))
        assert torch.equal(grads[i], before[3][i])


@pytest.mark.parametrize("width", (1, 15, 16, 17, 24, 31, 64, 100, 513, 4100))
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("layout", ("dense", "odd"))
def test_adamw_rows_of_every_width(width, dtype, layout):
    """Column slices at every distance from a boundary, the first and last columns among them; what
    lies between their rows is NaN."""
    g = gen(width)
    rows, grads = 40_000 // width, []
    for gap in (1, 3, 8, 16):
        for at in (0, gap):
            parent = torch.full((rows, width + gap), math.nan, device=DEV, dtype=dtype)
            grads.append(parent[:, at:at + width])
            grads[-1].copy_(torch.randn(rows, width, device=DEV, generator=g) * 0.1)
    p, m, v = state_like([x.shape for x in grads], g, layout)
    half = [torch.empty(x.shape, device=DEV, dtype=BF16) for x in grads]
    ref = [[x.double() for x in t] for t in (p, m, v)]
    each = [adamw_ref(*z, x.double(), HP, 5) for *z, x in zip(*ref, grads)]
    ts = absnt.GradTensors(grads, params=p, m=m, v=v, params_bf16=half)
    absnt.abs_grad_adamw(ts, HP, 5)
    for (rp, rm, rv, e_p, e_m, e_v), x, y, z, h in zip(each, p, m, v, half):
        assert ((x.double() - rp).abs() <= e_p).all()
        assert ((y.double() - rm).abs() <= e_m).all()
        assert ((z.double() - rv).abs() <= e_v).all()
        assert torch.equal(h, x.to(BF16))


@pytest.mark.parametrize("blocks", range(1, 17))
def test_cluster_of_every_size(blocks):
    """Lists that fill 1 to 16 blocks of a cluster (8192 bytes each), with tensors that lie in one block,
    reach into the next one, and go through all of them: each norm, and what every block makes of the
    sum."""
    g = gen(100 + blocks)
    n = 2048 * blocks
    for sizes in ((n,), (5, n - 5), (n - 5, 5), (n // 3, n // 3, n - 2 * (n // 3)), (700,) * (n // 700),
                  (3, n - 2003, 1000, 1000)):
        grads = [make((k,), F32, "dense", g, 0.1 * (i + 1)) for i, k in enumerate(sizes)]
        before = [x.clone() for x in grads]
        st = state_like([(k,) for k in sizes], g)
        ref = [[x.double() for x in t] for t in st]
        ts = absnt.GradTensors(grads, params=st[0], m=st[1], v=st[2])
        for order in ORDERS:
            absnt.abs_grad_norm(ts, norm_type=order)
            check_norms(ts, grads, order)
        absnt.abs_grad_adamw(ts, HP, 3, 0.5)
        total = check_norms(ts, grads, 2)
        factor = 0.5 / (total + 1e-6)
        for i, x in enumerate(before):
            w, m1, v1, e_p, e_m, e_v = adamw_ref(*(t[i] for t in ref), x.double() * factor, HP, 3)
            for got, want, tol in zip((t[i] for t in st), (w, m1, v1), (e_p, e_m, e_v)):
                assert ((got.double() - want).abs() <= tol).all()
        absnt.abs_grad_clip(ts, 0.5)
        check_norms(ts, before, 2)
        for x, b in zip(grads, before):
            check_scaled(x, b, factor, F32)


def test_adamw_is_the_flat_call():
    """On one dense fp32 tensor, without clipping: the update of abs_adamw_step, bit for bit."""
    g = gen(9)
    n = 300_001
    grad = torch.randn(n, device=DEV, generator=g) * 0.01
    p, m, v = (t[0] for t in state_like([(n,)], g))
    q = [t.clone() for t in (p, m, v)]
    ts = absnt.GradTensors([grad], params=[p], m=[m], v=[v])
    for step in (1, 2):
        absnt.abs_grad_adamw(ts, HP, step)
        absnt.abs_adamw_step(q[0], grad, q[1], q[2], HP, step)
    assert all(torch.equal(a, b) for a, b in zip((p, m, v), q))


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("order", (2, 1))
@pytest.mark.parametrize("size", (1e-42, 1e-30, 1e-21, 1e25, 1e37))
@pytest.mark.parametrize("more", ([], [(1_700_000,)]))
def test_range(more, size, order, dtype):
    """Squares and sums that leave the range of fp32: the norm is still that of the values."""
    g = gen(10)
    grads = [(torch.randn(s, device=DEV, generator=g).clamp(-3, 3) * size).to(dtype)
             for s in [(5,), (300, 70), (50_000,)] + more]
    grads.append(torch.randn(1000, device=DEV, generator=g))  # one of ordinary size
    ts = absnt.GradTensors(grads)
    absnt.abs_grad_norm(ts, norm_type=order, max_norm=1.0)
    total, each = ref_norms(grads, order, 1.0)
    fits = each < 3.4e38
    err = (ts.norms.double() - each).abs()
    assert (err[fits] <= NORM_REL * each[fits] + 2.0 ** -149).all()
    assert torch.isinf(ts.norms[~fits]).all()
    assert abs(float(ts.header[absnt.ABS_GRAD_NORM]) - float(total)) <= NORM_REL * float(total)
    assert float(ts.header[absnt.ABS_GRAD_FLAGS]) == 0.0
    coef = min(1.0, 1.0 / (float(total) + 1e-6))
    assert abs(float(ts.coef) - coef) <= 2 * NORM_REL * coef + 2.0 ** -149


def test_zeros_and_negative_zeros():
    grads = [torch.zeros(100_000, device=DEV), -torch.zeros(70_000, device=DEV, dtype=BF16)]
    ts = absnt.GradTensors(grads)
    for order in ORDERS:
        absnt.abs_grad_clip(ts, 1.0, norm_type=order)
        assert float(ts.norm) == 0.0 and float(ts.coef) == 1.0 and not ts.norms.any()


def test_empty_lists():
    ts = absnt.GradTensors([])
    assert float(absnt.abs_grad_norm(ts, max_norm=1.0)) == 0.0 and float(ts.coef) == 1.0
    assert ts.norms.numel() == 0
    empty = [torch.empty(0, device=DEV), torch.empty(3, 0, device=DEV, dtype=BF16)]
    ts = absnt.GradTensors(empty, params=[torch.empty_like(x, dtype=F32) for x in empty],
                           m=[torch.empty_like(x, dtype=F32) for x in empty],
                           v=[torch.empty_like(x, dtype=F32) for x in empty])
    for order in ORDERS:
        absnt.abs_grad_clip(ts, 1.0, norm_type=order)
        absnt.abs_grad_adamw(ts, HP, 1, 1.0, norm_type=order)
        assert float(ts.norm) == 0.0 and float(ts.coef) == 1.0 and not ts.norms.any()


@pytest.mark.parametrize("bad", (math.nan, math.inf, -math.inf))
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("more", MORE)
def test_not_finite(more, dtype, order, bad):
    """One such value: the flag is raised, nothing is clipped, AdamW leaves its state alone; the next
    call on mended gradients is an ordinary one."""
    g = gen(11)
    shapes = [(1000,), (70_001,), (30, 30)] + more
    grads = [make(s, dtype, "dense", g) for s in shapes]
    p, m, v = state_like(shapes, g)
    before = [[x.clone() for x in t] for t in (grads, p, m, v)]
    at = 65_536 + 777
    grads[1][at] = bad
    ts = absnt.GradTensors(grads, params=p, m=m, v=v)
    absnt.abs_grad_clip(ts, 0.5, norm_type=order)
    absnt.abs_grad_adamw(ts, HP, 3, 0.5, norm_type=order)
    assert not math.isfinite(float(ts.norm)) and math.isnan(float(ts.norm)) == math.isnan(bad)
    assert float(ts.coef) == 1.0
    assert float(ts.header[absnt.ABS_GRAD_FLAGS]) == binding.ABS_FLAG_NONFINITE
    assert math.isfinite(float(ts.norms[0])) and math.isfinite(float(ts.norms[2]))
    grads[1][at] = before[0][1][at]
    for now, then in zip((grads, p, m, v), before):
        assert all(torch.equal(a, b) for a, b in zip(now, then))
    absnt.abs_grad_adamw(ts, HP, 3, 0.5, norm_type=order)
    check_norms(ts, grads, order)
    assert not torch.equal(p[1], before[1][1])


def test_same_bits_every_time():
    g = gen(12)
    grads = [make((n,), (F32, BF16)[i % 2], "odd", g) for i, n in enumerate((5_000_001, 77, 900_000, 2_000_003))]
    ts = absnt.GradTensors(grads)
    for order in ORDERS:
        seen = set()
        for _ in range(20):
            absnt.abs_grad_norm(ts, norm_type=order)
            seen.add((tuple(ts.norms.tolist()), tuple(ts.header.tolist()[:3])))
        assert len(seen) == 1


@pytest.mark.parametrize("order", ORDERS)
def test_sum_from_elsewhere(order):
    """Two lists whose power sums are joined as two ranks would: both clip by the joint norm."""
    g = gen(13)
    parts = [[make((3000,), BF16, "dense", g)], [make((100, 90), F32, "odd", g), make((11,), F32, "dense", g)]]
    before = [[x.clone() for x in part] for part in parts]
    sets = [absnt.GradTensors(part) for part in parts]
    for ts in sets:
        absnt.abs_grad_norm(ts, norm_type=order)
    sums = torch.stack([ts.header[absnt.ABS_GRAD_SUM] for ts in sets])
    joint = sums.max() if order == math.inf else sums.sum()
    total = float(ref_norms(before[0] + before[1], order, 1.0)[0])
    for ts, part, b in zip(sets, parts, before):
        own = ts.norms.clone()
        ts.header[absnt.ABS_GRAD_SUM] = joint  # the header itself may carry it
        absnt.abs_grad_clip(ts, 0.25, norm_type=order, sum_in=ts.header)
        assert abs(float(ts.norm) - total) <= NORM_REL * total
        assert torch.equal(own, ts.norms)
        for x, y in zip(part, b):
            check_scaled(x, y, 0.25 / (total + 1e-6), x.dtype)


def test_sum_for_the_flat_calls():
    """The header's SUM is where abs_adamw_step_clipped looks for the squared norm."""
    g = gen(14)
    n = 50_000
    flat = torch.randn(n, device=DEV, generator=g)
    p, m, v = (t[0] for t in state_like([(n,)], g))
    q = [t.clone() for t in (p, m, v)]
    ts = absnt.GradTensors([flat[:20_000], flat[20_000:]])
    absnt.abs_grad_norm(ts)
    absnt.abs_adamw_step_clipped(p, flat, m, v, HP, 5, 1.0, ts.header)
    total = float(ref_norms([flat], 2, 1.0)[0])
    w, m1, v1, e_p, e_m, e_v = adamw_ref(*(t.double() for t in (*q, flat / (total + 1e-6))), HP, 5)
    assert ((m.double() - m1).abs() <= e_m + 2.0 ** -22 * m1.abs()).all()
    assert ((p.double() - w).abs() <= 2 * e_p).all()


@pytest.mark.parametrize("more", MORE)
def test_other_streams_and_graphs(more):
    g = gen(15)
    shapes = [(100, 100), (33_333,)] + more
    grads = [make(s, BF16, "dense", g, 0.1) for s in shapes]
    p, m, v = state_like(shapes, g)
    q = [[x.clone() for x in t] for t in (p, m, v)]
    ts = absnt.GradTensors(grads, params=p, m=m, v=v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        absnt.abs_grad_adamw(ts, HP, 1, 1.0)
    absnt.abs_grad_adamw(ts, HP, 2, 1.0, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        absnt.abs_grad_adamw(ts, HP, 3, 1.0)
        absnt.abs_grad_clip(ts, 1.0)
    then = [x.clone() for x in grads]
    graph.replay()
    torch.cuda.synchronize()
    rs = absnt.GradTensors(then, params=q[0], m=q[1], v=q[2])
    for step in (1, 2, 3):
        absnt.abs_grad_adamw(rs, HP, step, 1.0)
    absnt.abs_grad_clip(rs, 1.0)
    for a, b in zip((p, m, v, grads), (*q, then)):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("columns", (1, 2))
@pytest.mark.parametrize("more", ([], [(2_000_000,)]))
def test_far_apart_rows(more, columns):
    """Views whose rows lie so far apart that offsets within one unit pass 31 bits."""
    g = gen(20)
    rows, pitch = 40_000, 70_000
    parent = torch.zeros(rows, pitch, device=DEV, dtype=BF16)
    target = torch.zeros(rows, pitch, device=DEV, dtype=BF16)
    at = slice(pitch - 7, pitch - 7 + columns)
    view = parent[:, at]
    view.copy_(torch.randn(rows, columns, device=DEV, generator=g))
    rest = [make(s, F32, "dense", g, 0.01) for s in more]
    before = [x.clone() for x in [view] + rest]
    p, m, v = state_like([x.shape for x in before], g)
    st = [[x.clone() for x in t] for t in (p, m, v)]
    ts = absnt.GradTensors([view] + rest, out=[target[:, at]] + [torch.empty_like(x) for x in rest],
                           params=p, m=m, v=v)
    for order in ORDERS:
        absnt.abs_grad_norm(ts, norm_type=order)
        check_norms(ts, before, order)
    for sums in (None, ts.header):
        absnt.abs_grad_norm(ts)
        absnt.abs_grad_clip(ts, 1.0, sum_in=sums)
        total = check_norms(ts, before, 2)
        check_scaled(target[:, at], before[0], 1.0 / (total + 1e-6), BF16)
        assert int(torch.count_nonzero(target)) == int(torch.count_nonzero(target[:, at]))
        target.zero_()
    absnt.abs_grad_adamw(ts, HP, 3, 1.0)
    w, m1, v1, e_p, e_m, e_v = adamw_ref(*(t[0].double() for t in st),
                                         before[0].double() / (total + 1e-6), HP, 3)
    for got, ref, tol in zip((p[0], m[0], v[0]), (w, m1, v1), (e_p, e_m, e_v)):
        assert ((got.double() - ref).abs() <= tol).all()
    del target
    ts = absnt.GradTensors([view] + rest)  # in place
    absnt.abs_grad_clip(ts, 1.0)
    check_scaled(view, before[0], 1.0 / (total + 1e-6), BF16)
    assert int(torch.count_nonzero(parent)) == int(torch.count_nonzero(view))


def test_beyond_32_bits():
    """A tensor of more than 2^32 elements, and one after it."""
    n = (1 << 32) + 70_001
    big = torch.zeros(n, device=DEV, dtype=BF16)
    at = [0, 12_345, (1 << 31) - 1, 1 << 31, (1 << 32) - 1, 1 << 32, (1 << 32) + 5, n - 1]
    for i, a in enumerate(at):
        big[a] = float(i + 1)
    last = torch.full((9,), 2.0, device=DEV)
    ts = absnt.GradTensors([big, last])
    absnt.abs_grad_norm(ts, norm_type=1)
    assert float(ts.norm) == 36.0 + 18.0 and ts.norms.tolist() == [36.0, 18.0]
    absnt.abs_grad_clip(ts, 27.0, norm_type=1)
    assert [float(big[a]) for a in at] == [0.5 * (i + 1) for i in range(len(at))]
    assert int(torch.count_nonzero(big[:1 << 31])) == 3
    assert torch.equal(last, torch.ones_like(last))
    wide = big[:(1 << 32)].view(1 << 16, 1 << 16)[:, 1:60_001]  # rows that begin beyond 2^31
    ts = absnt.GradTensors([wide])
    absnt.abs_grad_norm(ts, norm_type=math.inf)
    assert float(ts.norm) == 1.0  # 12,345: half of 2; the others lie outside the columns


# ------------------------------------------------------------------------------------ refusals
def test_refusals():
    a = torch.zeros(100, 64, device=DEV)
    ok = [torch.zeros(5, device=DEV)]
    with pytest.raises(TypeError):
        absnt.GradTensors([a.double()])
    with pytest.raises(TypeError):
        absnt.GradTensors([torch.zeros(4, 1, device=DEV).expand(4, 3)])
    with pytest.raises(TypeError):
        absnt.GradTensors([torch.zeros(4, 5, 6, device=DEV)[:, :3, :2]])
    with pytest.raises(ValueError):
        absnt.GradTensors([torch.zeros(5)])  # not on the device
    with pytest.raises(ValueError):
        absnt.GradTensors(ok, out=[])
    with pytest.raises(ValueError):
        absnt.GradTensors(ok, out=[torch.zeros(1, 5, device=DEV)])
    with pytest.raises(ValueError):
        absnt.GradTensors(ok, params=[ok[0].clone()])
    with pytest.raises(ValueError):
        absnt.GradTensors(ok, groups=[16])
    with pytest.raises(TypeError):  # state of another type, or not dense in the gradient's order
        absnt.GradTensors(ok, params=[ok[0].bfloat16()], m=[ok[0].clone()], v=[ok[0].clone()])
    sw = a.t().contiguous().t()
    with pytest.raises(TypeError):
        absnt.GradTensors([a], params=[sw], m=[a.clone()], v=[a.clone()])
    with pytest.raises(TypeError):
        absnt.GradTensors([a], params=[a[:, ::2].new_zeros(100, 128)[:, ::2]], m=[a.clone()], v=[a.clone()])

    def status(f):
        with pytest.raises(absnt.AbsError) as e:
            f()
        return e.value.status

    flat = torch.zeros(100, device=DEV)
    assert status(lambda: absnt.GradTensors([flat[:50]], out=[flat[49:99]])) == binding.ABS_ERR_ALIAS
    assert status(lambda: absnt.GradTensors(ok, params=[flat[:5]], m=[flat[4:9]], v=[flat[20:25]])) == binding.ABS_ERR_ALIAS
    twice = absnt.GradTensors([flat[:60], flat[50:]])
    absnt.abs_grad_norm(twice)  # reading is fine
    assert status(lambda: absnt.abs_grad_clip(twice, 1.0)) == binding.ABS_ERR_ALIAS
    ts = absnt.GradTensors(ok)
    for bad in (0.0, -1.0, math.inf, math.nan):
        assert status(lambda: absnt.abs_grad_clip(ts, bad)) == binding.ABS_ERR_RANGE
    for bad in (0.0, math.inf, math.nan):
        assert status(lambda: absnt.abs_grad_norm(ts, grad_scale=bad)) == binding.ABS_ERR_RANGE
    assert status(lambda: absnt.abs_grad_adamw(ts, HP, 1)) == binding.ABS_ERR_NULL  # no state given
    with pytest.raises(ValueError):
        absnt.abs_grad_norm(ts, norm_type=3)
    with pytest.raises(TypeError):
        absnt.abs_grad_clip(ts, 1.0, sum_in=torch.zeros(1, device=DEV))
    st = [torch.zeros(5, device=DEV) for _ in range(3)]
    ts = absnt.GradTensors(ok, params=st[:1], m=st[1:2], v=st[2:], groups=[2])
    with pytest.raises(ValueError):
        absnt.abs_grad_adamw(ts, [HP, HP], 1)
    assert status(lambda: absnt.abs_grad_adamw(ts, [HP] * 3, 0)) == binding.ABS_ERR_RANGE
    assert status(lambda: absnt.abs_grad_adamw(ts, [HP, HP, dict(HP, beta1=1.0)], 1)) == binding.ABS_ERR_RANGE
