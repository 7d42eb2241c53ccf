"""abs_rms_norm and abs_rms_norm_grad against plain implementations in fp64.

Tolerances, from the arithmetic (e = 2^-24, half a step of fp32): a thread adds at most 32 squares, lanes and
warps add 10 levels more and every product rounds once, so the sum of squares (all terms positive) is off by at most
44 e of itself, rstd by 22 e and its approximation's 4 e; with the rounding of s, of 1/h and of two products a
normalised value is off by at most 32 e, and by one rounding to its own type.
A gradient: u is off by 32 e, sum g u by 32 e for u and at most 28 e for its additions, of the sum of the absolute
terms; with rstd and the products the two parts of dx are off by 34 e and 128 e of their sizes.
The weight's gradient of the row counts here: at most 128 additions follow one another."""
import pytest
import torch

import paper_2412_21124_b200 as absnt

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
E = 2.0 ** -24
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11, E4M3: 2.0 ** -4, E5M2: 2.0 ** -3}
STEP = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24, E4M3: 2.0 ** -9, E5M2: 2.0 ** -16}
LARGEST = {E4M3: 448.0, E5M2: 57344.0}
EPS = 1e-6
# every kernel: lanes of a row (8, 16, 32), pieces of a thread, blocks; multiples of 8, of 4, odd
WIDTHS = (1, 7, 40, 64, 100, 128, 200, 256, 264, 500, 512, 513, 768, 1000, 1024, 1032, 1537, 2048, 4100, 5000, 8192,
          16383, 16384)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rand(shape, dtype, g, std=1.0, layout="dense"):
    x = torch.randn(shape, device=DEV, generator=g) * std
    if layout == "dense":
        t = torch.empty(shape, device=DEV, dtype=dtype)
    elif layout == "odd":  # rows at odd addresses
        n = x.numel()
        t = torch.empty(n + 3, device=DEV, dtype=dtype)[3:].view(shape)
    else:  # columns of a wider matrix
        t = torch.empty(shape[:-1] + (2 * shape[-1] + 8,), device=DEV, dtype=dtype)[..., 8:8 + shape[-1]]
    t.copy_(x)
    return t


def plain(x, w, residual=None, eps=EPS):
    s = x.double() + (residual.double() if residual is not None else 0.0)
    y = s / (s.square().mean(-1, keepdim=True) + eps).sqrt()
    return s, y * (w.double() if w is not None else 1.0)


def near(got, ref, dtype, rel=32 * E):
    tol = ref.abs() * (rel + ROUND[dtype]) + STEP[dtype]
    bad = (got.double() - ref).abs() > tol
    assert not bad.any(), (got[bad][:4], ref[bad][:4], tol[bad][:4], bad.nonzero()[:4])


def near_scaled(q, scales, y, group):
    """8-bit values with their scales against y."""
    width = y.shape[-1]
    group = group or width
    assert scales.shape == y.shape[:-1] + (-(-width // group),)
    for k, part in enumerate(y.split(group, dim=-1)):
        s = scales[..., k].double()
        want = part.abs().amax(-1) / LARGEST[q.dtype]
        if scales.dtype == F32:
            assert ((s - want).abs() <= 34 * E * want)[want > 2.0 ** -126].all()
        else:
            assert (torch.frexp(s)[0] == 0.5).all()
            some = want > 2.0 ** -127
            assert ((s >= want * (1 - 32 * E)) & (s / 2 < want * (1 + 32 * E)))[some].all()
        assert (s[want == 0] == 1).all()
        got = q[..., k * group:(k + 1) * group].double() * s[..., None]
        tol = part.abs() * (ROUND[q.dtype] + 40 * E) + STEP[q.dtype] / 2 * s[..., None]
        assert ((got - part).abs() <= tol).all()


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
def test_norm_over_widths(width, dtype):
    g = gen(width)
    for rows in (1, 5, 167):
        w = 1 + 0.2 * torch.randn(width, device=DEV, generator=g)
        for k, stream in enumerate((None, dtype, F32)):
            layout = ("dense", "odd", "columns")[(rows + k) % 3]
            x = rand((rows, width), dtype, g, 0.7, layout)
            r = None if stream is None else rand((rows, width), stream, g, 2.0, layout)
            out = torch.empty(rows, width, device=DEV, dtype=dtype)
            s_out = torch.empty_like(r) if r is not None else None
            weight = w.to((dtype, F32, BF16)[k])
            absnt.abs_rms_norm(x, weight, out, EPS, residual=r, sum_out=s_out)
            s, y = plain(x, weight, r)
            near(out, y, dtype)
            if s_out is not None:
                near(s_out, s, stream, 0.0 if stream != F32 else E)


@pytest.mark.parametrize("group", (0, 32, 64, 128))
@pytest.mark.parametrize("width", (1, 33, 64, 100, 128, 260, 512, 1000, 1001, 2048, 4104, 9000, 16384))
@pytest.mark.parametrize("out", (E4M3, E5M2))
def test_norm_in_eight_bits(width, out, group):
    g = gen(width + group)
    groups = -(-width // group) if group else 1
    for dtype, scale_type, rows in ((BF16, F32, 3), (F32, E8M0, 200), (F16, E8M0, 1)):
        x = rand((rows, width), dtype, g)
        r = rand((rows, width), dtype, g, 3.0)
        x[0, :width // 2], r[0, :width // 2] = 0, 0  # groups of zeros
        w = 1 + 0.2 * torch.randn(width, device=DEV, generator=g)
        q = torch.empty(rows, width, device=DEV, dtype=out)
        scales = torch.empty(rows, groups, device=DEV, dtype=scale_type)
        absnt.abs_rms_norm(x, w, q, EPS, residual=r, scales_out=scales, group=group)
        near_scaled(q, scales, plain(x, w, r)[1], group)
        # scales of a product that wants them column by column
        again, turned = torch.empty_like(q), torch.empty(groups, rows, device=DEV, dtype=scale_type).t()
        absnt.abs_rms_norm(x, w, again, EPS, residual=r, scales_out=turned, group=group)
        assert torch.equal(turned.float(), scales.float()) and torch.equal(again.float(), q.float())


@pytest.mark.parametrize("width", (129, 132, 252, 255, 257, 385, 508, 511, 516, 520, 576, 700, 776, 1025, 1535, 1536, 1540, 4096, 4104))
def test_rows_where_the_work_is_dealt_out_another_way(width):
    """Both sides of the widths at which rows go from lanes to blocks and from few values a thread to more."""
    g = gen(width)
    for dtype, rows in ((BF16, 131), (F32, 70), (F16, 1)):
        x, r = rand((rows, width), dtype, g, 0.7), rand((rows, width), F32, g, 2.0)
        w = (1 + 0.2 * torch.randn(width, device=DEV, generator=g)).to(dtype)
        out, s_out = torch.empty_like(x), torch.empty_like(r)
        absnt.abs_rms_norm(x, w, out, EPS)
        near(out, plain(x, w)[1], dtype)
        absnt.abs_rms_norm(x, w, out, EPS, residual=r, sum_out=s_out)
        s, y = plain(x, w, r)
        near(out, y, dtype)
        near(s_out, s, F32, E)
        for group in (0, 32, 64, 128):
            q = torch.empty(rows, width, device=DEV, dtype=E4M3)
            scales = torch.empty(rows, -(-width // group) if group else 1, device=DEV)
            absnt.abs_rms_norm(x, w, q, EPS, residual=r, scales_out=scales, group=group)
            near_scaled(q, scales, y, group)


@pytest.mark.parametrize("width", (64, 80, 100, 128, 99))
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
def test_heads_of_a_fused_projection(width, dtype):
    g = gen(width)
    fused = rand((37, 12, width), dtype, g)
    x, tail = fused[:, 2:7], fused[:, 7:].clone()
    w = rand((width,), dtype, g)
    ref = plain(x, w)[1]
    out = torch.empty(37, 5, width, device=DEV, dtype=dtype)
    absnt.abs_rms_norm(x, w, out, EPS)
    near(out, ref, dtype)
    absnt.abs_rms_norm(x, w, x, EPS)  # in place, among the other heads
    assert torch.equal(x, out) and torch.equal(fused[:, 7:], tail)
    # into other columns of the same matrix
    absnt.abs_rms_norm(fused[:, :5], w, fused[:, 5:10], EPS)
    q = torch.empty(37, 5, width, device=DEV, dtype=E4M3)
    scales = torch.empty(37, 5, 1, device=DEV)
    absnt.abs_rms_norm(fused[:, :5], w, q, EPS, scales_out=scales)
    near_scaled(q, scales, plain(fused[:, :5], w)[1], 0)


def test_inputs_as_outputs_and_broadcast_ones():
    g = gen(1)
    for width in (96, 1000, 1001, 4096):
        x, r = rand((50, width), BF16, g), rand((50, width), BF16, g)
        s, y = plain(x, None, r)
        a, b = x.clone(), r.clone()
        absnt.abs_rms_norm(a, None, a, EPS, residual=b, sum_out=b)
        near(b, s, BF16, 0.0)
        near(a, y, BF16)
        a, b = x.clone(), r.clone()
        absnt.abs_rms_norm(a, None, b, EPS, residual=b, sum_out=a)
        near(a, s, BF16, 0.0)
        near(b, y, BF16)
        one = r[:1].expand(50, width)
        out = torch.empty_like(x)
        absnt.abs_rms_norm(x, None, out, EPS, residual=one)
        near(out, plain(x, None, one)[1], BF16)


@pytest.mark.parametrize("width", (64, 500, 768, 4096, 4097))
def test_rows_at_the_ends_of_the_range(width):
    g = gen(width)
    x = rand((9, width), F32, g)
    x[1] = 0
    x[2] *= 1e30
    x[3] *= 1e-25
    x[4, 0] = 3e38
    x[5, width // 2] = float("inf")
    x[6, width - 1] = float("nan")
    x[7] *= 1e18
    out = torch.empty_like(x)
    absnt.abs_rms_norm(x, None, out, EPS)
    fine = [0, 1, 2, 3, 4, 7, 8]
    near(out[fine], plain(x[fine], None)[1], F32)
    assert (out[1] == 0).all()
    assert torch.isnan(out[5, width // 2]) and (out[5, :width // 2] == 0).all() and torch.isnan(out[6]).all()
    q = torch.empty(9, width, device=DEV, dtype=E4M3)
    for kind in (F32, E8M0):
        scales = torch.empty(9, 1, device=DEV, dtype=kind)
        absnt.abs_rms_norm(x, None, q, EPS, scales_out=scales)
        near_scaled(q[fine], scales[fine], plain(x[fine], None)[1], 0)
        assert torch.isnan(scales.float()[5:7]).all() and torch.isnan(q.float()[5:7]).all()
    dy, dx, dw = rand((9, width), F32, g), torch.empty_like(x), torch.empty(width, device=DEV)
    absnt.abs_rms_norm_grad(dy, x, None, dx, dw, EPS, work=absnt.alloc_rms_norm_work(x))
    check_grad(dx[fine], dy[fine], x[fine], None, None, F32)
    assert torch.isnan(dx[6]).all() and torch.isnan(dw).all()


# ------------------------------------------------------------------------------------------ backward
def plain_grad(dy, s, w, add=None, eps=EPS):
    s, dy = s.double(), dy.double()
    g = dy * (w.double() if w is not None else 1.0)
    rstd = 1 / (s.square().mean(-1, keepdim=True) + eps).sqrt()
    u = s * rstd
    dx = rstd * (g - u * (g * u).mean(-1, keepdim=True))
    size = rstd * (34 * E * g.abs() + 128 * E * u.abs() * (g * u).abs().mean(-1, keepdim=True))
    if add is not None:
        dx, size = dx + add.double(), size + E * add.double().abs()
    return dx, size, dy * u


def check_grad(dx, dy, s, w, add, dtype):
    ref, size, part = plain_grad(dy, s, w, add)
    tol = size + ref.abs() * (ROUND[dtype] + E) + STEP[dtype]
    bad = (dx.double() - ref).abs() > tol
    assert not bad.any(), (dx[bad][:4], ref[bad][:4], bad.nonzero()[:4])
    return part


def check_weight(dw, part, scale=1.0):
    part = part.reshape(-1, part.shape[-1])
    ref, size = part.sum(0) * scale, part.abs().sum(0) * abs(scale)
    assert ((dw.double() - ref).abs() <= (128 + 34) * E * size + 2.0 ** -149).all()


def table(lengths, first=0):
    return torch.tensor([0] + list(lengths), device=DEV).cumsum(0).add(first).to(torch.int32)


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
def test_gradient_over_widths(width, dtype):
    g = gen(width)
    for rows, lengths in ((1, [1]), (5, [0, 2, 0, 3]), (701, [1, 1, 300, 0, 5, 394])):
        for k, stream in enumerate((dtype, F32)):
            layout = ("dense", "odd", "columns")[(rows + k) % 3]
            s = rand((rows, width), stream, g, 2.0, layout)
            dy = rand((rows, width), dtype, g, 1.0, layout)
            add = rand((rows, width), stream, g, 1.0, layout) if k else None
            w = (1 + 0.2 * torch.randn(width, device=DEV, generator=g)).to((F32, BF16)[k])
            dx = torch.empty(rows, width, device=DEV, dtype=(stream, dtype)[k])
            dw = torch.empty(width, device=DEV)
            wide = torch.full((len(lengths), width + 5), 7.0, device=DEV)
            work = absnt.alloc_rms_norm_work(s, len(lengths))
            work.fill_(255)  # NaN: nothing in it is read before it is written
            absnt.abs_rms_norm_grad(dy, s, w, dx, dw, EPS, dresidual=add, offsets=table(lengths),
                                    dweight_samples=wide[:, 2:2 + width], sample_scale=3.0, work=work)
            part = check_grad(dx, dy, s, w, add, dx.dtype)
            check_weight(dw, part)
            for b, p in enumerate(part.split(lengths)):
                check_weight(wide[b, 2:2 + width], p, 3.0)
            assert (wide[:, :2] == 7).all() and (wide[:, 2 + width:] == 7).all()
            # without a table, and the weight's gradient alone or not at all
            again, alone = torch.empty_like(dx), torch.empty_like(dw)
            absnt.abs_rms_norm_grad(dy, s, w, again, alone, EPS, dresidual=add, work=work)
            assert torch.equal(again, dx)
            check_weight(alone, part)
            absnt.abs_rms_norm_grad(dy, s, w, again.fill_(0), None, EPS, dresidual=add)
            assert torch.equal(again, dx)


@pytest.mark.parametrize("width", (64, 100, 128, 99))
def test_gradient_of_heads(width):
    g = gen(width)
    fused = rand((61, 9, width), BF16, g)
    s = fused[:, 2:6]
    dy, w = rand((61, 4, width), BF16, g), rand((width,), F32, g)
    lengths = [20, 1, 0, 40]
    dx, dw = torch.empty(61, 4, width, device=DEV, dtype=BF16), torch.empty(width, device=DEV)
    apart = torch.empty(4, width, device=DEV)
    absnt.abs_rms_norm_grad(dy, s, w, dx, dw, EPS, offsets=table(lengths), dweight_samples=apart,
                            work=absnt.alloc_rms_norm_work(s, 4))
    part = check_grad(dx, dy, s, w, None, BF16)
    check_weight(dw, part)
    for b, p in enumerate(part.split(lengths)):
        check_weight(apart[b], p)


def test_rows_of_no_sample_are_left_alone():
    g = gen(3)
    for width in (64, 1000, 1537, 4096):
        s, dy = rand((90, width), F32, g), rand((90, width), F32, g)
        s[:7], s[70:], dy[:7], dy[70:] = (float("nan"),) * 4  # not read either
        dx, dw = torch.full_like(s, 5.0), torch.empty(width, device=DEV)
        apart = torch.empty(3, width, device=DEV)
        work = absnt.alloc_rms_norm_work(s, 3)
        absnt.abs_rms_norm_grad(dy, s, None, dx, dw, EPS, offsets=table([13, 0, 50], 7), dweight_samples=apart, work=work)
        part = check_grad(dx[7:70], dy[7:70], s[7:70], None, None, F32)
        check_weight(dw, part)
        check_weight(apart[0], part[:13])
        check_weight(apart[2], part[13:])
        assert (apart[1] == 0).all() and (dx[:7] == 5).all() and (dx[70:] == 5).all()
        # no rows in any sample, and no rows at all: sums of zero
        absnt.abs_rms_norm_grad(dy, s, None, dx, dw.fill_(1), EPS, offsets=table([0, 0, 0], 90), dweight_samples=apart.fill_(1),
                                work=work)
        assert (dw == 0).all() and (apart == 0).all() and (dx[:7] == 5).all()
        none = s[:0]
        absnt.abs_rms_norm_grad(none, none, None, none, dw.fill_(1), EPS, offsets=table([0, 0, 0]),
                                dweight_samples=apart.fill_(1))
        assert (dw == 0).all() and (apart == 0).all()
        absnt.abs_rms_norm(none, None, none, EPS)


def test_gradient_into_its_inputs():
    g = gen(4)
    for width in (128, 1000, 1001, 6000):
        s, dy, add = (rand((40, width), BF16, g) for _ in range(3))
        ref = torch.empty_like(s)
        absnt.abs_rms_norm_grad(dy, s, None, ref, None, EPS, dresidual=add)
        for k in range(3):
            t = [dy.clone(), s.clone(), add.clone()]
            absnt.abs_rms_norm_grad(t[0], t[1], None, t[k], None, EPS, dresidual=t[2])
            assert torch.equal(t[k], ref)


def test_gradient_against_differences():
    """The gradients of sum(dy * y) in fp64 by central differences of the definition, at a step where their own
    error (third derivative) is far below the tolerance of fp32."""
    g = gen(5)
    s, dy, w = rand((3, 24), F32, g), rand((3, 24), F32, g), rand((24,), F32, g)
    dx, dw = torch.empty_like(s), torch.empty(24, device=DEV)
    absnt.abs_rms_norm_grad(dy, s, w, dx, dw, EPS, work=absnt.alloc_rms_norm_work(s))

    def loss(s, w):
        return float((dy.double() * s / (s.square().mean(-1, keepdim=True) + EPS).sqrt() * w).sum())

    step = 1e-5
    for i, j in ((0, 0), (1, 23), (2, 7)):
        d = torch.zeros(3, 24, dtype=torch.float64, device=DEV)
        d[i, j] = step
        diff = (loss(s.double() + d, w.double()) - loss(s.double() - d, w.double())) / (2 * step)
        assert abs(diff - float(dx[i, j])) <= 1e-6 * max(1.0, abs(diff))
        d = torch.zeros(24, dtype=torch.float64, device=DEV)
        d[j] = step
        diff = (loss(s.double(), w.double() + d) - loss(s.double(), w.double() - d)) / (2 * step)
        assert abs(diff - float(dw[j])) <= 1e-6 * max(1.0, abs(diff))


def test_results_are_the_same_every_time_and_in_a_graph():
    g = gen(6)
    s, dy, w = rand((5000, 1000), BF16, g), rand((5000, 1000), BF16, g), rand((1000,), BF16, g)
    offsets = table([1000, 1, 2999, 1000])
    work = absnt.alloc_rms_norm_work(s, 4)
    out, dx = torch.empty_like(s), torch.empty_like(s)
    dw, apart = torch.empty(1000, device=DEV), torch.empty(4, 1000, device=DEV)

    def both():
        absnt.abs_rms_norm(s, w, out, EPS)
        absnt.abs_rms_norm_grad(dy, s, w, dx, dw, EPS, offsets=offsets, dweight_samples=apart, work=work)

    both()
    first = [t.clone() for t in (out, dx, dw, apart)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both()
    torch.cuda.current_stream().wait_stream(side)
    for t in (out, dx, dw, apart):
        t.zero_()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(first, (out, dx, dw, apart)))
    offsets.copy_(table([5000, 0, 0, 0]))  # the graph reads the table it finds
    graph.replay()
    assert torch.equal(out, first[0]) and torch.equal(dx, first[1]) and (apart[1:] == 0).all()
    check_weight(apart[0], plain_grad(dy, s, w)[2])


def test_a_table_that_decreases_stays_inside():
    """Wrong numbers, but no access outside of the tensors: everything around them keeps its value."""
    g = gen(7)
    s, dy = rand((64, 256), F32, g), rand((64, 256), F32, g)
    room = torch.full((66, 256), 9.0, device=DEV)
    apart = torch.full((6, 256), 9.0, device=DEV)
    work = absnt.alloc_rms_norm_work(s, 4)
    held = torch.full((work.numel() + 64,), 3, dtype=torch.uint8, device=DEV)
    for bad in ([0, 50, 20, 60, 64], [-5, 10, 2 ** 31 - 1, 3, 64], [64, 0, 64, 0, 64], [10, 5, 5, 5, 200]):
        absnt.abs_rms_norm_grad(dy, s, None, room[1:65], torch.empty(256, device=DEV), EPS,
                                offsets=torch.tensor(bad, dtype=torch.int32, device=DEV), dweight_samples=apart[1:5],
                                work=held[32:32 + work.numel()])
        assert (room[0] == 9).all() and (room[65] == 9).all() and (apart[0] == 9).all() and (apart[5] == 9).all()
        assert (held[:32] == 3).all() and (held[32 + work.numel():] == 3).all()


def test_many_short_samples():
    g = gen(8)
    s, dy = rand((3000, 64), F16, g), rand((3000, 64), F16, g)
    dx, dw, apart = torch.empty_like(s), torch.empty(64, device=DEV), torch.empty(3000, 64, device=DEV)
    absnt.abs_rms_norm_grad(dy, s, None, dx, dw, EPS, offsets=table([1] * 3000), dweight_samples=apart,
                            work=absnt.alloc_rms_norm_work(s, 3000))
    part = check_grad(dx, dy, s, None, None, F16)
    check_weight(dw, part)
    assert ((apart.double() - part).abs() <= 34 * E * part.abs() + 2.0 ** -149).all()


def test_large_offsets():
    """Rows more than 2^31 elements from the first."""
    g = gen(9)
    base = torch.empty(70_000 * 33_000, device=DEV, dtype=BF16)
    x = base.as_strided((70_000, 128), (33_000, 1))
    x.copy_(rand((70_000, 128), BF16, g))
    out, dx, dw = torch.empty(70_000, 128, device=DEV, dtype=BF16), torch.empty(70_000, 128, device=DEV, dtype=BF16), None
    absnt.abs_rms_norm(x, None, out, EPS)
    near(out, plain(x, None)[1], BF16)
    absnt.abs_rms_norm_grad(out, x, None, dx, dw, EPS)
    check_grad(dx, out, x, None, None, BF16)


def test_refusals():
    x = torch.zeros(4, 64, device=DEV)
    out = torch.empty_like(x)
    f = absnt.abs_rms_norm
    with pytest.raises(ValueError):
        f(x, None, out[:3])
    with pytest.raises(ValueError):
        f(x, None, out.cpu())
    with pytest.raises(TypeError):
        f(x.t().contiguous().t(), None, out)
    with pytest.raises(TypeError):
        f(x, torch.ones(63, device=DEV), out)
    with pytest.raises(TypeError):
        f(x.double(), None, out)
    for bad in (dict(eps=0.0), dict(eps=float("nan")), dict(group=32), dict(sum_out=x.clone())):
        with pytest.raises(absnt.AbsError):
            f(x, None, out, **bad)
    with pytest.raises(absnt.AbsError):
        f(x, None, out.to(E4M3))
    with pytest.raises(absnt.AbsError):
        f(x, None, out.to(E4M3), scales_out=torch.empty(4, 4, device=DEV), group=16)
    wide = torch.zeros(2, 20_000, device=DEV)
    with pytest.raises(absnt.AbsError):
        f(wide, None, torch.empty_like(wide))
    flat = torch.zeros(300, device=DEV)
    with pytest.raises(absnt.AbsError):  # shifted by one
        f(flat[:256].view(4, 64), None, flat[1:257].view(4, 64))
    d = absnt.abs_rms_norm_grad
    dw = torch.empty(64, device=DEV)
    work = absnt.alloc_rms_norm_work(x)
    with pytest.raises(absnt.AbsError):
        d(x, x.clone(), None, out, dw)
    with pytest.raises(absnt.AbsError):
        d(x, x.clone(), None, out, dw, work=work[:64])
    with pytest.raises(absnt.AbsError):
        d(x, x.clone(), None, out, dw, work=work, offsets=torch.zeros(9, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        d(x, x.clone(), None, out, dw, work=work, dweight_samples=torch.empty(1, 64, device=DEV))
    with pytest.raises(TypeError):
        d(x, x.clone(), None, out, dw, work=work, offsets=torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(absnt.AbsError):
        d(x.bfloat16(), x.half(), None, out, None)
