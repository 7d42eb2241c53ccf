"""abs_distill_loss against a plain implementation in fp64.

Tolerances, from the arithmetic (e = 2^-24): an exponential 2^a is off by 4 e of itself for its approximation and by
ln 2 |a| 3 e for the roundings of a (a difference, a factor and their product).  A thread adds at most 256 of
them here one after the other, lanes, warps and blocks join in 16 more steps of two exponentials, so a sum of exponentials
is off by at most 400 e of itself, plus 3 |a| e of each of its terms; the logarithms and products of a loss add 8 e of their
sizes, and the teacher's mass outside of its top, 1 - sum p, is off by 60 e.  The approximate exponential gives 0 for
results below 2^-126, the smallest normal float: q_i, an exponential over a sum that is at least 1, and its share of
the rest may each lose that much, so their difference 2^-125 of the row's factor."""
import math

import pytest
import torch

import paper_2412_21124_b200 as absnt

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
E = 2.0 ** -24
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
STEP = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def table(lengths, first=0):
    return torch.tensor([0] + list(lengths), device=DEV).cumsum(0).add(first).to(torch.int32)


def make(rows, vocab, top, dtype, g, layout="dense", t_dtype=F32, sure=6.0):
    z = torch.randn(rows, vocab, device=DEV, generator=g) * 2
    ids = torch.rand(rows, vocab, device=DEV, generator=g).argsort(-1)[:, :top].contiguous()
    t = torch.randn(rows, top, device=DEV, generator=g) * 2 + sure
    z.scatter_add_(1, ids, t)
    if layout == "dense":
        out = torch.empty(rows, vocab, device=DEV, dtype=dtype)
    elif layout == "odd":
        out = torch.empty(rows * vocab + 1, device=DEV, dtype=dtype)[1:].view(rows, vocab)
    else:  # a vocabulary padded to a multiple of 64, and then some
        out = torch.empty(rows, (vocab + 63) // 64 * 64 + 64, device=DEV, dtype=dtype)[:, :vocab]
    out.copy_(z)
    return out, ids, t.to(t_dtype)


def plain(z, ids, t, tau=1.0, lse=None, weights=None, scale=1.0):
    """losses, gradient and the sizes that their errors are measured against"""
    rows, vocab = z.shape
    z, t = z.double() / tau, t.double() / tau
    named = (ids >= 0) & (ids < vocab)
    t = t.masked_fill(~named, -math.inf)
    at = ids.clamp(0, vocab - 1)
    inside = torch.zeros(rows, vocab + 1, device=DEV, dtype=torch.bool)
    inside = inside.scatter_(1, torch.where(named, ids, vocab), True)[:, :vocab]
    log_q = torch.log_softmax(z, -1)
    log_p = t - lse.double()[:, None] if lse is not None else torch.log_softmax(t, -1)
    log_p = log_p.masked_fill(t == -math.inf, -math.inf)  # no entry at all: none has a probability
    p = log_p.exp()
    some = p > 0
    each = torch.where(some, p * (log_p - log_q.gather(1, at)), 0.0)
    sizes = torch.where(some, p * (log_p.abs() + log_q.gather(1, at).abs() + 1), 0.0)
    losses, size = each.sum(-1), sizes.sum(-1)
    grad = log_q.exp()
    part = grad.clone()
    if lse is not None:
        rest = (1 - p.sum(-1)).clamp(min=0)
        log_rest = torch.logsumexp(log_q.masked_fill(inside, -math.inf), -1)
        rest = torch.where(log_rest == -math.inf, 0.0, rest)
        losses += torch.where(rest > 0, rest * (rest.log() - log_rest), 0.0)
        size += torch.where(rest > 0, (rest + 0.2) * ((rest.log() - log_rest).abs() + 2), 0.0)
        # q_i / q_r as the softmax over the rest: a difference of their logarithms would lose it for a rest at the
        # type's lowest value, 3e38, where even 64 bits hold no ln of the number of its values
        share = torch.softmax(z.masked_fill(inside, -math.inf), -1).nan_to_num(0.0)
        grad = grad - rest[:, None] * share
        part = part + (rest[:, None] + 0.2) * share
    else:
        grad = torch.where((p.sum(-1) > 0)[:, None], grad, 0.0)
    p_of = torch.zeros_like(grad).scatter_add_(1, at, torch.where(named, p, 0.0))
    p_log = torch.zeros_like(grad).scatter_add_(1, at, torch.where(some, p * log_p.abs(), 0.0))
    a = (z.amax(-1, keepdim=True) - z).clamp(max=1e4) * 1.4427
    err = part * (600 + 4 * a) * E + (p_of * 30 + 8 * p_log) * E + 2.0 ** -125
    w = (weights.double() if weights is not None else torch.ones(rows, device=DEV, dtype=torch.float64))
    f = (w * scale * tau)[:, None]
    losses = torch.where(w == 0, 0.0, losses) * tau ** 2
    return losses, (size * 600 + 30) * E * tau ** 2, torch.where(f == 0, 0.0, (grad - p_of) * f), err * f.abs()


def check(z, ids, t, dz, losses, **more):
    ref, tol, grad, err = plain(z, ids, t, **more)
    bad = (losses.double() - ref).abs() > tol
    assert not bad.any(), (losses[bad][:4], ref[bad][:4], tol[bad][:4])
    if dz is not None:
        bad = (dz.double() - grad).abs() > err + grad.abs() * ROUND[dz.dtype] + STEP[dz.dtype]
        assert not bad.any(), (dz[bad][:4], grad[bad][:4], err[bad][:4], bad.nonzero()[:4])
    return ref, tol


# every kernel and its borders: one block or several a row, one piece or many, any alignment
VOCABS = (1, 2, 7, 8, 100, 1000, 1003, 4096, 4104, 8192, 16384, 16392, 32000, 50257, 65536, 128256, 131072, 131080, 151936)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
def test_over_vocabularies(vocab, dtype):
    g = gen(vocab)
    for k, (rows, top) in enumerate(((1, 1), (6, 20), (31, 100))):
        top = min(top, vocab)
        layout = ("dense", "odd", "padded")[(k + vocab) % 3]
        z, ids, t = make(rows, vocab, top, dtype, g, layout, (F32, BF16, F16)[k])
        weights = torch.rand(rows, device=DEV, generator=g)
        weights[rows // 2:rows // 2 + 1] = 0 if rows > 1 else 1
        scale = 1000.0 if dtype == F16 else 1.0
        for tau, tail in ((1.0, False), (2.0, True), (0.7, True)):
            lse = torch.logsumexp(t.float() / tau, -1) + 0.3 if tail else None
            losses = torch.empty(rows, device=DEV)
            total = torch.empty(1, device=DEV)
            dz = torch.empty_like(z) if layout == "dense" else make(rows, vocab, top, dtype, g, layout)[0]
            args = dict(tau=tau, lse=lse, weights=weights)
            absnt.abs_distill_loss(z, ids, t, losses, tau, teacher_lse=lse, weights=weights, sample_losses_out=total,
                                   dlogits=dz, grad_scale=scale)
            ref, tol = check(z, ids, t, dz, losses, scale=scale, **args)
            assert abs(float(total) - float((ref * weights).sum())) <= float((tol * weights).sum()) + E * abs(float(total)) + 1e-30
            again = torch.empty(rows, device=DEV)
            absnt.abs_distill_loss(z, ids.int(), t, again, tau, teacher_lse=lse, weights=weights)
            check(z, ids, t, None, again, **args)
        same = z.clone()
        absnt.abs_distill_loss(z, ids, t, losses, tau, teacher_lse=lse, weights=weights, dlogits=dz, grad_scale=scale)
        if layout == "dense":  # in place
            absnt.abs_distill_loss(same, ids, t, losses, tau, teacher_lse=lse, weights=weights, dlogits=same, grad_scale=scale)
            assert torch.equal(same, dz)


@pytest.mark.parametrize("vocab,top", ((600, 512), (512, 512), (33, 33), (50257, 512), (128256, 300)))
def test_large_tops(vocab, top):
    g = gen(top)
    z, ids, t = make(9, vocab, top, BF16, g, t_dtype=BF16)
    for lse in (None, torch.logsumexp(t.float(), -1), torch.logsumexp(t.float(), -1) + 1):
        losses, dz = torch.empty(9, device=DEV), torch.empty_like(z)
        absnt.abs_distill_loss(z, ids, t, losses, teacher_lse=lse, dlogits=dz)
        if top == vocab and lse is not None:  # nothing is outside of the top
            assert torch.isfinite(losses).all()
        check(z, ids, t, dz, losses, lse=lse)


@pytest.mark.parametrize("vocab", (40, 5000, 50257, 128256))
@pytest.mark.parametrize("dtype", (F32, BF16))
def test_entries_left_out_and_named_twice(vocab, dtype):
    g = gen(vocab)
    z, ids, t = make(12, vocab, 16, dtype, g)
    ids[1, 5:] = -1
    ids[2, :] = -1                       # a teacher that names nothing
    ids[3, 3] = vocab
    ids[4, 1] = ids[4, 0]                # twice
    ids[5, :] = ids[5, 0]                # sixteen times
    ids[6, 0], ids[6, 9] = vocab - 1, 0
    t[7, :] = -math.inf
    t[8, 4] = -math.inf
    ids[9, 2] = -2 ** 40
    for lse in (None, torch.full((12,), 20.0, device=DEV)):
        losses, dz = torch.empty(12, device=DEV), torch.empty_like(z)
        absnt.abs_distill_loss(z, ids, t, losses, teacher_lse=lse, dlogits=dz)
        check(z, ids, t, dz, losses, lse=lse)
        if lse is None:
            assert (losses[[2, 7]] == 0).all() and (dz[[2, 7]] == 0).all()


@pytest.mark.parametrize("vocab", (64, 1001, 50257, 128256))
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
def test_masked_and_extreme_logits(vocab, dtype):
    g = gen(vocab + 1)
    z, ids, t = make(10, vocab, 8, dtype, g)
    low = torch.finfo(dtype).min
    keep = torch.zeros(10, vocab, dtype=torch.bool, device=DEV).scatter_(1, ids, True)
    z[1] = z[1].masked_fill(~keep[1], -math.inf)   # only the top is left
    z[2] = z[2].masked_fill(~keep[2], low)
    z[3, :vocab // 2] = low
    z[3].scatter_(0, ids[3], torch.ones(8, device=DEV, dtype=dtype))
    z[4] = low                                     # a row of the lowest value: uniform
    z[5] += 10000.0 if dtype != F16 else 1000.0
    z[6, ids[6, 0]] = 2000.0                       # a student that is sure
    z[7] = -z[7].abs() * 100                       # and one that is sure of the wrong
    losses, dz = torch.empty(10, device=DEV), torch.empty_like(z)
    for lse in (None, torch.logsumexp(t, -1) + 0.5):
        absnt.abs_distill_loss(z, ids, t, losses, teacher_lse=lse, dlogits=dz)
        check(z, ids, t, dz, losses, lse=lse)
    # infinities and NaN stay in their rows
    z[0, vocab - 1], z[2, 3], z[8] = math.nan, math.inf, -math.inf
    t[6, 0] = math.nan
    z[3, ids[3, 0]] = -math.inf                    # probability where the student has none
    fine = [1, 4, 5, 7, 9]
    absnt.abs_distill_loss(z, ids, t, losses, dlogits=dz)
    check(z[fine], ids[fine], t[fine], dz[fine], losses[fine])
    assert torch.isnan(losses[[0, 2, 6, 8]]).all() and losses[3] == math.inf
    assert torch.isnan(dz[[0, 2, 8]]).all() and torch.isfinite(dz[3]).all()
    assert torch.isnan(dz[6].gather(0, ids[6]))[0]


def test_samples_and_rows_of_none():
    g = gen(2)
    for vocab, dtype in ((1000, BF16), (50257, BF16), (32000, F16), (200, F32)):
        z, ids, t = make(40, vocab, 10, dtype, g)
        weights = torch.rand(40, device=DEV, generator=g)
        weights[[8, 20]] = 0
        z[:5], z[35:], z[8] = math.nan, math.nan, math.nan  # not read
        losses, each, dz = torch.full((40,), 3.0, device=DEV), torch.empty(4, device=DEV), torch.full_like(z, 3.0)
        offsets = table([1, 0, 20, 9], 5)
        absnt.abs_distill_loss(z, ids, t, losses, weights=weights, offsets=offsets, sample_losses_out=each, dlogits=dz)
        own = torch.arange(5, 35, device=DEV)
        own = own[own != 8]
        ref, tol = check(z[own], ids[own], t[own], dz[own], losses[own], weights=weights[own])
        assert losses[8] == 0 and (dz[8] == 0).all()
        for x in (losses[:5], losses[35:], dz[:5], dz[35:]):
            assert (x == 3).all()
        full, slack = torch.zeros(40, device=DEV, dtype=torch.float64), torch.zeros(40, device=DEV, dtype=torch.float64)
        full[own], slack[own] = ref * weights[own], tol * weights[own]
        ends = offsets.tolist()
        for b, (a, e) in enumerate(zip(ends, ends[1:])):
            assert abs(float(each[b]) - float(full[a:e].sum())) <= float(slack[a:e].sum()) + E * abs(float(each[b])) + 1e-30
        # a table outside of the rows, or one that decreases: nothing outside is touched
        room = torch.full((42, vocab), 3.0, device=DEV, dtype=dtype)
        for bad in ([-5, 3, 100, 2 ** 31 - 1, 60], [30, 20, 10, 5, 2]):
            absnt.abs_distill_loss(z, ids, t, losses, weights=weights, offsets=torch.tensor(bad, dtype=torch.int32, device=DEV),
                                   sample_losses_out=each, dlogits=room[1:41])
        assert (room[0] == 3).all() and (room[41] == 3).all()


def test_no_rows():
    z, ids, t = make(4, 100, 3, BF16, gen(0))
    total = torch.ones(1, device=DEV)
    absnt.abs_distill_loss(z[:0], ids[:0], t[:0], torch.empty(0, device=DEV), sample_losses_out=total, dlogits=z[:0].clone())
    assert total == 0
    each = torch.ones(2, device=DEV)
    absnt.abs_distill_loss(z[:0], ids[:0], t[:0], torch.empty(0, device=DEV), offsets=table([0, 0]), sample_losses_out=each)
    assert (each == 0).all()


def test_gradient_against_differences():
    """Central differences of the definition in fp64, whose own error is far below the tolerance of fp32."""
    g = gen(3)
    z, ids, t = make(2, 50, 6, F32, g, sure=1.0)
    w = torch.tensor([0.5, 2.0], device=DEV)
    for tau, lse in ((1.0, None), (2.0, torch.logsumexp(t / 2.0, -1) + 0.4)):
        dz = torch.empty_like(z)
        absnt.abs_distill_loss(z, ids, t, torch.empty(2, device=DEV), tau, teacher_lse=lse, weights=w, dlogits=dz, grad_scale=3.0)
        for i, j in ((0, int(ids[0, 0])), (0, 7), (1, 49), (1, int(ids[1, 5]))):
            d = torch.zeros(2, 50, dtype=torch.float64, device=DEV)
            d[i, j] = 1e-5
            up, down = (float((plain(z.double() + s * d, ids, t, tau, lse)[0] * w.double()).sum()) for s in (1, -1))
            assert abs(3.0 * (up - down) / 2e-5 - float(dz[i, j])) <= 3e-6


@pytest.mark.parametrize("vocab,top,more", ((50, 6, -0.5), (1000, 20, -0.1), (40, 40, 0.7), (300_000, 6, -0.3)))
def test_gradient_where_the_teachers_mass_is_not_one(vocab, top, more):
    """A log-sum-exp that is too small, and a top that is the whole vocabulary with less mass: what the header says the
    gradient then is beside the loss's derivative, which autograd takes from the definition in fp64."""
    z, ids, t = make(4, vocab, top, F32, gen(vocab), sure=1.0)
    lse = torch.logsumexp(t, -1) + more
    losses, dz = torch.empty(4, device=DEV), torch.empty_like(z)
    absnt.abs_distill_loss(z, ids, t, losses, teacher_lse=lse, dlogits=dz)
    leaf = z.double().requires_grad_()
    log_q = torch.log_softmax(leaf, -1)
    log_p = t.double() - lse.double()[:, None]
    loss = (log_p.exp() * (log_p - log_q.gather(1, ids))).sum(-1)
    derivative, = torch.autograd.grad(loss.sum(), leaf)
    mass = log_p.exp().sum(-1, keepdim=True)
    assert (mass > 1.05).all() if more < 0 else (mass < 0.95).all()
    assert ((losses.double() - loss.detach()).abs() <= plain(z, ids, t, lse=lse)[1]).all()
    want, err = derivative + log_q.detach().exp() * (1 - mass), plain(z, ids, t, lse=lse)[3]
    assert ((dz.double() - want).abs() <= err + want.abs() * ROUND[F32] + STEP[F32]).all()


@pytest.mark.parametrize("vocab,rows", ((50257, 300), (32000, 700), (1000, 3000), (4096, 2500), (128256, 150), (151936, 110),
                                        (300000, 20)))
def test_the_same_every_time_on_another_stream_and_in_a_graph(vocab, rows):
    g = gen(4)
    z, ids, t = make(rows, vocab, 20, BF16, g)
    ids[5::7, 3] = ids[5::7, 2]
    lse = torch.logsumexp(t, -1) + 0.2
    weights = torch.rand(rows, device=DEV, generator=g).clamp(min=0.3) - 0.3  # some are zero
    offsets = table([rows // 3, rows - rows // 3])
    losses, each, dz = torch.empty(rows, device=DEV), torch.empty(2, device=DEV), torch.empty_like(z)

    def call():
        absnt.abs_distill_loss(z, ids, t, losses, 2.0, teacher_lse=lse, weights=weights, offsets=offsets, sample_losses_out=each,
                               dlogits=dz)
    call()
    first = [x.clone() for x in (losses, each, dz)]
    check(z, ids, t, dz, losses, tau=2.0, lse=lse, weights=weights)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for x in (losses, each, dz):
            x.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(first, (losses, each, dz)))


def test_rows_far_from_the_first():
    """Logits beyond 2^32 bytes and 2^31 elements from the first."""
    g = gen(5)
    base = torch.empty(72_000 * 32_000, device=DEV, dtype=BF16)
    z = base.view(72_000, 32_000)
    few, ids, t = make(3, 32_000, 5, BF16, g)
    z[-3:] = few
    z[0] = few[0]
    losses = torch.zeros(72_000, device=DEV)
    weights = torch.zeros(72_000, device=DEV)
    weights[0], weights[-3:] = 1, 1
    all_ids, all_t = torch.zeros(72_000, 5, device=DEV, dtype=torch.int64), torch.zeros(72_000, 5, device=DEV)
    all_ids[0], all_ids[-3:], all_t[0], all_t[-3:] = ids[0], ids, t[0], t
    absnt.abs_distill_loss(z, all_ids, all_t, losses, weights=weights, dlogits=z)
    check(few, ids, t, z[-3:].clone(), losses[-3:])
    assert torch.equal(z[0], z[-3]) and (z[1:-3].view(-1)[::1009] == 0).all()


def test_refusals():
    z, ids, t = make(4, 100, 3, BF16, gen(0))
    losses = torch.empty(4, device=DEV)
    f = absnt.abs_distill_loss
    for bad in (dict(temperature=0.0), dict(temperature=float("nan")), dict(grad_scale=float("inf")),
                dict(sample_losses_out=losses[:1]), dict(dlogits=z.float()), dict(weights=losses)):
        with pytest.raises(absnt.AbsError):
            f(z, ids, t, losses, **bad)
    for bad in (dict(dlogits=z[:3]), dict(weights=losses.cpu())):
        with pytest.raises(ValueError):
            f(z, ids, t, losses, **bad)
    with pytest.raises(ValueError):
        f(z, ids, t[:, :2], losses)
    with pytest.raises(TypeError):
        f(z, ids.float(), t, losses)
    with pytest.raises(TypeError):
        f(z, ids, t, losses.double())
    with pytest.raises(TypeError):
        f(z, ids, t, losses, sample_losses_out=torch.empty(2, device=DEV))
    with pytest.raises(TypeError):
        f(z, ids, t, losses, offsets=torch.tensor([0], dtype=torch.int32, device=DEV))
    many = torch.zeros(4, 513, dtype=torch.int64, device=DEV)
    with pytest.raises(absnt.AbsError):
        f(torch.zeros(4, 600, device=DEV), many, many.float(), losses)
    with pytest.raises(absnt.AbsError):
        f(z.t().contiguous().t()[:, :1].expand(4, 100).contiguous()[:, :100], ids, t, losses, dlogits=z[:1].expand(4, 100))
