"""The comparisons of test_gpu_distill.py and test_gpu_rms_norm.py once more, in a form that a NaN fails.

Those files ask that no difference exceeds its tolerance, which is also true of a NaN; here every difference has to be at
most its tolerance (or both sides the same infinity).  Inputs, references and tolerances are theirs."""
import pytest

import tests.test_gpu_distill as distill
import tests.test_gpu_rms_norm as norm
from tests.test_gpu_distill import BF16, F16, F32

pytestmark = pytest.mark.gpu

E = distill.E


def within(got, ref, tol):
    got = got.double()
    ok = ((got - ref).abs() <= tol) | (got == ref)
    assert ok.all(), (got[~ok][:4], ref[~ok][:4], tol[~ok][:4], (~ok).nonzero()[:4])


def check(z, ids, t, dz, losses, **more):
    ref, tol, grad, err = distill.plain(z, ids, t, **more)
    within(losses, ref, tol)
    if dz is not None:
        within(dz, grad, err + grad.abs() * distill.ROUND[dz.dtype] + distill.STEP[dz.dtype])
    return ref, tol


def near(got, ref, dtype, rel=32 * E):
    within(got, ref, ref.abs() * (rel + norm.ROUND[dtype]) + norm.STEP[dtype])


def check_grad(dx, dy, s, w, add, dtype):
    ref, size, part = norm.plain_grad(dy, s, w, add)
    within(dx, ref, size + ref.abs() * (norm.ROUND[dtype] + E) + norm.STEP[dtype])
    return part


@pytest.fixture(autouse=True)
def _comparisons(monkeypatch):
    monkeypatch.setattr(distill, "check", check)
    monkeypatch.setattr(norm, "near", near)
    monkeypatch.setattr(norm, "check_grad", check_grad)


@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("vocab", distill.VOCABS)
def test_loss_over_vocabularies(vocab, dtype):
    distill.test_over_vocabularies(vocab, dtype)


@pytest.mark.parametrize("vocab,top", ((600, 512), (512, 512), (33, 33), (50257, 512), (128256, 300)))
def test_loss_of_large_tops(vocab, top):
    distill.test_large_tops(vocab, top)


@pytest.mark.parametrize("vocab", (40, 5000, 50257, 128256))
@pytest.mark.parametrize("dtype", (F32, BF16))
def test_loss_with_entries_left_out_and_named_twice(vocab, dtype):
    distill.test_entries_left_out_and_named_twice(vocab, dtype)


@pytest.mark.parametrize("vocab", (64, 1001, 50257, 128256))
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
def test_loss_of_masked_and_extreme_logits(vocab, dtype):
    distill.test_masked_and_extreme_logits(vocab, dtype)


def test_loss_of_samples_and_rows_far_from_the_first():
    distill.test_samples_and_rows_of_none()
    distill.test_rows_far_from_the_first()


@pytest.mark.parametrize("width", norm.WIDTHS)
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
def test_norm_and_gradient_over_widths(width, dtype):
    norm.test_norm_over_widths(width, dtype)
    norm.test_gradient_over_widths(width, dtype)


@pytest.mark.parametrize("width", (129, 255, 257, 511, 520, 776, 1025, 1536, 1540, 4104))
def test_norm_of_rows_where_the_work_is_dealt_out_another_way(width):
    norm.test_rows_where_the_work_is_dealt_out_another_way(width)


@pytest.mark.parametrize("width", (64, 100, 128, 99))
def test_norm_and_gradient_of_heads(width):
    for dtype in (F32, BF16, F16):
        norm.test_heads_of_a_fused_projection(width, dtype)
    norm.test_gradient_of_heads(width)


@pytest.mark.parametrize("width", (64, 500, 768, 4096, 4097))
def test_norm_of_rows_at_the_ends_of_the_range(width):
    norm.test_rows_at_the_ends_of_the_range(width)


def test_norm_in_place_by_samples_and_far_from_the_first():
    norm.test_inputs_as_outputs_and_broadcast_ones()
    norm.test_rows_of_no_sample_are_left_alone()
    norm.test_many_short_samples()
    norm.test_large_offsets()
