"""The Python side of the calls over a list of tensors, without a device: torch.cuda is replaced by a
model of it with numbered streams."""

import collections

import numpy as np
import pytest
import torch

from paper_2412_21124_b200 import binding, dist


class Stream:
    """A stream that writes down what is asked of it.  As in torch, a stream made for the number 0 is
    not the default stream but one out of a pool."""
    pool = 9000

    def __init__(self, number):
        self.cuda_stream, self.waits, self.capturing = number, [], False

    def wait_event(self, event):
        assert not self.capturing, "an event from outside would end the capture"
        self.waits.append(event)


class Cuda:
    """The parts of torch.cuda that a call uses."""

    def __init__(self):
        self.default = Stream(0)
        self.current = self.default
        self.external = {}

    def make_external(self, number, device=None):
        if number == 0:
            Stream.pool += 1
            return Stream(Stream.pool)
        return self.external.setdefault(number, Stream(number))

    def stream(self, s):
        cuda = self

        class Context:
            def __enter__(self):
                self.before, cuda.current = cuda.current, s

            def __exit__(self, *_):
                cuda.current = self.before
        return Context()


class Buffer:
    def __init__(self):
        self.recorded = []

    def record_stream(self, s):
        self.recorded.append(s)


@pytest.fixture
def cuda(monkeypatch):
    c = Cuda()
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", c.make_external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: c.default)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: c.current)
    monkeypatch.setattr(torch.cuda, "stream", c.stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: c.current.capturing)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: c.current.cuda_stream,
                        raising=False)
    return c


def tensors(uploaded_on=0, **more):
    """A GradTensors as its construction on the stream of that number leaves it, with no tensors."""
    ts = object.__new__(binding.GradTensors)
    fields = dict(_device=0, _uploaded_on=uploaded_on, _uploaded=object(), _work=Buffer(),
                  _results=Buffer(), _hparams=None, _hparams_of=None, n_groups=1)
    ts.__dict__.update(fields, **more)
    return ts


def entered(ts, stream, on):
    """The call on `stream` ran on `on`, which waited for the upload and keeps the buffers."""
    number = ts._enter(stream)
    assert number == on.cuda_stream
    assert on.waits == [ts._uploaded]
    assert ts._work.recorded == [on] and ts._results.recorded == [on]


@pytest.mark.parametrize("given", ("nothing", "stream", "number"))
def test_default_stream_waits_for_an_upload_elsewhere(cuda, given):
    ts = tensors(uploaded_on=77)
    entered(ts, {"nothing": None, "stream": cuda.default, "number": 0}[given], cuda.default)


@pytest.mark.parametrize("given", ("nothing", "stream", "number"))
def test_side_stream_waits_for_an_upload_on_the_default_one(cuda, given):
    ts, side = tensors(uploaded_on=0), cuda.make_external(77)
    if given == "nothing":
        cuda.current = side
    entered(ts, {"nothing": None, "stream": side, "number": 77}[given], side)


def test_the_uploading_stream_waits_for_nothing(cuda):
    ts = tensors(uploaded_on=0)
    assert ts._enter(None) == 0 and ts._enter(cuda.default) == 0
    assert not cuda.default.waits and not ts._work.recorded


def test_capture_of_the_given_stream(cuda):
    """No wait for an event from outside goes into a stream that is being captured, whatever stream is
    the current one."""
    ts, side = tensors(uploaded_on=0), cuda.make_external(77)
    side.capturing = True
    for stream in (side, 77):
        assert ts._enter(stream) == 77
    assert not side.waits and cuda.current is cuda.default


def test_capture_of_another_stream(cuda):
    """A given stream that is not captured waits, though the current one is being captured."""
    ts, side, captured = tensors(uploaded_on=0), cuda.make_external(77), cuda.make_external(78)
    captured.capturing = True
    cuda.current = captured
    entered(ts, side, side)
    assert cuda.current is captured and not captured.waits


HP = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)


def lrs(ts, hparams):
    return [pytest.approx(h.lr, rel=1e-6) for h in ts._groups(hparams)]


@pytest.mark.parametrize("scalar", (lambda: torch.tensor(1e-3), lambda: np.array(1e-3)))
@pytest.mark.parametrize("form", (lambda hp: hp, lambda hp: [hp], lambda hp: (hp,)))
def test_a_learning_rate_that_is_changed_in_place(scalar, form):
    ts, lr = tensors(), scalar()
    hparams = form(dict(HP, lr=lr))
    assert lrs(ts, hparams) == [1e-3]
    lr *= 0.1
    assert lrs(ts, hparams) == [1e-4]


def test_hparams_that_change():
    ts = tensors(n_groups=2)
    hp = dict(HP)
    assert lrs(ts, hp) == [1e-3, 1e-3]
    hp["lr"] = 2e-3
    assert lrs(ts, hp) == [2e-3, 2e-3]
    pair = [hp, dict(HP)]
    assert lrs(ts, pair) == [2e-3, 1e-3]
    pair[1]["lr"] = 3e-3
    assert lrs(ts, pair) == [2e-3, 3e-3]
    struct = binding.abs_adamw_hparams(4e-3, 0.9, 0.999, 1e-8, 0.1)
    assert lrs(ts, struct) == [4e-3, 4e-3]
    struct.lr = 5e-3
    assert lrs(ts, struct) == [5e-3, 5e-3]
    kept = ts._groups(pair)
    assert ts._groups([dict(h) for h in pair]) is kept  # the same values: not converted again


def test_hparams_in_a_named_tuple():
    Pair = collections.namedtuple("Pair", "matrices vectors")
    assert lrs(tensors(n_groups=2), Pair(HP, dict(HP, lr=2e-3))) == [1e-3, 2e-3]


def test_no_hparams_after_others():
    """None is refused, not taken for those of the call before."""
    ts = tensors()
    for before in (binding.abs_adamw_hparams(1e-3, 0.9, 0.999, 1e-8, 0.1), HP):
        ts._groups(before)
        with pytest.raises(TypeError):
            ts._groups(None)


class Library:
    """The three launching calls, always answering ABS_OK; writes down which were made."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        return lambda *arguments: self.made.append(name) or 0


@pytest.fixture
def library(monkeypatch):
    calls = Library()
    monkeypatch.setattr(binding, "_lib", calls)
    return calls


def test_adamw_without_clipping_returns_no_norm(cuda, library):
    """No norm is computed then: what the object holds is that of an earlier call, or nothing at all."""
    ts = tensors(norm=object(), _plan_ptr=0, _work_ptr=0, _results_ptr=0)
    assert binding.abs_grad_adamw(ts, HP, 1) is None
    assert binding.abs_grad_adamw(ts, HP, 1, max_norm=1.0) is ts.norm
    assert library.made == ["abs_grad_adamw"] * 2


def test_sharded_adamw_without_clipping(cuda, library, monkeypatch):
    """Over ranks too: no norm, nothing exchanged."""
    monkeypatch.setattr(dist.dist, "is_initialized", lambda: True)
    monkeypatch.setattr(dist.dist, "get_world_size", lambda group=None: 2)
    ts = tensors(norm=object(), header=torch.zeros(8, dtype=torch.float64), _plan_ptr=0, _work_ptr=0,
                 _results_ptr=0)
    monkeypatch.setattr(dist, "join_power_sums", None)  # not to be called
    assert dist.sharded_grad_adamw(ts, HP, 1, 0.0) is None
    assert library.made == ["abs_grad_adamw"]


class Sum:
    """A float64 tensor on a CUDA device."""
    is_cuda, dtype = True, torch.float64

    def __init__(self, index):
        self.device = torch.device("cuda", index)

    def numel(self):
        return 1

    def data_ptr(self):
        return 4096


def test_a_sum_on_another_device(cuda, library, monkeypatch):
    """Its address means nothing to the kernels of this one."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    ts = tensors(norm=object(), _plan_ptr=0, _work_ptr=0, _results_ptr=0)
    for call in (lambda s: binding.abs_grad_clip(ts, 1.0, sum_in=s),
                 lambda s: binding.abs_grad_adamw(ts, HP, 1, 1.0, sum_in=s)):
        with pytest.raises(ValueError):
            call(Sum(1))
        assert call(Sum(0)) is ts.norm
    assert library.made == ["abs_grad_clip", "abs_grad_adamw"]
