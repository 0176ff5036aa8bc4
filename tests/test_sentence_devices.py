"""Which device and stream the binding of the recurrence, the word scores and dropout launches on, with stand-ins for tensors of several GPUs."""
import inspect

import pytest
import torch

from paper_1809_00832_amd import binding
from test_decoder_devices import On, launches, stream_of  # noqa: F401

F32, I32, I64 = torch.float32, torch.int32, torch.int64


@pytest.fixture()
def calls(launches, monkeypatch):  # noqa: F811
    monkeypatch.setattr(binding, "_recur_workspace", lambda r, backward, device: (None, 0))
    monkeypatch.setattr(On, "__getitem__", lambda self, i: self, raising=False)
    monkeypatch.setattr(On, "new_empty", lambda self, shape, dtype=None: On(self.device.index, *shape, dtype=dtype or self.dtype))
    return launches


def recur(d, **change):
    t = dict(g=On(d, 9, 64), x=On(d, 9, 64), off=On(d, 4, dtype=I32), h0=On(d, 3, 64), h=On(d, 9, 64), h_last=On(d, 3, 64))
    t.update(change)
    return lambda **kw: binding.tl_recur(**t, with_tape=True, **kw)


def recur_backward(d, **change):
    t = dict(g=On(d, 9, 64), x=On(d, 9, 64), off=On(d, 4, dtype=I32), tape=On(d, 3, 64), d_h=On(d, 9, 64), d_last=On(d, 3, 64))
    t.update(change)
    return lambda **kw: binding.tl_recur_backward(**t, **kw)


def score(d, **change):
    t = dict(logits=On(d, 5, 100), word=On(d, 5, dtype=I32))
    t.update(change)
    return lambda **kw: binding.tl_score(**t, n_top=3, **kw)


def score_backward(d, **change):
    t = dict(logits=On(d, 5, 100), word=On(d, 5, dtype=I32), stats=On(d, 3, 5), d_logprob=On(d, 5), d_entropy=On(d, 5), d_logits=On(d, 5, 100))
    t.update(change)
    return lambda **kw: binding.tl_score_backward(**t, **kw)


def dropout(d, **change):
    t = dict(x=On(d, 5, 100), numbers=On(d, 2, dtype=I64), residual=On(d, 5, 100), y=On(d, 5, 100))
    t.update(change)
    return lambda **kw: binding.tl_dropout(**t, p=0.1, **kw)


ALL = [recur, recur_backward, score, score_backward, dropout]


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("device", [0, 1])
def test_launches_go_to_the_tensors_device(calls, device, call):
    call(device)()
    call(device)(stream=stream_of(device, 7))
    assert [(d, s) for _, d, s in calls] == [(device, 100 + device), (device, 7)]


@pytest.mark.parametrize("call", ALL)
def test_tensors_of_two_devices_are_refused(calls, call):
    tensors = inspect.getclosurevars(call(0)).nonlocals["t"]     # (every tensor in turn but the first, which says where the call goes)
    for name in list(tensors)[1:]:
        here = tensors[name]
        with pytest.raises(AssertionError):
            call(0, **{name: On(1, *here.shape, dtype=here.dtype)})()
    assert not calls


@pytest.mark.parametrize("call", ALL)
def test_a_stream_of_another_device_is_refused(calls, call):
    with pytest.raises(AssertionError):
        call(0)(stream=stream_of(1, 7))
    assert not calls


@pytest.mark.parametrize("call,change", [(recur, dict(x=On(0, 9, 64, dtype=torch.bfloat16))), (recur, dict(x=On(0, 9, 63))), (recur, dict(off=On(0, 4, dtype=I64))),
                                         (recur, dict(h0=On(0, 2, 64))), (recur, dict(h0=On(0, 3, 64, dtype=torch.bfloat16))), (recur, dict(h=On(0, 8, 64))),
                                         (recur, dict(h_last=On(0, 3, 65))), (recur_backward, dict(tape=On(0, 2, 64))), (recur_backward, dict(d_h=On(0, 9, 64, dtype=torch.float16))),
                                         (recur_backward, dict(d_last=On(0, 9, 64))), (score, dict(word=On(0, 5, dtype=I64))), (score, dict(word=On(0, 4, dtype=I32))),
                                         (score, dict(logits=On(0, 5, 100, dtype=torch.float64))), (score_backward, dict(stats=On(0, 3, 4))),
                                         (score_backward, dict(d_logprob=On(0, 4))), (score_backward, dict(d_logits=On(0, 5, 100, dtype=torch.bfloat16))),
                                         (dropout, dict(numbers=On(0, 2, dtype=I32))), (dropout, dict(numbers=On(0, 3, dtype=I64))), (dropout, dict(residual=On(0, 5, 99))),
                                         (dropout, dict(y=On(0, 5, 100, dtype=torch.float16)))])
def test_shapes_and_types_are_checked(calls, call, change):
    with pytest.raises(AssertionError):
        call(0, **change)()
    assert not calls
