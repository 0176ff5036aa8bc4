"""Which device and stream the binding of the decoder's operators launches on, with stand-ins for tensors of several GPUs."""
import contextlib

import pytest
import torch

from paper_1809_00832_amd import binding


class On:
    """As much of a contiguous CUDA tensor as the binding looks at."""

    is_cuda = True

    def __init__(self, device, *shape, dtype=torch.float32):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", device)

    def get_device(self):
        return self.device.index

    def stride(self, i=None):
        s = [1]
        for n in self.shape[:0:-1]:
            s.insert(0, s[0] * n)
        return tuple(s) if i is None else s[i]

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def new_empty(self, shape):
        return On(self.device.index, *shape, dtype=self.dtype)


@pytest.fixture()
def launches(monkeypatch):
    """What is called, as (entry point, current device, stream): streams are numbers, 100 + device unless another was chosen."""
    seen, now = [], dict(device=0, stream={})

    class Library:
        def __getattr__(self, name):
            def call(*args):
                seen.append((name, now["device"], args[-1]))
                return 0
            return call

    @contextlib.contextmanager
    def use(device, stream=None):
        before = dict(device=now["device"], stream=dict(now["stream"]))
        now["device"] = device
        if stream is not None:
            now["stream"][device] = stream
        yield
        now.update(before)

    monkeypatch.setattr(binding, "lib", lambda: Library())
    monkeypatch.setattr(binding, "_attend_workspace", lambda a, backward, device: (None, 0))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now["device"], raising=False)
    monkeypatch.setattr(torch.cuda, "device", lambda index: use(torch.device("cuda", index).index if isinstance(index, int) else index.index))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: use(s.device_index, s.number))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: now["stream"].get(i, 100 + i), raising=False)
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, lambda like, dtype=torch.float32, device=None: like if device is None else
                            On(device.index, *(like if isinstance(like, (tuple, torch.Size)) else (like,)), dtype=dtype))
    return seen


def attention(device, **change):
    i32 = torch.int32
    t = dict(q=On(device, 3, 4, 64), k=On(device, 9, 2, 64), v=On(device, 9, 2, 64), q_off=On(device, 3, dtype=i32), kv_off=On(device, 3, dtype=i32),
             kv_mask=On(device, 9, dtype=torch.uint8))
    t.update(change)
    return t


def stream_of(device, number):
    return type("Stream", (), dict(device_index=device, number=number))()


@pytest.mark.parametrize("device", [0, 1])
def test_launches_go_to_the_tensors_device(launches, device):
    t = attention(device)
    binding.tl_attend(**t)
    binding.tl_attend(**t, stream=stream_of(device, 7))
    rest = dict(o=On(device, 3, 4, 64), lse=On(device, 3, 4), d_o=On(device, 3, 4, 64))
    binding.tl_attend_backward(**t, **rest)
    binding.tl_attend_backward(**t, **rest, stream=stream_of(device, 8))
    binding.tl_sample(On(device, 3, 100), On(device, 3))
    binding.tl_sample(On(device, 3, 100), On(device, 3), stream=stream_of(device, 9))
    assert [(d, s) for _, d, s in launches] == [(device, s) for s in (100 + device, 7, 100 + device, 8, 100 + device, 9)]


@pytest.mark.parametrize("name", ["k", "v", "q_off", "kv_off", "kv_mask"])
def test_tensors_of_two_devices_are_refused(launches, name):
    other = attention(1)[name]
    with pytest.raises(AssertionError):
        binding.tl_attend(**attention(0, **{name: other}))
    with pytest.raises(AssertionError):
        binding.tl_attend_backward(**attention(0, **{name: other}), o=On(0, 3, 4, 64), lse=On(0, 3, 4), d_o=On(0, 3, 4, 64))
    assert not launches


def test_other_arguments_of_two_devices_are_refused(launches):
    rest = dict(o=On(0, 3, 4, 64), lse=On(0, 3, 4), d_o=On(0, 3, 4, 64))
    for name in rest:
        with pytest.raises(AssertionError):
            binding.tl_attend_backward(**attention(0), **dict(rest, **{name: On(1, *rest[name].shape)}))
    with pytest.raises(AssertionError):
        binding.tl_attend(**attention(0), o=On(1, 3, 4, 64))
    for i in range(5):
        args = [On(0, 3), None, None, None, None]
        args[i] = On(1, 3, dtype=torch.int32 if i == 2 else torch.float32)
        with pytest.raises(AssertionError):
            binding.tl_sample(On(0, 3, 100), *args)
    for call in (lambda s: binding.tl_attend(**attention(0), stream=s), lambda s: binding.tl_sample(On(0, 3, 100), On(0, 3), stream=s)):
        with pytest.raises(AssertionError):
            call(stream_of(1, 7))
    assert not launches
