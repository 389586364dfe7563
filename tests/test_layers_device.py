"""Which device a call of the layer operators runs on: that of its tensors, current or not.  No GPU: tensors, the current device and the library are
stood in for, and what the library's functions see is written down."""
import math
import types

import pytest
import torch

from paper_1907_03329_amd import layers


class Tensor:
    """What the binding asks of a tensor."""

    def __init__(self, shape, dtype, device):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device(device)

    def stride(self):
        return tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def view(self, dtype):
        return Tensor(self.shape, dtype, self.device)


@pytest.fixture
def calls(monkeypatch):
    """[(function, current device, stream)], with cuda:0 as the current device and the raw stream 100 + i as device i's."""
    current, seen = [0], []

    class Device:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.before

    def size_of(*args):     # the size goes where the last argument points
        args[-1]._obj.value = 256
        return 0

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes") or name.endswith("_elements"):
                size_of.__name__ = name
                return size_of
            return lambda *args: seen.append((name, current[0], args[-1])) or 0

    library = Library()
    make = lambda shape, dtype=torch.float32, device="cuda": Tensor(shape if isinstance(shape, (tuple, torch.Size)) else (shape,), dtype, device)  # noqa: E731
    monkeypatch.setattr(layers, "_library", lambda: library)
    monkeypatch.setattr(layers, "_current_device", lambda: current[0], raising=False)
    for owner, name in ((layers, "_raw_stream"), (torch._C, "_cuda_getCurrentRawStream")):
        monkeypatch.setattr(owner, name, lambda index: 100 + index, raising=False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch, "empty", make)
    monkeypatch.setattr(torch, "zeros", make)
    return seen


def run_all(device, stream=None):
    f = torch.float32
    x, p, state = Tensor((2, 5, 8), f, device), Tensor((8,), f, device), Tensor((2, 8), f, device)
    scan = layers.GatedRecurrence(2, 5, 8, device=device)
    scan.forward(x, x, stream=stream)
    scan.backward(x, x, x, stream=stream)
    layers.recurrence_step(state, state, state, state, stream=stream)
    norm = layers.GroupNorm(2, 5, 8, 2, device=device)
    norm.forward(x, p, p, stream=stream)
    norm.backward(x, p, p, x, stream=stream)
    adam = layers.AdamW([Tensor((256,), f, device)], [Tensor((256,), f, device)])
    adam.step(1, stream=stream)


LAUNCHED = ["esrnn_recurrence_forward", "esrnn_recurrence_backward", "esrnn_recurrence_step", "esrnn_group_norm_forward",
            "esrnn_group_norm_backward", "esrnn_adamw_bind", "esrnn_adamw_update"]


@pytest.mark.parametrize("index", [0, 1])
def test_every_call_runs_on_the_device_of_its_tensors(calls, index):
    run_all(f"cuda:{index}")
    assert [c for c in calls if c[0] in LAUNCHED] == [(name, index, 100 + index) for name in LAUNCHED]
    assert layers._current_device() == 0


def test_a_stream_of_the_tensors_device(calls):
    run_all("cuda:1", types.SimpleNamespace(device=torch.device("cuda:1"), cuda_stream=7))
    assert [c for c in calls if c[0] in LAUNCHED] == [(name, 1, 101 if name == "esrnn_adamw_bind" else 7) for name in LAUNCHED]


def test_a_stream_of_another_device_is_refused(calls):
    other = types.SimpleNamespace(device=torch.device("cuda:0"), cuda_stream=7)
    x, p, f = Tensor((2, 5, 8), torch.float32, "cuda:1"), Tensor((8,), torch.float32, "cuda:1"), Tensor((2, 8), torch.float32, "cuda:1")
    scan, norm = layers.GatedRecurrence(2, 5, 8, device="cuda:1"), layers.GroupNorm(2, 5, 8, 2, device="cuda:1")
    scan.forward(x, x)
    norm.forward(x, p, p)
    adam = layers.AdamW([p], [p])
    del calls[:]
    for call in (lambda: scan.forward(x, x, stream=other), lambda: scan.backward(x, x, x, stream=other),
                 lambda: layers.recurrence_step(f, f, f, f, stream=other), lambda: norm.forward(x, p, p, stream=other),
                 lambda: norm.backward(x, p, p, x, stream=other), lambda: adam.step(1, stream=other)):
        with pytest.raises(ValueError):
            call()
    assert not [c for c in calls if c[0] in LAUNCHED]
