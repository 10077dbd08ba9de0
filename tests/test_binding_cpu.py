"""What the binding decides before it calls the library (no device here)."""
import inspect
import re
import types

import pytest
import torch

from paper_2607_01844_b200 import binding


class Library:
    """Stands in for the shared library: every call succeeds and leaves its arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "_lib", lib)
    return lib


@pytest.mark.parametrize("private", [True, False], ids=["raw", "stream"])
def test_without_a_stream_a_call_runs_on_the_current_one_of_its_own_device(monkeypatch, library, private):
    """Device 0 is current, the context and the vocabulary call are on device 1."""
    current = {0: 10, 1: 11}
    if private:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", current.__getitem__, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=0: types.SimpleNamespace(cuda_stream=current[d]))
    ctx = binding.Context(4, 8, 4, 2, 8, device=1)
    binding.mop_poll(ctx)
    binding.mop_moe_combine(ctx, None, None, None)
    binding.mop_vocab_poll(1, None)
    binding.mop_moe_combine(ctx, None, None, None, stream=5)
    assert [args[-1] for name, args in library.calls[1:]] == [11, 11, 11, 5]
    assert binding._stream(None) == 10


def test_every_call_names_its_device_where_it_asks_for_the_stream():
    for name, fn in inspect.getmembers(binding, inspect.isfunction):
        if name.startswith("mop_") and "stream" in inspect.signature(fn).parameters:
            first = next(iter(inspect.signature(fn).parameters))
            want = {"ctx": "ctx.device", "device": "device"}[first]
            assert re.findall(r"_stream\(stream, ([\w.]+)\)", inspect.getsource(fn)) == [want], name


def test_a_device_that_is_not_there_is_left_to_the_library(monkeypatch):
    def raw(device):
        if device != 0:
            raise RuntimeError("invalid device")
        return 10
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", raw, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert binding._stream(None, 9) == 10
