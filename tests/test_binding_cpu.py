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

    def mop_status_string(self, code):
        return b""

    def workspace_bytes(self, *args):
        return 300

    mop_moe_balance_workspace_bytes = mop_vocab_distill_workspace_bytes = mop_vocab_distill_bwd_workspace_bytes = workspace_bytes

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


def fresh(n, dtype):
    """n zeros on the host, from a 256-byte boundary on."""
    raw = torch.zeros((n * 8 + 512,), dtype=torch.uint8)
    at = -raw.data_ptr() % 256
    return raw[at:at + n * torch.empty((), dtype=dtype).element_size()].view(dtype)


def balance_arguments():
    """A context's shape and, in the order of the calls, every tensor of the balance loss on the host (which stands in for its device)."""
    T, d, E, k, S = 33, 16, 5, 2, 3
    ctx = binding.Context(T, d, E, k, 8)
    ctx.device = -1
    f32, i32, b16 = torch.float32, torch.int32, torch.bfloat16
    t = {n: torch.zeros(shape, dtype=dtype) for n, shape, dtype in (
        ("logits", (T, E), f32), ("bias", (E,), f32), ("topk_idx", (T, k), i32), ("seq_offsets", (S + 1,), i32), ("counts", (S, E), i32),
        ("prob", (S, E), f32), ("loss", (S,), f32), ("dloss", (S,), f32), ("x", (T, d), b16), ("W_r", (d, E), f32), ("dlogits", (T, E), f32),
        ("dW_r", (d, E), f32), ("dbias", (E,), f32), ("dX", (T, d), b16), ("workspace", (300,), torch.uint8))}
    return ctx, t


def distill_arguments():
    N, H, V, K = 9, 16, 24, 3
    f32, b16 = torch.float32, torch.bfloat16
    return {n: torch.zeros(shape, dtype=dtype) for n, shape, dtype in (
        ("X", (N, H), b16), ("W_voc", (H, V), b16), ("teacher_idx", (N, K), torch.int32), ("teacher_logits", (N, K), f32),
        ("teacher_lse", (N,), f32), ("loss", (N,), f32), ("student", (N, K), f32), ("lse", (N,), f32), ("dloss", (N,), f32),
        ("dX", (N, H), b16), ("dW_voc", (H, V), b16), ("workspace", (300,), torch.uint8))}


def losses_calls(device):
    """{call: (function of its tensors by name, the names)}"""
    ctx, _ = balance_arguments()
    ctx.device = device
    calls = {}
    for name, fn, extra in (("balance_fwd", binding.mop_moe_balance_loss_fwd, {"ctx": ctx}),
                            ("balance_bwd", binding.mop_moe_balance_loss_bwd, {"ctx": ctx, "accumulate": False}),
                            ("distill_fwd", binding.mop_vocab_distill_fwd, {"device": device, "temperature": 1.0}),
                            ("distill_bwd", binding.mop_vocab_distill_bwd, {"device": device, "temperature": 1.0})):
        names = [n for n in inspect.signature(fn).parameters if n not in extra and n != "stream"]
        calls[name] = (lambda t, fn=fn, extra=extra: fn(**extra, **t, stream=5), names)
    return calls


SIZES_FROM = {"loss", "dloss", "X", "W_voc", "teacher_idx"}      # tensors that a call takes its sizes from: the others have to fit


@pytest.mark.parametrize("call", ["balance_fwd", "balance_bwd", "distill_fwd", "distill_bwd"])
def test_tensors_that_a_call_would_read_or_write_past_their_end_are_refused(library, call):
    fn, names = losses_calls(-1)[call]
    every = {**balance_arguments()[1], **distill_arguments()} if call.startswith("distill") else balance_arguments()[1]
    t = {n: every[n] for n in names}
    fn(t)
    assert library.calls[-1][0] == "mop_" + {"b": "moe_", "d": "vocab_"}[call[0]] + call.replace("_", "_loss_" if call[0] == "b" else "_")
    sent = [a for a in library.calls[-1][1] if isinstance(a, int)]
    assert all(t[n].data_ptr() in sent for n in names)
    for name in names:
        def refused(wrong):
            before = len(library.calls)
            with pytest.raises(binding.MopError, match=name) as e:
                fn({**t, name: wrong})
            assert e.value.code == 1 and not [c for c in library.calls[before:] if c[0].startswith(("mop_moe_balance_loss", "mop_vocab_distill"))
                                              and "bytes" not in c[0]]
        flat = t[name].reshape(-1)
        if name not in SIZES_FROM:
            refused(fresh(flat.numel() - 1, flat.dtype))
            fn({**t, name: fresh(2 * flat.numel(), flat.dtype)})          # more than is used is the caller's business
    # what leads nowhere is the library's to refuse: a tensor off its 16 bytes, and none
    last = "lse" if call.startswith("distill") else "logits"
    long = torch.zeros((t[last].numel() + 1,), dtype=t[last].dtype)
    fn({**t, last: long[1:][:t[last].numel() - 4]})
    fn({**t, last: None})
    fn({**t, last: 4096})                                     # an address
    with pytest.raises(binding.MopError, match="workspace"):
        fn({**t, last: 4096, "workspace": fresh(299, torch.uint8)})
    with pytest.raises(AssertionError, match="dense"):
        fn({**t, last: fresh(2 * t[last].numel(), t[last].dtype)[::2]})


@pytest.mark.parametrize("call", ["balance_fwd", "balance_bwd", "distill_fwd", "distill_bwd"])
def test_tensors_on_another_device_are_refused(library, call):
    fn, names = losses_calls(0)[call]
    every = {**balance_arguments()[1], **distill_arguments()} if call.startswith("distill") else balance_arguments()[1]
    with pytest.raises(binding.MopError, match="on cpu"):
        fn({n: every[n] for n in names})
    assert not [c for c in library.calls if c[0].startswith(("mop_moe_balance_loss", "mop_vocab_distill")) and "bytes" not in c[0]]
