"""Calls of the training operators that the library takes or refuses before a device is touched."""
import ctypes

import pytest

from paper_2512_15773_b200 import binding, build

P = 1 << 16                                 # an address that is never followed


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def test_an_empty_batch_with_copies_is_a_call_with_nothing_to_do(lib):
    """Tensors without values have no address: neither x nor the copies."""
    n, none = binding.NormT(1, 0, 16, 64, 8, 1, 1e-5), binding.SavedT(None, None)
    for sx, sy in ((none, None), (None, none), (none, none)):
        assert lib.tsdp_group_norm(0, n, None, 0, 64, P, P, None, None, 0, 64, None, None, sx, sy, None) == 0
    one = binding.NormT(1, 1, 16, 64, 8, 1, 1e-5)
    assert lib.tsdp_group_norm(0, one, P, 0, 64, P, P, None, P, 0, 64, None, None, none, None, None) == 1


class Rows:
    """Stands for a dense tensor on a GPU: sizes and an address, no memory."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, *shape, dtype="bfloat16"):
        import torch
        self.shape, self.dtype = shape, getattr(torch, dtype)

    def stride(self):
        s = [1]
        for v in self.shape[:0:-1]:
            s.append(s[-1] * v)
        return tuple(reversed(s))

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def data_ptr(self):
        return P

    def numel(self):
        n = 1
        for v in self.shape:
            n *= v
        return n

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True


class Taken:
    """Stands for the library: takes every call, keeps its arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*a):
            self.calls.append((name, a))
            return 16 if name.endswith("_workspace") else 0
        return call


def taken(monkeypatch):
    t = Taken()
    monkeypatch.setattr(binding, "load_library", lambda: t)
    return t


FAR = 2**32 + 8


@pytest.mark.parametrize("far", [FAR, -FAR, 2**31])
def test_counts_past_an_int_are_not_cut(monkeypatch, far):
    """2^32 + 8 groups are not eight; nor are so many input channels or taps."""
    lib = taken(monkeypatch)
    x, f32 = Rows(2, 16, 64), Rows(64, dtype="float32")
    stat, ws, dy = Rows(2 * FAR, dtype="float32"), Rows(1 << 20, dtype="uint8"), Rows(32, 64)
    stat.numel = lambda: 2 * far
    for call in (lambda: binding.group_norm(x, f32, f32, far, x, stream=0), lambda: binding.group_norm_grad_workspace(x, far),
                 lambda: binding.group_norm_grad(x, x, f32, f32, far, stat, stat, x, f32, f32, ws, stream=0),
                 lambda: binding.weight_grad_workspace(dy, far), lambda: binding.weight_grad_workspace(dy, 64, taps=far),
                 lambda: binding.weight_grad_workspace(dy, 64, length=far)):
        with pytest.raises(ValueError):
            call()
    assert not lib.calls
    binding.group_norm(x, f32, f32, 8, x, stream=0)
    assert lib.calls[0][0] == "tsdp_group_norm"


@pytest.mark.parametrize("given,taken_as", [({}, 77), (dict(stream=None), 77), (dict(stream=0), 0), (dict(stream=5), 5)])
def test_a_call_goes_to_the_current_stream_unless_one_is_given(monkeypatch, given, taken_as):
    """Between torch operations under torch.cuda.stream(s), or in a capture, the default stream would be another one than that of the tensors' own work."""
    lib = taken(monkeypatch)
    monkeypatch.setattr(binding, "_current_stream", lambda device: 77 + device)
    x, f32, dW = Rows(2, 16, 64), Rows(64, dtype="float32"), Rows(64, 64, dtype="float32")
    saved = Rows(2, 16, 64, dtype="int8"), Rows(2, 16, 2, dtype="uint8")
    flat = Rows(32, 64, dtype="int8"), Rows(32, 2, dtype="uint8")
    stat, ws = Rows(2, 8, dtype="float32"), Rows(1 << 20, dtype="uint8")
    binding.checkpoint_pack(x, saved, **given)
    binding.checkpoint_unpack(saved, x, **given)
    binding.group_norm(x, f32, f32, 8, x, **given)
    binding.group_norm_grad(x, x, f32, f32, 8, stat, stat, x, f32, f32, ws, **given)
    binding.weight_grad(flat, Rows(32, 64), dW, ws, **given)
    assert [a[-1] for _, a in lib.calls] == [taken_as] * 5
