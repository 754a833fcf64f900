"""Calls on a stream that the caller gives: on which stream their memory is allocated and which device is current when they
launch, without a GPU.  The allocator hands a block that was freed on a stream out again for that stream at once, while its
last use there may still be running; what is allocated under one stream and written on another is therefore a race."""
import contextlib
import types

import pytest
import torch

import paper_2503_08040_amd as fq


class Allocated:
    """A torch.empty on the GPU, as far as the Python layer looks at it."""
    is_cuda = True

    def __init__(self, shape, dtype, under):
        self.shape, self.dtype, self.under, self.kept_for = tuple(shape), dtype, under, []
        self.device = "cuda:0"

    def data_ptr(self):
        return 4096

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def stride(self, d=None):
        s = (self.shape[-1], 1)
        return s if d is None else s[d]

    def record_stream(self, stream):
        self.kept_for.append(stream)


class Library:
    """Sizes and bindings from the library itself, every launch noted with the stream that is current."""

    def __init__(self, real, world):
        self.real, self.world = real, world

    def __getattr__(self, name):
        if name.endswith(("_bytes", "_bind", "_string", "_tag")):
            return getattr(self.real, name)

        def call(*args):
            self.world.launches.append((name, self.world.current))
            return fq.FQ_OK
        return call


@pytest.fixture
def world(monkeypatch):
    """Notes every allocation and launch; `current` is the stream that torch would say is current."""
    w = types.SimpleNamespace(current="the caller's", made=[], launches=[])

    @contextlib.contextmanager
    def under(stream):
        before, w.current = w.current, stream
        yield
        w.current = before

    def empty(*shape, dtype=torch.float32, device=None):
        shape = shape[0] if len(shape) == 1 and not isinstance(shape[0], int) else shape
        w.made.append(Allocated(shape, dtype, w.current))
        return w.made[-1]

    fq.lib()
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: w.current)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: empty(t.shape, dtype=t.dtype))
    monkeypatch.setattr(torch, "zeros", empty)
    monkeypatch.setattr(fq, "_lib", Library(fq.lib(), w))
    return w


def given(*shape, dtype=torch.bfloat16):
    t = Allocated(shape, dtype, "the caller's")
    t.is_contiguous, t.numel = lambda: True, lambda: shape[0]
    return t


def mx(rows, cols):
    """An MxTensor of the caller's."""
    t = fq.MxTensor(rows, cols, fq.FQ_MX_BOTH)
    return t


MX_CALLS = {
    "quantize": lambda s, q, w: fq.fq_mx_quantize(given(40, 32), stream=s),
    "quantize_sr": lambda s, q, w: fq.fq_mx_quantize_sr(given(40, 32), 3, stream=s),
    "dequantize": lambda s, q, w: fq.fq_mx_dequantize(q, stream=s),
    "gemm": lambda s, q, w: fq.fq_mx_gemm(fq.FQ_OP_NT, q, w, stream=s),
    "linear": lambda s, q, w: fq.fq_mx_linear(given(40, 32), w, stream=s),
    "linear, one row": lambda s, q, w: fq.fq_mx_linear(given(1, 32), w, stream=s),
}


def returned(r):
    return r.storage if hasattr(r, "storage") else r


@pytest.mark.parametrize("name", MX_CALLS)
def test_memory_of_an_mx_call_is_allocated_under_its_stream(name, world):
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0)
    q, w = mx(40, 32), mx(48, 32)
    del world.made[:]
    r = returned(MX_CALLS[name](stream, q, w))
    assert len(world.made) == (2 if name == "linear" else 1)            # Q(x) and y
    assert all(t.under is stream for t in world.made)
    # its device is the current one at the launch, which is also what the library asks for compute units
    assert [s for _, s in world.launches] == [stream] and world.current == "the caller's"
    # what is handed out is kept for the stream that the caller goes on with
    assert r in world.made and "the caller's" in r.kept_for


@pytest.mark.parametrize("name", MX_CALLS)
def test_nothing_changes_without_a_stream(name, world, monkeypatch):
    monkeypatch.setattr(fq, "_native", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(fq, "_current_stream", lambda: 9)
    monkeypatch.setattr(torch.cuda, "stream", None)
    q, w = mx(40, 32), mx(48, 32)
    r = returned(MX_CALLS[name](None, q, w))
    assert r.under == "the caller's" and r.kept_for == [] and len(world.launches) == 1


def test_what_the_caller_gives_stays_the_callers(world):
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0)
    q, w, y = mx(40, 32), mx(48, 32), given(40, 48)
    del world.made[:]
    fq.fq_mx_quantize(given(40, 32), out=q, stream=stream)
    fq.fq_mx_gemm(fq.FQ_OP_NT, q, w, out=y, stream=stream)
    fq.fq_mx_linear(given(40, 32), w, xq=q, out=y, stream=stream)
    assert world.made == [] and y.kept_for == q.storage.kept_for == []
    assert [s for _, s in world.launches] == [stream] * 3
