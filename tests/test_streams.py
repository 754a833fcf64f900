"""Calls on a stream that the caller gives: on which stream their memory is allocated and which device is current when they
launch, without a GPU.  The allocator hands a block that was freed on a stream out again for that stream at once, while its
last use there may still be running; what is allocated under one stream and written on another is therefore a race."""
import contextlib
import math
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

    def is_contiguous(self):
        return True

    def numel(self):
        return math.prod(self.shape)

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

    fq.MxTensor(1, 1, device="cpu")                     # the native module is looked for with the library itself
    monkeypatch.setattr(fq, "_has_device", False)
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: w.current)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: empty(t.shape, dtype=t.dtype))
    monkeypatch.setattr(torch, "zeros", empty)
    monkeypatch.setattr(fq, "_lib", Library(fq.lib(), w))
    return w


def given(*shape, dtype=torch.bfloat16):
    return Allocated(shape, dtype, "the caller's")


def mx(rows, cols):
    return fq.MxTensor(rows, cols, fq.FQ_MX_BOTH)


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
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0, stream_id=3)
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
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0, stream_id=3)
    q, w, y = mx(40, 32), mx(48, 32), given(40, 48)
    del world.made[:]
    fq.fq_mx_quantize(given(40, 32), out=q, stream=stream)
    fq.fq_mx_gemm(fq.FQ_OP_NT, q, w, out=y, stream=stream)
    fq.fq_mx_linear(given(40, 32), w, xq=q, out=y, stream=stream)
    assert world.made == [] and y.kept_for == q.storage.kept_for == []
    assert [s for _, s in world.launches] == [stream] * 3


def _int8_calls():
    """The other calls that allocate, by name: call(stream) -> what it returns, all of it allocated by the call."""
    x, dy, w = given(40, 256), given(40, 256), given(256)
    q, v = fq.QTensor(40, 256, want_transposed=True), fq.QTensor(48, 256)
    ctx = given(40, 2, 160, dtype=torch.uint8), given(40, 2, dtype=torch.float32)
    rstd, tiled = given(40, dtype=torch.float32), given(2, 16384, dtype=torch.int8)
    return {
        "quantize": lambda s: fq.fq_quantize(x, fq.FQ_CRIT_NONE, 0.0, stream=s),
        "quantize_sr": lambda s: fq.fq_quantize_sr(x, 3, stream=s),
        "quantize_topk": lambda s: fq.fq_quantize_topk(x, 1, stream=s),
        "gemm": lambda s: fq.fq_gemm(fq.FQ_OP_NT, q, v, stream=s),
        "gemm_plain": lambda s: fq.fq_gemm_plain(fq.FQ_OP_NT, q, v, stream=s),
        "gemm_biased": lambda s: fq.fq_gemm_biased(fq.FQ_OP_NT, q, v, stream=s),
        "gemm_debug_partials": lambda s: fq.fq_gemm_debug_partials(fq.FQ_OP_NT, q, v, 0, 0, stream=s),
        "codes_to_rowmajor": lambda s: fq.fq_codes_to_rowmajor(tiled, 40, 256, stream=s),
        "ctx_dequantize": lambda s: fq.fq_ctx_dequantize(*ctx, 40, 256, stream=s),
        "glu_forward": lambda s: fq.fq_glu_forward(x, dy, stream=s),
        "glu_backward": lambda s: fq.fq_glu_backward(dy, ctx, ctx, stream=s),
        "rmsnorm_forward": lambda s: fq.fq_rmsnorm_forward(x, w, 1e-5, stream=s),
        "rmsnorm_backward": lambda s: fq.fq_rmsnorm_backward(dy, ctx, rstd, w, stream=s),
        "ctx_quantize": lambda s: fq.fq_ctx_quantize(x, stream=s),
    }


def _tensors(r):
    if isinstance(r, (tuple, list)):
        return [t for v in r for t in _tensors(v)]
    return [returned(r)]


INT8_CALLS = ["quantize", "quantize_sr", "quantize_topk", "gemm", "gemm_plain", "gemm_biased", "gemm_debug_partials",
              "codes_to_rowmajor", "ctx_quantize", "ctx_dequantize", "glu_forward", "glu_backward", "rmsnorm_forward",
              "rmsnorm_backward"]


@pytest.mark.parametrize("name", INT8_CALLS)
def test_memory_of_the_other_calls_is_allocated_under_their_stream(name, world):
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0, stream_id=3)
    call = _int8_calls()[name]
    del world.made[:]
    out = _tensors(call(stream))
    hidden = [t for t in world.made if not any(t is o for o in out)]
    assert world.made and all(t.under is stream for t in world.made)
    assert len(hidden) == (1 if name == "rmsnorm_backward" else 0)      # its partial sums
    assert [s for _, s in world.launches] == [stream] and world.current == "the caller's"
    assert all("the caller's" in t.kept_for for t in out)


@pytest.mark.parametrize("name", INT8_CALLS)
def test_nothing_changes_in_the_other_calls_without_a_stream(name, world, monkeypatch):
    monkeypatch.setattr(fq, "_native", None)
    monkeypatch.setattr(fq, "_current_stream", lambda: 9)
    monkeypatch.setattr(torch.cuda, "stream", None)
    call = _int8_calls()[name]
    del world.made[:]
    out = _tensors(call(None))
    assert all(t.under == "the caller's" and t.kept_for == [] for t in out) and len(world.launches) == 1


@pytest.mark.parametrize("device,current,makes,switched", [(0, 5, False, False), (0, 7, False, False), (0, 5, True, False),
                                                           (0, 7, True, True), (1, 5, False, True), (1, 5, True, True),
                                                           (1, 7, True, True)])
def test_the_stream_is_made_current_only_where_that_matters(device, current, makes, switched, world, monkeypatch):
    """A call that allocates, on a stream that is not the current one, or any call on another device's."""
    monkeypatch.setattr(fq, "_has_device", True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device)
    monkeypatch.setattr(fq, "_current_stream", lambda: current)
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0, stream_id=3)
    q = mx(40, 32)
    out = fq.fq_mx_quantize(given(40, 32), out=None if makes else q, sides=fq.FQ_MX_BOTH, stream=stream)
    fq.fq_gemm(fq.FQ_OP_NT, fq.QTensor(40, 32), fq.QTensor(48, 32), out=None if makes else given(40, 48), stream=stream)
    assert [s for _, s in world.launches] == [stream if switched else "the caller's"] * 2
    assert out.storage.kept_for == (["the caller's"] if makes and switched else [])


def test_an_object_with_a_handle_alone_is_launched_on(world):
    handle = types.SimpleNamespace(cuda_stream=5)
    q = fq.fq_quantize(given(40, 32), fq.FQ_CRIT_NONE, 0.0, stream=handle)
    fq.fq_gemm(fq.FQ_OP_NT, q, q, stream=handle)
    assert [s for _, s in world.launches] == ["the caller's"] * 2 and q.storage.kept_for == []
