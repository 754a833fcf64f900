"""When the native module becomes visible to calls: other threads take it as soon as it does."""
import ctypes as C
import sys
import types

import pytest
import torch

import paper_2503_08040_amd as fq


def test_the_native_module_is_used_once_it_has_every_entry_point(monkeypatch):
    """A call through it in between would jump to address 0."""
    monkeypatch.setattr(fq, "_native", None)
    seen = {}

    def setup(name, *args):
        seen[name] = (fq._native, args)

    module = types.SimpleNamespace(torch_version=torch.__version__, header_tag=fq.fq_header_tag(),
                                   setup=lambda *a: setup("setup", *a), setup_mx=lambda *a: setup("setup_mx", *a))
    monkeypatch.setattr(fq, "_fqnative", module, raising=False)
    monkeypatch.setitem(sys.modules, "paper_2503_08040_amd._fqnative", module)
    fq._native_setup()
    assert fq._native is module
    assert [seen[n][0] for n in ("setup", "setup_mx")] == [None, None]
    address = lambda n: C.cast(getattr(fq.lib(), n), C.c_void_p).value
    assert seen["setup"][1][:3] == tuple(address(n) for n in ("fq_quantize", "fq_quantize_sr", "fq_gemm"))
    assert seen["setup_mx"][1] == tuple(address("fq_mx_" + n) for n in ("quantize", "quantize_sr", "dequantize", "gemm", "linear"))


def test_a_setup_that_fails_leaves_the_calls_to_ctypes(monkeypatch):
    def fails(*args):
        raise TypeError

    monkeypatch.setattr(fq, "_native", None)
    module = types.SimpleNamespace(torch_version=torch.__version__, header_tag=fq.fq_header_tag(), setup=lambda *a: None,
                                   setup_mx=fails)
    monkeypatch.setattr(fq, "_fqnative", module, raising=False)
    monkeypatch.setitem(sys.modules, "paper_2503_08040_amd._fqnative", module)
    with pytest.raises(TypeError):
        fq._native_setup()
    assert fq._native is None
