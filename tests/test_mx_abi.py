"""Host-side checks of the microscaled calls that need no GPU: sizes, binding, and what is refused before anything is
launched; what the Python layer hands over and refuses."""
import ctypes as C
import types

import pytest
import torch

import paper_2503_08040_amd as fq

X = C.c_void_p(0x2000)


def _side(R, Cc):
    up = lambda n: -(-n // 256) * 256
    return up(-(-R // 16) * -(-Cc // 128) * 1024) + up(-(-R // 64) * -(-Cc // 128) * 256)


def test_bytes():
    for R, Cc in [(0, 0), (0, 7), (1, 1), (16, 128), (17, 129), (300, 70)]:
        assert fq.fq_mx_bytes(R, Cc, fq.FQ_MX_ROWS) == 256 + _side(R, Cc)
        assert fq.fq_mx_bytes(R, Cc, fq.FQ_MX_COLS) == 256 + _side(Cc, R)
        assert fq.fq_mx_bytes(R, Cc, fq.FQ_MX_BOTH) == 256 + _side(R, Cc) + _side(Cc, R)
    for bad in [(-1, 5, 1), (5, -1, 1), (5, 5, 0), (5, 5, 4), (5, 5, -1)]:
        assert fq.fq_mx_bytes(*bad) == 0
    most = 2 ** 23 * 128
    assert fq.fq_mx_bytes(1, most) > 0 and fq.fq_mx_bytes(1, most + 1) == 0 == fq.fq_mx_bytes(most + 1, 1)
    assert fq.fq_mx_bytes(2 ** 31 - 1, 2 ** 31 - 1, 3) == 0


def _bind(rows, cols, sides=fq.FQ_MX_BOTH, base=0x100000):
    t = fq.fq_mx_tensor()
    assert fq.lib().fq_mx_bind(C.c_void_p(base), rows, cols, sides, C.byref(t)) == fq.FQ_OK
    return t


def test_bind():
    t = _bind(130, 200)
    assert (t.rows, t.cols) == (130, 200)
    ptrs = [t.codes, t.scales, t.codes_t, t.scales_t]
    assert all(p % 256 == 0 for p in ptrs) and sorted(set(ptrs)) == ptrs and ptrs[0] == 0x100000
    assert t.scales_t + 4 * 2 * 256 <= 0x100000 + fq.fq_mx_bytes(130, 200, 3)
    r, c = _bind(130, 200, fq.FQ_MX_ROWS), _bind(130, 200, fq.FQ_MX_COLS)
    assert r.codes and r.scales and not r.codes_t and not r.scales_t
    assert c.codes_t and c.scales_t and not c.codes and not c.scales
    bind, out = fq.lib().fq_mx_bind, C.byref(fq.fq_mx_tensor())
    assert bind(None, 4, 4, 1, out) == bind(X, 4, 4, 1, None) == fq.FQ_ERR_NULL
    assert bind(X, 4, 4, 0, out) == bind(X, 4, 4, 4, out) == fq.FQ_ERR_ENUM
    assert bind(C.c_void_p(0x2010), 4, 4, 1, out) == bind(X, -4, 4, 1, out) == bind(X, 1, 2 ** 31 - 1, 1, out) == fq.FQ_ERR_SHAPE


def test_quantize_refusals():
    t = _bind(256, 200)
    L, r = fq.lib(), C.byref(t)
    for call in (lambda x, m, n, ld, out, rule=0: L.fq_mx_quantize(x, m, n, ld, rule, out, None),
                 lambda x, m, n, ld, out, rule=0: L.fq_mx_quantize_sr(x, m, n, ld, 7, out, None)):
        assert call(X, 256, 200, 200, None) == call(None, 256, 200, 200, r) == fq.FQ_ERR_NULL
        for m, n, ld in [(256, 200, 199), (-1, 200, 200), (256, -1, 200), (255, 200, 200), (256, 201, 201)]:
            assert call(X, m, n, ld, r) == fq.FQ_ERR_SHAPE
    assert L.fq_mx_quantize(X, 256, 200, 200, 2, r, None) == fq.FQ_ERR_ENUM
    assert L.fq_mx_quantize(X, 256, 200, 200, -1, r, None) == fq.FQ_ERR_ENUM
    for field, value, want in [("codes", None, fq.FQ_ERR_NULL), ("scales", None, fq.FQ_ERR_NULL),
                               ("scales_t", None, fq.FQ_ERR_NULL), ("codes_t", 0x100008, fq.FQ_ERR_SHAPE),
                               ("rows", -1, fq.FQ_ERR_SHAPE), ("cols", 2 ** 31 - 1, fq.FQ_ERR_SHAPE)]:
        b = _bind(256, 200)
        setattr(b, field, value)
        assert L.fq_mx_quantize(X, 256, 200, 200, 0, C.byref(b), None) == want, field
    none = fq.fq_mx_tensor(rows=4, cols=4)
    assert L.fq_mx_quantize(X, 4, 4, 4, 0, C.byref(none), None) == fq.FQ_ERR_NULL
    for rows, cols in [(0, 5), (5, 0), (0, 0)]:
        assert L.fq_mx_quantize(None, rows, cols, cols, 0, C.byref(_bind(rows, cols)), None) == fq.FQ_OK


def test_dequantize_refusals():
    L, t = fq.lib(), _bind(40, 50)
    d = lambda t, side, out, odt=0, ldo=50: L.fq_mx_dequantize(C.byref(t) if t else None, side, out, odt, ldo, None)
    assert d(None, 1, X) == d(t, 1, None) == fq.FQ_ERR_NULL
    assert d(t, 0, X) == d(t, 3, X) == d(t, 1, X, 2) == d(t, 1, X, -1) == fq.FQ_ERR_ENUM
    assert d(t, 1, X, 0, 49) == fq.FQ_ERR_SHAPE
    assert d(_bind(40, 50, fq.FQ_MX_COLS), fq.FQ_MX_ROWS, X) == d(_bind(40, 50, 1), fq.FQ_MX_COLS, X) == fq.FQ_ERR_NULL
    assert d(_bind(0, 50), 1, None) == d(_bind(40, 0), 2, None, 1, 0) == fq.FQ_OK


def test_gemm_refusals():
    L = fq.lib()
    ref = lambda t: C.byref(t) if t is not None else None
    g = lambda op, a, b, c=X, cdt=0, ldc=384: L.fq_mx_gemm(op, ref(a), ref(b), c, cdt, ldc, None)
    a, b = _bind(256, 512), _bind(384, 512)
    assert g(0, None, b) == g(0, a, None) == g(0, a, b, None) == fq.FQ_ERR_NULL
    assert g(3, a, b) == g(-1, a, b) == g(0, a, b, cdt=2) == g(0, a, b, cdt=-1) == fq.FQ_ERR_ENUM
    assert g(0, a, b, ldc=383) == g(0, a, _bind(384, 640)) == g(1, a, b, ldc=512) == g(2, a, b, ldc=512) == fq.FQ_ERR_SHAPE
    rows, cols = fq.FQ_MX_ROWS, fq.FQ_MX_COLS
    for op, sa, sb in [(0, cols, rows), (0, rows, cols), (1, cols, cols), (1, rows, rows), (2, rows, cols), (2, cols, rows)]:
        shape = {0: ((64, 32), (96, 32)), 1: ((64, 32), (32, 96)), 2: ((32, 64), (32, 96))}[op]
        assert g(op, _bind(*shape[0], sa), _bind(*shape[1], sb)) == fq.FQ_ERR_NULL, (op, sa, sb)
    wide = _bind(2 ** 18, 1, rows), _bind(2 ** 18 + 64, 1, rows)       # 2^12 and 2^12 + 1 tiles of 64
    assert g(0, *wide, ldc=2 ** 19) == fq.FQ_ERR_SHAPE
    long, short = _bind(2 ** 27 + 1, 1, rows), _bind(1, 1, rows)       # 2^21 + 1 tiles of 64, cut into smaller ones
    assert g(0, long, short, ldc=1) == g(0, short, long, ldc=2 ** 28) == fq.FQ_ERR_SHAPE
    assert g(0, _bind(0, 512), b, None) == g(0, a, _bind(0, 512), None, ldc=0) == fq.FQ_OK


def test_linear_refusals():
    L = fq.lib()
    ref = lambda t: C.byref(t) if t is not None else None
    f = lambda w, q, x=X, rows=40, ld=512, rule=0, y=X, ydt=0, ldy=384: \
        L.fq_mx_linear(x, rows, ld, rule, ref(w), ref(q), y, ydt, ldy, None)
    w, q = _bind(384, 512), _bind(40, 512, base=0x900000)
    assert f(None, q) == f(w, None) == f(w, q, x=None) == f(w, q, y=None) == fq.FQ_ERR_NULL
    assert f(w, q, rule=2) == f(w, q, ydt=2) == fq.FQ_ERR_ENUM
    assert f(w, q, rows=41) == f(w, q, rows=-1) == f(w, q, ld=511) == f(w, q, ldy=383) == f(w, _bind(40, 513, base=0x900000)) == fq.FQ_ERR_SHAPE
    assert f(q, q) == fq.FQ_ERR_SHAPE                # the space for Q(X) is W itself
    assert f(_bind(384, 512, fq.FQ_MX_COLS), q) == f(w, _bind(40, 512, fq.FQ_MX_COLS, 0x900000)) == fq.FQ_ERR_NULL
    assert f(w, _bind(0, 512, base=0x900000), x=None, rows=0, y=None) == fq.FQ_OK


def test_form_says_which_tiles_run():
    form = lambda *a: fq.fq_mx_gemm_form(*a, 256)
    for M, N, K, want in [(1, 11008, 4096, (fq.FQ_MX_FORM_32x64, True)), (16, 4096, 11008, (fq.FQ_MX_FORM_32x32, False)),
                          (256, 512, 512, (fq.FQ_MX_FORM_32x32, True)), (256, 1024, 11008, (fq.FQ_MX_FORM_32x32, False)),
                          (128, 4096, 4096, (fq.FQ_MX_FORM_32x64, False)), (1024, 1024, 4096, (fq.FQ_MX_FORM_64x64, False)),
                          (64, 11008, 4096, (fq.FQ_MX_FORM_64x64, False)), (1024, 2048, 640, (fq.FQ_MX_FORM_64x64, False)),
                          (2048, 2048, 2048, (fq.FQ_MX_FORM_128x128, False)), (2048, 4096, 4096, (fq.FQ_MX_FORM_128x256, False)),
                          (5000, 129, 4096, (fq.FQ_MX_FORM_64x64, False)), (20000, 128, 4096, (fq.FQ_MX_FORM_128x128, False)), (512, 11008, 128, (fq.FQ_MX_FORM_128x128, False)),
                          (1500, 11008, 4096, (fq.FQ_MX_FORM_128x128, False)), (4096, 11008, 4096, (fq.FQ_MX_FORM_256x256, False)),
                          (8192, 8192, 8192, (fq.FQ_MX_FORM_256x256, False)), (3000, 3000, 4096, (fq.FQ_MX_FORM_256x256, False)),
                          (3000, 3000, 2048, (fq.FQ_MX_FORM_128x128, False)),
                          (16, 2 ** 20, 256, (fq.FQ_MX_FORM_32x64, True)), (2 ** 20, 40, 256, (fq.FQ_MX_FORM_64x64, False)),
                          (0, 5, 5, (0, False)), (4096, 4096, 0, (fq.FQ_MX_FORM_64x64, False))]:
        assert form(M, N, K) == want, (M, N, K, form(M, N, K))
    # a linear layer in one launch has the sums of the product of stored codes: 8 parts of the contraction
    for M in (1, 5, 16, 17, 40, 128, 300):
        for N in (1, 64, 1000, 4096, 20000, 300000):
            for K in (32, 512, 4096, 65536, 10 ** 6):
                tiles, one = form(M, N, K)
                assert not one or tiles in (fq.FQ_MX_FORM_32x32, fq.FQ_MX_FORM_32x64)
                assert M > fq.FQ_MX_LINEAR_ROWS or tiles in (fq.FQ_MX_FORM_32x32, fq.FQ_MX_FORM_32x64)
    assert fq.fq_mx_gemm_form(512, 512, 2048, 1)[0] == fq.FQ_MX_FORM_256x256
    assert fq.fq_mx_gemm_form(300, 300, 256, 1)[0] == fq.FQ_MX_FORM_128x128
    p = (C.c_int32 * 2)()
    for bad in [(-1, 5, 5), (5, -1, 5), (5, 5, -1)]:
        assert fq.lib().fq_mx_gemm_form(*bad, 4, p) == fq.FQ_ERR_SHAPE
    assert fq.lib().fq_mx_gemm_form(5, 5, 5, 4, None) == fq.FQ_ERR_NULL


class _Recorder:
    def __init__(self):
        self.calls = []
        self.fq_status_string = fq.lib().fq_status_string

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return fq.FQ_OK
        return call


def _tensor(rows, cols, sides=3, device=0):
    """An MxTensor whose storage says that it is on that GPU."""
    t = fq.MxTensor(rows, cols, sides, device="cpu")
    t.keep = t.storage
    t.storage = types.SimpleNamespace(is_cuda=True, get_device=lambda: device, device="cpu")
    return t


def _matrix(rows, cols, pitch, dtype=torch.bfloat16, device=0):
    return types.SimpleNamespace(dtype=dtype, is_cuda=True, shape=(rows, cols), dim=lambda: 2, device="cpu",
                                 stride=lambda d=None: (pitch, 1) if d is None else (pitch, 1)[d], data_ptr=lambda: 256,
                                 get_device=lambda: device)


def test_python_layer(monkeypatch):
    """Shapes, pitches, types, sides and devices as they reach the library; what the Python functions refuse."""
    q, w, q1, w1 = _tensor(4, 32), _tensor(6, 32), _tensor(4, 32, device=1), _tensor(6, 32, device=1)
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0)
    rec = _Recorder()
    monkeypatch.setattr(fq, "_lib", rec)
    x = _matrix(4, 32, 40)
    fq.fq_mx_quantize(x, out=q, rule=fq.FQ_MX_COVER, stream=stream)
    fq.fq_mx_quantize_sr(x, 2 ** 40 + 1, out=q, stream=stream)
    y = _matrix(4, 6, 11, torch.float32)
    fq.fq_mx_gemm(fq.FQ_OP_NT, q, w, out=y, stream=stream)
    fq.fq_mx_dequantize(q, fq.FQ_MX_COLS, out=x, stream=stream)
    fq.fq_mx_linear(x, w, out=_matrix(4, 6, 7), stream=stream)
    names, args = zip(*rec.calls)
    assert names == ("fq_mx_quantize", "fq_mx_quantize_sr", "fq_mx_gemm", "fq_mx_dequantize", "fq_mx_linear")
    assert all(a[-1] == 5 for a in args)
    assert args[0][:5] == (256, 4, 32, 40, 1) and args[1][:4] == (256, 4, 32, 40) and args[1][4].value == 2 ** 40 + 1
    assert args[2][0] == fq.FQ_OP_NT and args[2][3:6] == (256, fq.FQ_OUT_F32, 11)
    assert args[3][1:5] == (fq.FQ_MX_COLS, 256, fq.FQ_OUT_BF16, 40)
    assert args[4][:4] == (256, 4, 40, fq.FQ_MX_FLOOR) and args[4][5] is None and args[4][7:9] == (fq.FQ_OUT_BF16, 7)
    refused = [lambda: fq.fq_mx_quantize(_matrix(4, 32, 40, torch.float32), out=q, stream=stream),
               lambda: fq.fq_mx_gemm(fq.FQ_OP_NT, q, w, out=torch.empty((4, 6)), stream=stream),      # not on the GPU
               lambda: fq.fq_mx_gemm(fq.FQ_OP_NT, q, w, out=_matrix(6, 4, 4, torch.float32), stream=stream),
               # tensors on another device than the stream's
               lambda: fq.fq_mx_quantize(_matrix(4, 32, 40, device=1), out=q, stream=stream),
               lambda: fq.fq_mx_quantize_sr(x, 1, out=q1, stream=stream),
               lambda: fq.fq_mx_gemm(fq.FQ_OP_NT, q, w1, out=y, stream=stream),
               lambda: fq.fq_mx_gemm(fq.FQ_OP_NT, q, w, out=_matrix(4, 6, 6, torch.float32, 1), stream=stream),
               lambda: fq.fq_mx_dequantize(q1, out=x, stream=stream),
               lambda: fq.fq_mx_linear(x, w, xq=q1, out=y, stream=stream),
               lambda: fq.fq_mx_linear(x, w1, out=y, stream=stream)]
    for call in refused:
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(KeyError):
        fq.fq_mx_gemm(fq.FQ_OP_NT, q, w, out=_matrix(4, 6, 6, torch.float16), stream=stream)
    for call in (lambda: fq.fq_mx_linear(_matrix(4, 33, 33), w, stream=stream), lambda: fq.fq_mx_gemm(7, q, w, stream=stream)):
        with pytest.raises(fq.FqError):
            call()
    assert len(rec.calls) == 5


def test_space_taken_for_a_call_is_kept_for_its_stream(monkeypatch):
    """The space for Q(x) that fq_mx_linear takes by itself is freed when it returns, while the given stream uses it."""
    w = _tensor(6, 32)
    kept = []
    make = lambda rows, cols, sides, device: types.SimpleNamespace(
        _ref=None, storage=types.SimpleNamespace(is_cuda=True, get_device=lambda: 0, record_stream=kept.append))
    monkeypatch.setattr(fq, "_lib", _Recorder())
    monkeypatch.setattr(fq, "MxTensor", make)
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0)
    fq.fq_mx_linear(_matrix(40, 32, 32), w, out=_matrix(40, 6, 6), stream=stream)
    assert kept == [stream]
    fq.fq_mx_linear(_matrix(16, 32, 32), w, out=_matrix(16, 6, 6), stream=stream)
    assert kept == [stream]


def test_the_current_device_counts_without_a_stream(monkeypatch):
    q = _tensor(4, 32)
    rec = _Recorder()
    for device, taken in ((0, True), (1, False)):
        cuda = types.SimpleNamespace(current_device=lambda: device, current_stream=lambda: types.SimpleNamespace(cuda_stream=9))
        monkeypatch.setattr(fq, "_lib", rec)
        monkeypatch.setattr(fq, "_torch", types.SimpleNamespace(_C=types.SimpleNamespace(), cuda=cuda, bfloat16=torch.bfloat16))
        monkeypatch.setattr(fq, "_current_stream", None)
        n = len(rec.calls)
        if taken:
            fq.fq_mx_quantize(_matrix(4, 32, 32), out=q)
            assert len(rec.calls) == n + 1 and rec.calls[-1][1][-1] == 9
        else:
            with pytest.raises(AssertionError):
                fq.fq_mx_quantize(_matrix(4, 32, 32), out=q)
            assert len(rec.calls) == n


def test_views():
    q = fq.MxTensor(4, 32, 3, device="cpu")
    assert q.view("codes").shape == (1, 1, 1024) and q.view("scales_t").shape == (1, 1, 256)
    assert q.view("codes_t").shape == (2, 1, 1024) and fq.MxTensor(4, 4, 1, device="cpu").view("codes_t") is None
    assert q.view("codes").data_ptr() == q.c.codes and q.view("scales_t").data_ptr() == q.c.scales_t
    for bad in [(-1, 4, 1), (4, 4, 0), (4, 4, 4)]:
        with pytest.raises(fq.FqError):
            fq.MxTensor(*bad, device="cpu")


def test_the_native_module_leaves_anything_unusual_to_the_python_code():
    native = pytest.importorskip("paper_2503_08040_amd._fqnative")
    q, w = fq.MxTensor(4, 8, 3, device="cpu"), fq.MxTensor(6, 8, 3, device="cpu")
    x = torch.zeros((4, 8), dtype=torch.bfloat16)                    # nothing is on the GPU
    for first in (x, None, 3, x.float(), x[0], torch.nn.Parameter(x)):
        assert native.mx_quantize(first, 0, q._addr, q.storage) is None
        assert native.mx_quantize_sr(first, 1, q._addr, q.storage) is None
        assert native.mx_linear(first, w._addr, w.storage, 0, None, 0, None, None) is None
    assert native.mx_gemm("0", q._addr, w._addr, q.storage, w.storage, None, None) is None
    assert native.mx_dequantize(q._addr, None, 1, None, None) is None
    with pytest.raises(TypeError):
        native.setup_mx(1, 2)
