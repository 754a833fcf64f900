"""Microscaled calls from several threads, each on a stream of its own."""
import threading

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_08040_amd as fq
from tests import gpu_util as gu
from tests.test_gpu_mx_streams import matrix


@pytest.mark.parametrize("native", [True, False])
def test_several_threads(native, monkeypatch):
    """A layer's step in each of four threads, on a stream and tensors of its own."""
    if not native:
        monkeypatch.setattr(fq, "_native", None)
    M, K, N = 200, 700, 1100

    def step(i, x, W, dy):
        q, s = fq.MxTensor(M, K, fq.FQ_MX_BOTH), fq.MxTensor(M, N, fq.FQ_MX_BOTH)
        fq.fq_mx_quantize(x, out=q)
        fq.fq_mx_quantize_sr(dy, 100 + i, out=s)
        return [fq.fq_mx_linear(x, W), fq.fq_mx_linear(x[:2], W), fq.fq_mx_gemm(fq.FQ_OP_NN, s, W),
                fq.fq_mx_gemm(fq.FQ_OP_TN, s, q, out_dtype=torch.bfloat16), fq.fq_mx_dequantize(s, fq.FQ_MX_COLS)]

    inputs = [(matrix(M, K, 3 * i), fq.fq_mx_quantize(matrix(N, K, 3 * i + 1), sides=fq.FQ_MX_BOTH), matrix(M, N, 3 * i + 2))
              for i in range(4)]
    want = [step(i, *t) for i, t in enumerate(inputs)]
    torch.cuda.synchronize()
    failed, start = [], threading.Barrier(4)

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(30)
                for _ in range(20):
                    got = step(i, *inputs[i])
                    torch.cuda.current_stream().synchronize()
                    assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
        except BaseException as e:
            failed.append((i, e))

    gu.announce(f"mx calls from four threads, native {native}")
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(100)
    assert not failed and not any(t.is_alive() for t in threads)
