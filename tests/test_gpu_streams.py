"""The INT8 path's calls on a stream that the caller gives: the same values, in blocks of that stream."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_08040_amd as fq
from tests import gpu_util as gu
from tests.test_gpu_mx_streams import matrix, stream_of


def flat(r):
    return [t for v in r for t in flat(v)] if isinstance(r, (tuple, list)) else [r]


def test_the_int8_paths_calls_on_a_given_stream():
    x, dy, w = matrix(200, 384, 1), matrix(200, 384, 2), matrix(1, 384, 3)[0]
    q, v = fq.fq_quantize(x, fq.FQ_CRIT_NONE, 0.0), fq.fq_quantize(matrix(300, 384, 4), fq.FQ_CRIT_NONE, 0.0)
    ctx, other = fq.fq_ctx_quantize(x), fq.fq_ctx_quantize(dy)
    rstd = fq.fq_rmsnorm_forward(x, w, 1e-5)[1]
    calls = {"quantize": lambda s: fq.fq_quantize(x, fq.FQ_CRIT_NONE, 0.0, stream=s),
             "quantize_sr": lambda s: fq.fq_quantize_sr(x, 3, stream=s),
             "quantize_topk": lambda s: fq.fq_quantize_topk(x, 1, stream=s),
             "gemm": lambda s: fq.fq_gemm(fq.FQ_OP_NT, q, v, stream=s),
             "codes_to_rowmajor": lambda s: fq.fq_codes_to_rowmajor(q.view("codes"), 200, 384, stream=s),
             "gemm_debug_partials": lambda s: fq.fq_gemm_debug_partials(fq.FQ_OP_NT, q, v, 1, 0, stream=s),
             "ctx_quantize": lambda s: fq.fq_ctx_quantize(x, stream=s),
             "ctx_dequantize": lambda s: fq.fq_ctx_dequantize(*ctx, 200, 384, stream=s),
             "glu_forward": lambda s: fq.fq_glu_forward(x, dy, stream=s),
             "glu_backward": lambda s: fq.fq_glu_backward(dy, ctx, other, stream=s),
             "rmsnorm_forward": lambda s: fq.fq_rmsnorm_forward(x, w, 1e-5, stream=s),
             "rmsnorm_backward": lambda s: fq.fq_rmsnorm_backward(dy, ctx, rstd, w, stream=s)}
    side = torch.cuda.Stream()
    for name, call in calls.items():
        gu.announce(f"{name} on a given stream")
        want = call(None)
        torch.cuda.synchronize()
        got = call(side)
        side.synchronize()
        if isinstance(got, fq.QTensor):
            assert stream_of(got.storage) == side.cuda_stream, name
            assert all(torch.equal(got.view(f), want.view(f)) for f in ("codes", "scales", "mask")), name
        else:
            assert all(stream_of(t) == side.cuda_stream for t in flat(got)), name
            assert all(torch.equal(a, b) for a, b in zip(flat(got), flat(want))), name
