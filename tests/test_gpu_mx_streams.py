"""Microscaled calls on streams that the caller gives: whose blocks their memory is, and captured on a forked stream."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_08040_amd as fq
from tests import gpu_util as gu


def matrix(rows, cols, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((rows, cols), device="cuda", generator=g).to(torch.bfloat16)


def stream_of(t):
    """The stream for which the allocator took the memory of a tensor."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


def test_memory_comes_from_the_given_streams_blocks(monkeypatch):
    x, few, W = matrix(40, 5000, 1), matrix(3, 5000, 2), fq.fq_mx_quantize(matrix(300, 5000, 3), sides=fq.FQ_MX_BOTH)
    q = fq.fq_mx_quantize(x, sides=fq.FQ_MX_BOTH)
    assert not fq.fq_mx_gemm_form(40, 300, 5000)[1]                    # so Q(x) is stored
    spaces, make = [], fq.MxTensor
    monkeypatch.setattr(fq, "MxTensor", lambda *a: spaces.append(make(*a)) or spaces[-1])
    calls = [lambda s: fq.fq_mx_quantize(x, sides=fq.FQ_MX_BOTH, stream=s).storage,
             lambda s: fq.fq_mx_quantize_sr(x, 5, sides=fq.FQ_MX_BOTH, stream=s).storage,
             lambda s: fq.fq_mx_dequantize(q, fq.FQ_MX_COLS, stream=s), lambda s: fq.fq_mx_gemm(fq.FQ_OP_NT, q, W, stream=s),
             lambda s: fq.fq_mx_linear(x, W, stream=s), lambda s: fq.fq_mx_linear(few, W, stream=s)]
    side = torch.cuda.Stream()
    want = [c(None) for c in calls]
    torch.cuda.synchronize()
    del spaces[:]
    gu.announce("mx calls on a given stream")
    got = [c(side) for c in calls]
    assert torch.cuda.current_stream() != side
    assert all(stream_of(t) == side.cuda_stream for t in got)
    assert len(spaces) == 3 and all(stream_of(s.storage) == side.cuda_stream for s in spaces)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got[2:], want[2:]))


def test_captured_on_a_forked_stream():
    """With the space for Q(x) and the output allocated in the capture."""
    x, W = matrix(40, 5000, 1), fq.fq_mx_quantize(matrix(300, 5000, 2))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    fq.fq_mx_linear(x, W, stream=side)
    torch.cuda.synchronize()
    gu.announce("capturing an mx call on a forked stream")
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        y = fq.fq_mx_linear(x, W, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        x.copy_(matrix(40, 5000, 10 + rep))
        want = fq.fq_mx_linear(x, W)
        y.zero_()
        with torch.cuda.stream(side):
            torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda")         # what eager work there takes and gives back
        torch.cuda.synchronize()
        gu.announce(f"replay {rep}")
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
