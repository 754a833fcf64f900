"""Products of microscaled matrices at both ends of binary32's range.

Low end, tolerance: whatever the order inside an instruction, each of a block's 128 products and its sum with the accumulator
is cut to a multiple of 2^-149 at the worst, and so is each of at most 32 additions that join the parts of a split
contraction: (129 n + 32) 2^-149 for n blocks of 128, beside the bound of test_gpu_mx_gemm, (n + 33) 2^-23 of the sum of
magnitudes.  A bf16 result is off by 2^-8 of itself more, or by half of the smallest bf16 number, 2^-134.
High end: an output whose sum of magnitudes stays below the range is computed as anywhere; one that is beyond the range
comes out infinite or, where parts of both signs pass it on the way, NaN."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_08040_amd as fq
from tests import gpu_util as gu
from tests.test_gpu_mx_gemm import F64, values

MOST = float(torch.finfo(torch.float32).max)


def scaled(rows, cols, e, seed, positive=False):
    """Normal values times 2^e, also where 2^e is no bf16 number."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, cols), device="cuda", generator=g).to(F64)
    return ((x.abs() if positive else x) * 2.0 ** e).to(torch.bfloat16)


def bound(a, b, dtype):
    n = -(-a.shape[1] // 128)
    size = a.abs() @ b.abs().T
    t = (n + 33) * 2.0 ** -23 * size + (129 * n + 32) * 2.0 ** -149
    return t if dtype == torch.float32 else t + 2.0 ** -8 * ((a @ b.T).abs() + t) + 2.0 ** -134


# (compute units the planner is told of, M, N): contractions split over wavefronts, and tiles through LDS
FORMS = [(256, 20, 40, fq.FQ_MX_FORM_32x32), (1, 300, 260, fq.FQ_MX_FORM_128x128)]


@pytest.mark.parametrize("cus,M,N,tiles", FORMS)
@pytest.mark.parametrize("K", [32, 400])
def test_small_results(cus, M, N, tiles, K, monkeypatch):
    """Results around and below the smallest normal number keep their bits down to 2^-149; both operands at their lowest
    scales give 0."""
    monkeypatch.setenv("FQ_GEMM_CUS", str(cus))
    for ea, eb in [(-126, 0), (-100, -30), (-66, -66), (-20, -115), (-70, -72), (-130, -131)]:
        gu.announce(f"mx product of values around 2^{ea} and 2^{eb}, {M}x{N}x{K}")
        A, B = fq.fq_mx_quantize(scaled(M, K, ea, 1)), fq.fq_mx_quantize(scaled(N, K, eb, 2))
        assert fq.fq_mx_gemm_form(M, N, K)[0] in (tiles, fq.FQ_MX_FORM_128x256)
        a, b = values(A, fq.FQ_MX_ROWS), values(B, fq.FQ_MX_ROWS)
        for dt in (torch.float32, torch.bfloat16):
            got = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B, out_dtype=dt).to(F64)
            assert not ((got - a @ b.T).abs() > bound(a, b, dt)).any(), (ea, eb, dt)
        if ea + eb > -140:
            f32 = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B)
            assert ((f32 != 0) & (f32.abs() < 2.0 ** -126)).any() or ea + eb > -128
        if ea + eb < -200:
            assert not got.any()


@pytest.mark.parametrize("cus,M,N,tiles", FORMS)
@pytest.mark.parametrize("K", [32, 400])
def test_large_results(cus, M, N, tiles, K, monkeypatch):
    monkeypatch.setenv("FQ_GEMM_CUS", str(cus))
    for ea, eb in [(60, 60), (124, -1), (63, 62), (64, 62), (63, 64), (120, 120)]:
        for positive in (False, True):
            gu.announce(f"mx product of values around 2^{ea} and 2^{eb}, {M}x{N}x{K}")
            A = fq.fq_mx_quantize(scaled(M, K, ea, 3, positive))
            B = fq.fq_mx_quantize(scaled(N, K, eb, 4, positive))
            a, b = values(A, fq.FQ_MX_ROWS), values(B, fq.FQ_MX_ROWS)
            want, size = a @ b.T, a.abs() @ b.abs().T
            for dt in (torch.float32, torch.bfloat16):
                t = bound(a, b, dt)
                got = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B, out_dtype=dt).to(F64)
                inside, beyond = size + t < MOST * (1 - 2.0 ** -8), want.abs() - t > MOST * (1 + 2.0 ** -8)
                assert got[inside].isfinite().all() and not ((got - want).abs()[inside] > t[inside]).any(), (ea, eb, dt)
                assert not got[beyond].isfinite().any(), (ea, eb, dt)
                if positive:
                    assert not got.isnan().any() and (got[beyond] == float("inf")).all()
        # that the operands reach both: 400 products of mean 2^120 * 2 / pi sum up to 2^128, some below it
        assert ea + eb > 120 or (inside.all() if K == 32 else inside.any())
        assert ea + eb < 200 or beyond.all()


def test_small_tokens_through_the_linear_layer():
    """X quantized on its way into the product: the same bits at the low end."""
    for e, ew in [(-126, -10), (-133, 0), (-100, -35)]:
        for M, K in [(1, 700), (5, 33), (40, 300)]:
            x, W = scaled(M, K, e, 5), fq.fq_mx_quantize(scaled(90, K, ew, 6))
            for rule in (fq.FQ_MX_FLOOR, fq.FQ_MX_COVER):
                y = fq.fq_mx_linear(x, W, rule=rule)
                assert torch.equal(y, fq.fq_mx_gemm(fq.FQ_OP_NT, fq.fq_mx_quantize(x, rule=rule), W))
