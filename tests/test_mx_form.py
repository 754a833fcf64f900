"""fq_mx_gemm_form at the ends of its ranges: outputs that fq_mx_gemm refuses, sizes near 2^31, many compute units, the
longest contraction of the large tiles."""
import ctypes as C

import pytest

import paper_2503_08040_amd as fq

MOST = 2 ** 31 - 1


def status(M, N, K, cus=256):
    return fq.lib().fq_mx_gemm_form(M, N, K, cus, (C.c_int32 * 2)())


def refused_by_the_product(M, N):
    """Whether fq_mx_gemm refuses an M x N output of an empty contraction (which launches nothing: C is NULL)."""
    a, b = fq.fq_mx_tensor(), fq.fq_mx_tensor()
    for t, n in ((a, M), (b, N)):
        assert fq.lib().fq_mx_bind(C.c_void_p(0x100000), n, 0, fq.FQ_MX_ROWS, C.byref(t)) == fq.FQ_OK
    s = fq.lib().fq_mx_gemm(fq.FQ_OP_NT, C.byref(a), C.byref(b), None, fq.FQ_OUT_F32, max(N, 1), None)
    assert s in (fq.FQ_ERR_SHAPE, fq.FQ_ERR_NULL) or M * N == 0
    return s == fq.FQ_ERR_SHAPE


@pytest.mark.parametrize("M,N", [(MOST, 40), (40, MOST), (MOST, MOST), (2 ** 27, 64), (2 ** 27 + 1, 64), (64, 2 ** 27), (1, 2 ** 27 + 1),
                                 (MOST - 199, 40), (2 ** 18, 2 ** 17), (2 ** 18, 2 ** 17 + 1), (2 ** 22 + 64, 128 * 64),
                                 (2 ** 18 - 5, 2 ** 17 - 7), (MOST, 0), (0, MOST)])
def test_a_form_is_given_for_outputs_that_can_be_computed(M, N):
    for K in (0, 1, 256, MOST):
        assert status(M, N, K) == (fq.FQ_ERR_SHAPE if refused_by_the_product(M, N) else fq.FQ_OK), K


@pytest.mark.parametrize("M,N,K,small", [(2048, 2048, 2048, fq.FQ_MX_FORM_32x32), (1, 11008, 4096, fq.FQ_MX_FORM_32x32),
                                         (128, 2 ** 20, 256, fq.FQ_MX_FORM_32x64)])
def test_more_compute_units_never_turn_the_choice_round(M, N, K, small):
    """Tiles get smaller with the number of units and stay small, up to the largest number there is."""
    edges = {fq.FQ_MX_FORM_32x32: 32 * 32, fq.FQ_MX_FORM_32x64: 32 * 64, fq.FQ_MX_FORM_64x64: 64 * 64,
             fq.FQ_MX_FORM_128x128: 128 * 128, fq.FQ_MX_FORM_128x256: 128 * 256, fq.FQ_MX_FORM_256x256: 256 * 256}
    units = [1, 256, 2 ** 14, 2 ** 16, 2 ** 20, 2 ** 24, 2 ** 29, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 5, MOST]
    sizes = [edges[fq.fq_mx_gemm_form(M, N, K, u)[0]] for u in units]
    assert sizes == sorted(sizes, reverse=True)
    assert fq.fq_mx_gemm_form(M, N, K, MOST)[0] == small
    one = [fq.fq_mx_gemm_form(M, N, K, u)[1] for u in units[3:]]
    assert len(set(one)) == 1


@pytest.mark.parametrize("M,N", [(8192, 8192), (512, 2 ** 18), (2 ** 18, 2 ** 17)])
def test_the_launch_stays_within_the_grid_for_any_number_of_compute_units(M, N):
    """Workgroups times threads of the smallest tiles chosen are below 2^32."""
    threads = {fq.FQ_MX_FORM_32x32: (32, 32, 512), fq.FQ_MX_FORM_32x64: (32, 64, 512), fq.FQ_MX_FORM_64x64: (64, 64, 256)}
    for u in (2 ** 16, 2 ** 24, 2 ** 27, 2 ** 30, MOST):
        for K in (64, 2 ** 20):
            r, c, n = threads.get(fq.fq_mx_gemm_form(M, N, K, u)[0], (128, 128, 256))
            assert -(-M // r) * -(-N // c) * n < 2 ** 32, (u, K)


def test_contractions_whose_offsets_pass_31_bits_leave_the_large_tiles():
    """A strip's codes over 2^21 blocks of 128 are 2 GiB, the reach of the large tiles' 32-bit offsets."""
    block = 128
    for cus, M, N, large in [(1, 512, 512, fq.FQ_MX_FORM_256x256), (4, 400, 256, fq.FQ_MX_FORM_128x128)]:
        assert fq.fq_mx_gemm_form(M, N, (2 ** 21 - 1) * block, cus)[0] in (large, fq.FQ_MX_FORM_128x256)
        for K in ((2 ** 21 - 1) * block + 1, 2 ** 21 * block, MOST):
            assert fq.fq_mx_gemm_form(M, N, K, cus)[0] == fq.FQ_MX_FORM_64x64, K
