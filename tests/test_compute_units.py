"""The number of compute units that the choices of tiles assume is found in one place."""
import ctypes as C
import glob
import os

import pytest

import paper_2503_08040_amd as fq
from paper_2503_08040_amd import build


def test_one_place_reads_it():
    readers = [os.path.basename(f) for f in glob.glob(os.path.join(build.CSRC, "*.*"))
               if "std::getenv" in open(f).read() or "MultiprocessorCount" in open(f).read()]
    assert readers == ["fq_gemm.hip"]


@pytest.mark.parametrize("cus", [1, 8, 64, 256, 304])
def test_the_variable_counts_for_every_choice(cus, monkeypatch):
    queries = [lambda n: fq.fq_gemm_tile_plan(5120, 5120, n), lambda n: fq.fq_gemm_path(2048, 2048, n),
               lambda n: fq.fq_gemm_form(2048, 2048, 2048, n), lambda n: fq.fq_mx_gemm_form(2048, 2048, 2048, n)]
    want = [q(cus) for q in queries]
    monkeypatch.setenv("FQ_GEMM_CUS", str(cus))
    assert [q(0) for q in queries] == want


def test_without_a_device_the_microscaled_choice_says_so(monkeypatch):
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    monkeypatch.delenv("FQ_GEMM_CUS", raising=False)
    for _ in range(2):
        assert fq.lib().fq_mx_gemm_form(64, 64, 64, 0, (C.c_int32 * 2)()) == fq.FQ_ERR_HIP
