"""The benchmark's count of HBM traffic belongs to the GEMM source and to the headers that it includes."""
import hashlib
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import bench


def test_a_change_of_an_included_header_makes_the_count_stale(tmp_path, monkeypatch):
    files = {"k.hip": '#include <vector>\n#include "a.h"\n  #include "sub/b.h"\nkernel\n', "a.h": '#pragma once\n#include "sub/b.h"\nint a;\n',
             "sub/b.h": '#include "../a.h"\nint b;\n', "c.h": "int c;\n"}
    (tmp_path / "sub").mkdir()
    for name, text in files.items():
        (tmp_path / name).write_text(text)
    # each once, in the order in which they are first included
    want = hashlib.sha256("".join(files[n] for n in ("k.hip", "a.h", "sub/b.h")).encode()).hexdigest()
    prof = tmp_path / "p.md"
    prof.write_text(f"gemm_traffic: workload=w bytes_per_launch=77 fq_gemm_hip_sha256={want}\n")
    monkeypatch.setattr(bench, "GEMM_SOURCE", str(tmp_path / "k.hip"))
    monkeypatch.setattr(bench, "TRAFFIC_PROFILE", str(prof))
    assert bench.measured_gemm_traffic("w") == 77
    (tmp_path / "c.h").write_text("int d;\n")              # not included
    assert bench.measured_gemm_traffic("w") == 77
    for name in ("a.h", "sub/b.h", "k.hip"):
        (tmp_path / name).write_text(files[name] + "int more;\n")
        assert bench.measured_gemm_traffic("w") is None, name
        (tmp_path / name).write_text(files[name])
        assert bench.measured_gemm_traffic("w") == 77
    os.remove(tmp_path / "a.h")
    assert bench.measured_gemm_traffic("w") is None


def test_the_headers_of_the_gemm_source_are_found():
    assert [os.path.basename(f) for f in bench.source_and_headers(bench.GEMM_SOURCE)] == \
        ["fq_gemm.hip", "fq_device.h", "fq_gemm_unit.h", "fq_kernels.h"]
