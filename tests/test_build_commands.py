"""The compiler calls behind the ablation libraries, without making them."""
import types

from paper_2503_08040_amd import build


def test_ablation_libraries_compile_first_and_link_objects_alone(monkeypatch):
    """hipcc takes an object behind a .hip file on its command line for source."""
    calls = []

    def run(cmd, **kw):
        calls.append(cmd)
        return types.SimpleNamespace(returncode=0, stderr="")

    monkeypatch.setattr(build.subprocess, "run", run)
    names = ["no_dma", "extra_salu_40"]
    assert build.build_ablations(names, jobs=2) == [build.ablation_lib(n) for n in names]
    compiled = [c for c in calls if "-c" in c]
    linked = [c for c in calls if "-c" not in c]
    assert len(compiled) == len(build.SOURCES) - 1 + len(names) and len(linked) == len(names)
    assert all("-shared" not in c and sum(a.endswith(".hip") for a in c) == 1 for c in compiled)
    outputs = [c[c.index("-o") + 1] for c in compiled]
    assert len(set(outputs)) == len(outputs)
    for c in linked:
        assert "-shared" in c and not any(a.endswith(".hip") for a in c)
        objects = [a for a in c if a.endswith(".o")]
        assert len(objects) == len(build.SOURCES) and set(objects) <= set(outputs)
    for n in names:
        assert sum(all(f in c for f in build.ABLATIONS[n]) for c in compiled) == 1
