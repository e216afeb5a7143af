"""The libraries need neither g++ nor torch's headers: they are linked where _tensors.so, which does, cannot be built (no GPU)."""
import pytest

from paper_2603_06588_amd import build


def test_libraries_are_linked_where_the_front_end_does_not_build(monkeypatch, tmp_path):
    ran = []

    def no_headers():
        raise RuntimeError("g++ failed: no headers")
    monkeypatch.setattr(build, "OBJ", str(tmp_path))
    monkeypatch.setattr(build, "_run", ran.append)
    monkeypatch.setattr(build, "_build_tensors", no_headers)
    with pytest.raises(RuntimeError, match="no headers"):
        build.build_lib()
    linked = [cmd[cmd.index("-o") + 1] for cmd in ran if "-shared" in cmd]
    assert linked == [build.LIB, build.BENCH_LIB]
