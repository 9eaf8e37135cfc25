"""When the binding's extension is compiled again, and what the library's build needs (no compiler runs here)."""
import os
import types

import pytest

from paper_2605_15250_b200 import build as gbuild


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    """Commands that would have run; each writes its output file with the stamp of this torch and Python."""
    ran = []

    def run(cmd, **kwargs):
        ran.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "wb") as f:
            f.write(b"\0" + gbuild._marshal_stamp() + b"\0")
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(gbuild.subprocess, "run", run)
    monkeypatch.setattr(gbuild, "MARSHAL_PATH", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(gbuild, "LIB_PATH", str(tmp_path / "libgqla.so"))
    return ran


def test_extension_of_another_torch_or_python_is_compiled_again(compilers):
    path = gbuild.build_marshal()
    assert len(compilers) == 1 and gbuild.build_marshal() == path and len(compilers) == 1
    for other in (b"", b"built for torch 1.0.0, Python 3.12;", gbuild._marshal_stamp().replace(b"Python 3.", b"Python 2.")):
        with open(path, "wb") as f:
            f.write(other)
        gbuild.build_marshal()
        with open(path, "rb") as f:
            assert gbuild._marshal_stamp() in f.read()
    assert len(compilers) == 4
    os.utime(path, (1, 1))
    gbuild.build_marshal()
    assert len(compilers) == 5
    gbuild.build_marshal(force=True)
    assert len(compilers) == 6


def test_the_extension_that_is_built_carries_the_stamp():
    """The real one, by its own words."""
    gbuild.build()
    from paper_2605_15250_b200 import binding as B

    assert B._marshal().stamp.encode() == gbuild._marshal_stamp()
    with open(gbuild.MARSHAL_PATH, "rb") as f:
        assert gbuild._marshal_stamp() in f.read()


def test_extension_of_another_torch_or_python_is_not_loaded(monkeypatch, tmp_path):
    from paper_2605_15250_b200 import binding as B

    other = tmp_path / "_marshal.so"
    other.write_bytes(b"built for torch 1.0.0, Python 3.12;")
    monkeypatch.setattr(gbuild, "MARSHAL_PATH", str(other))
    monkeypatch.setattr(B, "_marshal_module", None)
    with pytest.raises(B.GqlaError, match="another torch or Python.*build it again"):
        B._marshal()


def test_library_comes_first_and_alone_without_torch(compilers, monkeypatch):
    gbuild.build()
    assert [os.path.basename(c[c.index("-o") + 1]).split(".so")[0] for c in compilers] == ["libgqla", "_marshal"]
    compilers.clear()
    find = gbuild.importlib.util.find_spec
    monkeypatch.setattr(gbuild.importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    gbuild.build(force=True)
    assert len(compilers) == 1


def test_cuda_headers_are_those_of_the_compiler(compilers, monkeypatch):
    monkeypatch.setenv("NVCC", "/opt/cuda-x/bin/nvcc")
    gbuild.build(force=True)
    assert compilers[0][0] == "/opt/cuda-x/bin/nvcc" and "-I/opt/cuda-x/include" in compilers[1]
