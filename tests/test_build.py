"""The order of the build: the library does not wait for the Python binding's native part."""
import os

import pytest

from paper_2606_02091_amd import build as b


def planned(tmp_path, monkeypatch, fails):
    """A build whose compilers only write their outputs; the commands that `fails` names raise."""
    lib = tmp_path / "_lib"
    monkeypatch.setattr(b, "LIBDIR", str(lib))
    monkeypatch.setattr(b, "LIB", str(lib / "libdflare.so"))
    monkeypatch.setattr(b, "BINDING", str(lib / "_binding.so"))
    monkeypatch.setattr(b, "hipcc", lambda: "hipcc")

    def run(cmd, verbose):
        if fails in cmd:
            raise RuntimeError("build failed")
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write(cmd[0])
    monkeypatch.setattr(b, "_run", run)
    return lib


def test_library_is_built_where_the_binding_is_not(tmp_path, monkeypatch):
    lib = planned(tmp_path, monkeypatch, "g++")
    lib.mkdir()
    (lib / "_binding.so").write_text("of an older library")
    with pytest.raises(RuntimeError, match="without _binding.so"):
        b.build()
    assert os.listdir(lib) == ["libdflare.so"]


def test_library_is_built_without_torch(tmp_path, monkeypatch):
    def no_torch(out):
        raise ImportError("No module named 'torch'")
    lib = planned(tmp_path, monkeypatch, None)
    monkeypatch.setattr(b, "_binding_command", no_torch)
    with pytest.raises(RuntimeError, match="No module named 'torch'"):
        b.build()
    assert os.listdir(lib) == ["libdflare.so"]


def test_both_parts_are_built(tmp_path, monkeypatch):
    lib = planned(tmp_path, monkeypatch, None)
    assert b.build() == str(lib / "libdflare.so")
    assert sorted(os.listdir(lib)) == ["_binding.so", "libdflare.so"]


def test_a_library_that_fails_leaves_both_as_they_were(tmp_path, monkeypatch):
    lib = planned(tmp_path, monkeypatch, "-c")  # (compiles a source of the library)
    lib.mkdir()
    for part in ("libdflare.so", "_binding.so"):
        (lib / part).write_text("before")
    with pytest.raises(RuntimeError):
        b.build()
    assert all((lib / part).read_text() == "before" for part in ("libdflare.so", "_binding.so"))
