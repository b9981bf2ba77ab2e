"""Building: libconef.so needs hipcc alone; _face.so, which only calls on torch tensors go through, may stay unbuilt until they are made."""
import subprocess
import sys

import pytest

from paper_2312_08538_amd import build


@pytest.fixture
def built(monkeypatch, tmp_path):
    """The commands that a build runs (none is run), by their first word; `fails`: an exception for one of them."""
    ran, fails = [], {}

    def run(cmd, **_):
        ran.append(cmd)
        if cmd[0] in fails:
            raise fails[cmd[0]]
        return subprocess.CompletedProcess(cmd, 0)

    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "FACE", str(tmp_path / "_face.so"))
    monkeypatch.setenv("CXX", "host-compiler")
    return ran, fails


def linked(ran):
    return [c for c in ran if c[0] == build.HIPCC and "-shared" in c]


def test_every_part_is_built(built):
    ran, _ = built
    assert build.build_library() == build.LIB
    assert len(ran) == len(build.SOURCES) + 2 and len(linked(ran)) == 1 and [c[0] for c in ran].count("host-compiler") == 1


@pytest.mark.parametrize("why", ["no torch", "no compiler", "no headers"])
def test_the_library_is_built_without_what_only_the_face_needs(built, monkeypatch, capfd, why):
    ran, fails = built
    open(build.FACE, "w").close()                               # an earlier build's, which need not fit the library any more
    if why == "no torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        fails["host-compiler"] = FileNotFoundError("host-compiler") if why == "no compiler" else subprocess.CalledProcessError(1, "host-compiler")
    assert build.build_library() == build.LIB
    assert len(linked(ran)) == 1
    said = capfd.readouterr().err
    assert "_face.so" in said
    with pytest.raises(FileNotFoundError):
        open(build.FACE)


def test_an_error_in_a_kernel_is_one(built):
    _, fails = built
    fails[build.HIPCC] = subprocess.CalledProcessError(1, build.HIPCC)
    with pytest.raises(subprocess.CalledProcessError):
        build.build_library()
