"""CPU: the C library is built where the Python binding's compiled part cannot be."""
import pytest


@pytest.fixture
def commands(monkeypatch, tmp_path):
    from paper_2506_02024_amd import build

    ran = []

    def run(cmd, verbose):
        if any(c.endswith("marshal.cpp") for c in cmd):
            raise RuntimeError("no Python.h")
        ran.append(cmd)
    monkeypatch.setattr(build, "_run", run)
    monkeypatch.setattr(build, "PKG", str(tmp_path))
    return build, ran


def _linked(build, ran):
    return [cmd for cmd in ran if "-shared" in cmd and cmd[cmd.index("-o") + 1] == build.LIB]


@pytest.mark.parametrize("missing", ["headers", "torch"])
def test_the_library_is_linked_before_the_error(commands, monkeypatch, missing):
    build, ran = commands
    if missing == "torch":
        def no_torch():
            raise ImportError("no torch")
        monkeypatch.setattr(build, "_marshal_command", no_torch)
    with pytest.raises(RuntimeError, match="the library is built"):
        build.build_library()
    assert len(ran) == len(build.sources()) + 1 and len(_linked(build, ran)) == 1 and ran[-1] in _linked(build, ran)


def test_the_library_alone(commands):
    build, ran = commands
    assert build.build_library(binding=False) == build.LIB
    assert len(ran) == len(build.sources()) + 1 and len(_linked(build, ran)) == 1


def test_a_source_that_does_not_compile_is_an_error(commands, monkeypatch):
    build, ran = commands

    def run(cmd, verbose):
        if "-c" in cmd:
            raise RuntimeError("hipcc failed")
        ran.append(cmd)
    monkeypatch.setattr(build, "_run", run)
    with pytest.raises(RuntimeError, match="hipcc failed"):
        build.build_library(binding=False)
    assert not _linked(build, ran)
