"""The build: the C library needs nvcc alone, and the Python call module goes with the installed torch."""
import importlib.util
import os

import pytest


@pytest.fixture()
def built(monkeypatch, tmp_path):
    """The build module with its commands recorded instead of run, and outputs in an empty folder."""
    from paper_1905_05686_b200 import build
    ran = []

    def run(cmd, check):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "liblrbi.so"))
    return build, ran, tmp_path


def compilers(ran):
    return {os.path.basename(c[0]) for c in ran}


def test_without_torch(built, monkeypatch, capsys):
    build, ran, at = built
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    assert build.build() == str(at / "liblrbi.so")
    assert os.path.exists(build.LIB) and compilers(ran) == {"nvcc"}
    assert "torch is not installed" in capsys.readouterr().err


def test_another_torch(built, monkeypatch):
    build, ran, _ = built
    build.build()
    assert compilers(ran) == {"nvcc", "g++"}
    ran.clear()
    build.build()
    assert not ran                                      # nothing is out of date
    own = build.calls_path()
    monkeypatch.setattr(build, "torch_version", lambda: "0.0.1")
    build.build()
    assert compilers(ran) == {"g++"} and build.calls_path() != own and os.path.exists(build.calls_path())


def test_every_source_is_compiled_and_linked(built):
    build, ran, _ = built
    build.build()
    sources = {f for f in os.listdir(build.CSRC) if f.endswith(".cu")}
    compiled = [os.path.basename(a) for c in ran for a in c if a.endswith(".cu")]
    assert sorted(compiled) == sorted(sources)
    link = next(c for c in ran if "-shared" in c and os.path.basename(c[0]) == "nvcc")
    assert {os.path.basename(a)[:-2] for a in link if a.endswith(".o")} >= {s[:-3] for s in sources}


def test_binding_loads_what_was_built():
    torch = pytest.importorskip("torch")
    from paper_1905_05686_b200 import binding, build
    assert build.torch_version() == torch.__version__ and binding.CALLS_PATH == build.calls_path()
