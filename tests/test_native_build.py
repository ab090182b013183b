"""The native module belongs to one Python and one torch: a build for another one is made again, and is not used."""
import os

import pytest


@pytest.fixture
def build(monkeypatch, tmp_path):
    from paper_2602_11937_b200 import build as b
    calls = []

    def compiler(cmd, **kw):
        calls.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(b.subprocess, "check_call", compiler)
    monkeypatch.setattr(b, "LIB_DIR", str(tmp_path / "lib"))
    monkeypatch.setattr(b, "CALL_LIB", str(tmp_path / "lib" / "_puzzle_call.so"))
    monkeypatch.setattr(b, "CALL_STAMP", str(tmp_path / "_build" / "call.txt"))
    b.calls = calls
    yield b
    del b.calls


def test_a_new_torch_or_python_builds_again(build, monkeypatch):
    build.build_call()
    build.build_call()
    assert len(build.calls) == 1                                    # up to date
    monkeypatch.setattr(build, "call_target", lambda: "python 9.9 torch 9.9.9")
    build.build_call()
    assert len(build.calls) == 2
    build.build_call()
    assert len(build.calls) == 2
    os.remove(build.CALL_STAMP)                                     # built by an older version of this file
    build.build_call()
    assert len(build.calls) == 3
    build.build_call(force=True)
    assert len(build.calls) == 4


def test_the_target_names_what_runs():
    import platform

    import torch
    from paper_2602_11937_b200 import binding, build
    assert build.call_target() == "python %s.%s torch %s" % (*platform.python_version_tuple()[:2], torch.__version__)
    assert binding._native().built_for == build.call_target()


def test_a_module_for_another_torch_is_not_used(monkeypatch):
    import torch
    from paper_2602_11937_b200 import binding
    binding._native()
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_call", None)
    monkeypatch.setattr(torch, "__version__", "1.0")
    for _ in range(2):
        with pytest.raises(RuntimeError, match="was built for python .* torch .*, this is python .* torch 1.0: build it again"):
            binding._native()
