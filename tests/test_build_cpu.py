"""The compiled calls belong to one interpreter and one torch; a build after either changed makes them anew."""
import os
import subprocess
import sys

import pytest
import torch

import paper_1810_09868_b200 as p
from paper_1810_09868_b200 import build


def test_the_path_names_interpreter_and_torch(monkeypatch):
    paths = {build.calls_path()}
    monkeypatch.setattr(torch, "__version__", "9.9.9+cu999")
    paths.add(build.calls_path())
    monkeypatch.setattr(torch.version, "git_version", "0123456789")
    paths.add(build.calls_path())
    monkeypatch.setattr(sys.implementation, "cache_tag", "cpython-399")
    paths.add(build.calls_path())
    assert len(paths) == 4 and all(os.path.dirname(q) == build.PKG for q in paths)


def test_another_torch_is_built_for_and_never_loaded_by_chance(monkeypatch, tmp_path):
    made = []

    def compiler(cmd, check):
        assert check
        made.append(cmd[cmd.index("-o") + 1])
        open(made[-1], "wb").close()

    monkeypatch.setattr(build, "PKG", str(tmp_path))
    monkeypatch.setattr(subprocess, "run", compiler)
    first = build.build_calls()
    assert build.build_calls() == first and len(made) == 1 and made[0] != first and os.listdir(tmp_path) == [os.path.basename(first)]
    monkeypatch.setattr(torch, "__version__", "9.9.9+cu999")  # newer than no source, and yet not built for
    monkeypatch.setattr(p.binding, "_tensor_calls", None)
    monkeypatch.setattr(p.binding, "load", lambda: None)
    with pytest.raises(RuntimeError, match="9.9.9.*build"):
        p.binding._calls()
    second = build.build_calls()
    assert second != first and len(made) == 2 and os.path.exists(second)


def test_what_is_built_here_loads():
    import __graft_entry__ as g
    g.build()
    calls = p.binding._calls()
    assert calls.logprobs(1, 2, 3) is None and os.path.samefile(calls.__file__, build.calls_path())
