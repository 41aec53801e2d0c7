"""The order of a build: the C library does not wait for what only its torch binding needs."""
import os
import types

import pytest

from paper_2401_06145_amd import build


def test_library_is_linked_where_the_binding_cannot_be(tmp_path, monkeypatch):
    linked = []

    def run(cmd, **_):
        out = cmd[cmd.index("-o") + 1]
        linked.append(out)
        with open(out, "w") as f:
            f.write("library")
        return types.SimpleNamespace(returncode=0, stderr="")

    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path))
    monkeypatch.setattr(build, "TORCH_OPS", str(tmp_path / "ops.so"))
    monkeypatch.setattr(build, "_compile", lambda src: src + ".o")
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    with pytest.raises(RuntimeError, match="torch"):
        build.build()
    assert linked == [build.LIB + ".tmp"] and os.path.exists(build.LIB)
