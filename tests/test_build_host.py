"""The build step with compilers that are replaced: what is written where, and what it needs."""

import os
import subprocess
import sys

import pytest

from paper_2609_33645_b200 import build


class Compilers:
    """Stands in for subprocess.run: writes the output file, and remembers what was asked for."""

    def __init__(self, monkeypatch):
        self.calls, self.fails, self.seen = [], False, []
        monkeypatch.setattr(build.subprocess, "run", self)

    def __call__(self, cmd, **kw):
        out = cmd[cmd.index("-o") + 1]
        self.calls.append((os.path.basename(cmd[0]), out))
        with open(out, "w") as f:
            f.write("half")
        self.seen.append(open(build.MARSHAL_PATH).read() if os.path.exists(build.MARSHAL_PATH) else None)
        if not self.fails:
            with open(out, "w") as f:
                f.write("whole")
        return subprocess.CompletedProcess(cmd, int(self.fails), "", "no such luck")


@pytest.fixture
def tree(monkeypatch, tmp_path):
    monkeypatch.setattr(build, "MARSHAL_PATH", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "OBJ_DIR", str(tmp_path / "build" / "obj"))
    return tmp_path


def test_the_module_is_moved_into_place_when_it_is_whole(tree, monkeypatch):
    c = Compilers(monkeypatch)
    (tree / "_marshal.so").write_text("old")
    build.build_marshal()
    assert c.seen == ["old"] and (tree / "_marshal.so").read_text() == "whole"
    c.fails = True
    (tree / "_marshal.so.built_for").unlink()
    with pytest.raises(RuntimeError, match="no such luck"):
        build.build_marshal()
    assert (tree / "_marshal.so").read_text() == "whole"
    assert sorted(p.name for p in tree.iterdir()) == ["_marshal.so"]        # no parts are left


def test_a_copied_tree_is_built_for_its_own_torch(tree, monkeypatch):
    import torch

    c = Compilers(monkeypatch)
    (tree / "_marshal.so").write_text("made elsewhere")                     # nothing says for which torch
    build.build_marshal()
    assert len(c.calls) == 1
    build.build_marshal()
    assert len(c.calls) == 1                                                # up to date
    monkeypatch.setattr(torch, "__version__", "0.0")
    build.build_marshal()
    assert len(c.calls) == 2


def test_the_library_needs_no_torch(tree, monkeypatch, capsys):
    c = Compilers(monkeypatch)
    monkeypatch.setitem(sys.modules, "torch", None)                         # import torch fails
    assert build.build() == str(tree / "lib.so") and (tree / "lib.so").read_text() == "whole"
    assert len(c.calls) == len(build.sources()) + 1 and {name for name, _ in c.calls} == {"nvcc"}
    assert all(out.endswith(".part") for _, out in c.calls)
    assert "torch" in capsys.readouterr().err and not (tree / "_marshal.so").exists()
