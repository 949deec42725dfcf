"""What the build runs, with the compilers replaced: the library is plain ROCm and is built
without torch; the layer over torch's tensors is built where torch is."""
import os
import sys

import pytest

from paper_2402_09900_amd import build as b


class Done:
    def __init__(self, args, status=0):
        self.args, self.status = args, status

    def wait(self):
        return self.status


@pytest.fixture
def ran(monkeypatch, tmp_path):
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libmemoroid.so"))
    monkeypatch.setattr(b, "LAYER", str(tmp_path / "_torch_layer.so"))
    monkeypatch.setattr(b, "HERE", str(tmp_path))
    monkeypatch.setattr(b, "sources", lambda: ["a.hip"])
    commands = []

    def run(cmd, verbose):
        commands.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write(cmd[0])
        return Done(cmd)

    monkeypatch.setattr(b, "_run", run)
    return commands


def test_library_without_torch(ran, monkeypatch, tmp_path, capsys):
    for name in [m for m in sys.modules if m == "torch" or m.startswith("torch.")]:
        monkeypatch.delitem(sys.modules, name)
    monkeypatch.setitem(sys.modules, "torch", None)
    assert b.build() == b.LIB
    assert [c[0] for c in ran] == ["hipcc"]
    assert os.listdir(tmp_path) == ["libmemoroid.so"]
    assert "torch" in capsys.readouterr().out


def test_library_and_layer(ran, tmp_path):
    pytest.importorskip("torch")
    assert b.build() == b.LIB
    assert sorted(c[0] for c in ran) == ["g++", "g++", "hipcc"]
    assert sorted(os.listdir(tmp_path)) == ["_torch_layer.so", "libmemoroid.so"]
