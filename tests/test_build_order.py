"""The library is built whether or not its tensor-level entry can be: that one needs torch's headers and the host compiler."""
import os
import subprocess

import pytest

from paper_2409_09242_amd import build as BLD


class _Tools:
    """Stands in for the compilers: writes what -o names, fails for dw_torch.cpp or for the module's link if told to."""

    def __init__(self, fail=()):
        self.fail, self.made = fail, []

    def run(self, cmd, **kw):
        out = cmd[cmd.index("-o") + 1]
        step = "torch" if out.endswith("dw_torch.cpp.o") else "module" if out == BLD.TORCH_LIB else "library" if out == BLD.LIB else "object"
        if step in self.fail:
            return subprocess.CompletedProcess(cmd, 1, "", "no such header")
        with open(out, "w") as f:
            f.write("new")
        self.made.append(step)
        return subprocess.CompletedProcess(cmd, 0, "", "")


@pytest.fixture
def tree(tmp_path, monkeypatch):
    for name, file in (("LIB", "libdw.so"), ("TORCH_LIB", "_dw_torch.so"), ("STAMP", "stamp"), ("OBJ", "obj")):
        monkeypatch.setattr(BLD, name, str(tmp_path / file))
    monkeypatch.setattr(BLD, "check_transposed_reads", lambda: "")
    monkeypatch.setattr(BLD, "_hipcc", lambda: "hipcc")
    for old in (BLD.LIB, BLD.TORCH_LIB):
        with open(old, "w") as f:
            f.write("old")
    return monkeypatch


@pytest.mark.parametrize("step", ["torch", "module"])
def test_without_the_module_there_is_the_library(tree, step):
    tools = _Tools(fail=(step,))
    tree.setattr(BLD.subprocess, "run", tools.run)
    with pytest.raises(RuntimeError, match="no such header"):
        BLD.build(verbose=False)
    assert open(BLD.LIB).read() == "new" and not os.path.exists(BLD.STAMP)
    assert not os.path.exists(BLD.TORCH_LIB)                # an old module does not stay beside a new library


def test_both(tree):
    tools = _Tools()
    tree.setattr(BLD.subprocess, "run", tools.run)
    BLD.build(verbose=False)
    assert open(BLD.LIB).read() == "new" and open(BLD.TORCH_LIB).read() == "new" and os.path.exists(BLD.STAMP)
    assert tools.made.index("library") < tools.made.index("module")


def test_a_failing_library_leaves_everything(tree):
    tools = _Tools(fail=("object",))
    tree.setattr(BLD.subprocess, "run", tools.run)
    with pytest.raises(RuntimeError):
        BLD.build(verbose=False)
    assert open(BLD.LIB).read() == "old" and open(BLD.TORCH_LIB).read() == "old" and not os.path.exists(BLD.STAMP)
