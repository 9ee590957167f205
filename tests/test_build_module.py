"""The build of the worker-side operators' Python module: made again for another torch, and no condition for the aggregation."""
import os
import shutil

import pytest

from paper_1907_12205_b200 import binding, build


@pytest.fixture
def apart(tmp_path, monkeypatch):
    """The built library, and a place of its own for the module."""
    build.build()
    monkeypatch.setattr(build, "MODULE", str(tmp_path / "_worker.so"))
    monkeypatch.setattr(build, "MODULE_STAMP", str(tmp_path / "worker_module.txt"))
    runs = []

    def fake_run(cmd, **kw):
        runs.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return type("R", (), {"returncode": 0, "stdout": "", "stderr": ""})

    monkeypatch.setattr(build.subprocess, "run", fake_run)
    return runs


def test_the_module_is_made_again_for_another_torch_and_only_then(apart, monkeypatch):
    build.build()
    assert len(apart) == 1 and apart[0][0] == "g++"
    build.build()
    assert len(apart) == 1
    monkeypatch.setattr(build, "_module_stamp", lambda: "another torch\n")
    build.build()
    assert len(apart) == 2 and open(build.MODULE_STAMP).read() == "another torch\n"
    build.build()
    assert len(apart) == 2


def test_without_a_compiler_the_aggregation_is_built_all_the_same(apart, monkeypatch):
    real = shutil.which
    monkeypatch.setattr(shutil, "which", lambda name, *a: None if name == "g++" else real(name, *a))
    with pytest.warns(UserWarning, match="no g\\+\\+"):
        lib = build.build()
    assert lib == build.LIB and os.path.exists(lib) and apart == [] and not os.path.exists(build.MODULE)


def test_without_the_module_its_operators_say_so(monkeypatch):
    import sys
    import torch
    build.build()
    monkeypatch.setattr(binding, "_worker_module", None)
    monkeypatch.setitem(sys.modules, "paper_1907_12205_b200._worker", None)
    monkeypatch.delattr("paper_1907_12205_b200._worker", raising=False)
    with pytest.raises(ImportError):
        binding.detox_checkpoint_pack(torch.zeros(2, 2))
