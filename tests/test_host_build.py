"""What `python -m paper_1905_10138_amd.build` makes of what it finds (no compiler runs here)."""
import os
import sys

import pytest

from paper_1905_10138_amd import build


@pytest.fixture
def runs(tmp_path, monkeypatch):
    """The commands of a build; those that have a word of `runs.fails` in them fail."""
    class Runs(list):
        fails = ()

        def __call__(self, cmd):
            self.append(cmd)
            if any(word in part for part in cmd for word in self.fails):
                raise RuntimeError("failed: " + " ".join(cmd))
            with open(cmd[cmd.index("-o") + 1], "w") as f:
                f.write("made")
            return ""
    run = Runs()
    monkeypatch.setattr(build, "_run", run)
    monkeypatch.setattr(build, "hipcc_path", lambda: "/opt/rocm/bin/hipcc")
    for name in ("OBJ_DIR", "LIB_PATH", "EXT_PATH"):
        monkeypatch.setattr(build, name, str(tmp_path / os.path.basename(getattr(build, name))))
    return run


def test_library_and_extension(runs):
    assert build.build_library() == build.LIB_PATH
    assert os.path.exists(build.LIB_PATH) and os.path.exists(build.EXT_PATH)
    # the extension is linked against the library, which has to be there
    outputs = [cmd[cmd.index("-o") + 1] for cmd in runs]
    assert outputs.index(build.LIB_PATH + ".tmp") < outputs.index(build.EXT_PATH + ".tmp")


def test_library_without_torch(runs, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)   # import torch raises
    assert build.build_library() == build.LIB_PATH
    assert os.path.exists(build.LIB_PATH) and not os.path.exists(build.EXT_PATH)
    assert "torch" in capsys.readouterr().out          # and says what is not there
    assert not any("xorenc_torch" in part for cmd in runs for part in cmd)


def test_library_where_the_extension_does_not_compile(runs):
    runs.fails = ("xorenc_torch_fp8.cpp",)
    with pytest.raises(RuntimeError, match="xorenc_torch_fp8"):
        build.build_library()
    assert os.path.exists(build.LIB_PATH) and not os.path.exists(build.EXT_PATH)


def test_no_library_where_it_does_not_compile(runs):
    runs.fails = ("xorenc_moe.hip",)
    with pytest.raises(RuntimeError, match="xorenc_moe"):
        build.build_library()
    assert not os.path.exists(build.LIB_PATH) and not os.path.exists(build.EXT_PATH)
