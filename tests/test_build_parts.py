"""What building gives where a part of it cannot be built."""
import os
import subprocess

from paper_2409_19256_amd import build as b


def test_library_without_the_torch_module(tmp_path, monkeypatch, capfd):
    """A machine without Python's headers or a usable host compiler still gets the library; an older module does not stay behind."""
    for name in ("LIB", "BENCH_EXE", "TORCH_MODULE"):
        monkeypatch.setattr(b, name, str(tmp_path / name))
    open(b.TORCH_MODULE, "w").write("older")

    def run(cmd, check, cwd):
        if any(str(x).endswith("rollout_torch.cpp") for x in cmd):
            raise subprocess.CalledProcessError(1, cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(b.subprocess, "run", run)
    assert b.build_library(verbose=False) == b.LIB
    assert os.path.exists(b.LIB) and os.path.exists(b.BENCH_EXE) and not os.path.exists(b.TORCH_MODULE)
    assert "_rollout" in capfd.readouterr().err


def test_a_failed_library_is_an_error(tmp_path, monkeypatch):
    import pytest
    for name in ("LIB", "BENCH_EXE", "TORCH_MODULE"):
        monkeypatch.setattr(b, name, str(tmp_path / name))

    def run(cmd, check, cwd):
        raise subprocess.CalledProcessError(1, cmd)

    monkeypatch.setattr(b.subprocess, "run", run)
    with pytest.raises(subprocess.CalledProcessError):
        b.build_library(verbose=False)
