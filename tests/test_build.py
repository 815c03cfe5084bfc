"""What build() makes on machines that lack something, with the compilers replaced by a recorder that writes empty files."""
import os
import subprocess

import pytest

from paper_2501_05633_b200 import binding


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    """A package directory without built files, and commands that succeed unless `fails` says otherwise; the list of them."""
    for name in ("_LIB", "_TRAIN_LIB", "_TRAIN_MODULE"):
        monkeypatch.setattr(binding, name, str(tmp_path / os.path.basename(getattr(binding, name))))
    seen = []

    class Compiler:
        fails = staticmethod(lambda cmd: False)

        def __init__(self, cmd, **kw):
            seen.append(cmd)
            self.args, self.returncode = cmd, 1 if Compiler.fails(cmd) else 0
            if not self.returncode:
                open(cmd[cmd.index("-o") + 1], "w").close()

        def wait(self):
            return self.returncode

    def run(cmd, check=False, **kw):
        done = Compiler(cmd)
        if check and done.returncode:
            raise subprocess.CalledProcessError(done.returncode, cmd)
        return done

    monkeypatch.setattr(binding.subprocess, "Popen", Compiler)
    monkeypatch.setattr(binding.subprocess, "run", run)
    return Compiler, seen


def test_everything(compilers, recwarn):
    _, seen = compilers
    assert binding.build() == binding._LIB and not recwarn
    assert all(os.path.exists(f) for f in (binding._LIB, binding._TRAIN_LIB, binding._TRAIN_MODULE))
    before = len(seen)
    binding.build()
    assert len(seen) == before, "nothing is stale"
    binding.build(force=True)
    assert len(seen) == 2 * before


@pytest.mark.parametrize("lacks", ["g++", "Python.h", "torch"])
def test_without_what_the_module_needs(compilers, monkeypatch, lacks):
    """The sparsifier, which needs nvcc alone, is built, with a warning; the training operators' own build raises."""
    which, exists = binding.shutil.which, os.path.exists
    monkeypatch.setattr(binding.shutil, "which", lambda c: None if c == lacks else which(c))
    monkeypatch.setattr(binding.os.path, "exists", lambda f: False if str(f).endswith({"Python.h": "Python.h", "torch": "python_variable.h"}.get(lacks, "\0")) else exists(f))
    with pytest.warns(UserWarning, match="training operators"):
        assert binding.build() == binding._LIB
    assert exists(binding._LIB) and not exists(binding._TRAIN_MODULE)
    with pytest.raises(RuntimeError):
        binding.build_training()


def test_errors_are_raised(compilers):
    """A source that does not compile is an error, but one of the training operators' leaves the sparsifier built."""
    compiler, _ = compilers
    compiler.fails = staticmethod(lambda cmd: any("grouped_matmul" in a for a in cmd))
    with pytest.raises(subprocess.CalledProcessError):
        binding.build()
    assert os.path.exists(binding._LIB)
    compiler.fails = staticmethod(lambda cmd: any(a.endswith("regtopk.cu") for a in cmd))
    with pytest.raises(subprocess.CalledProcessError):
        binding.build(force=True)
