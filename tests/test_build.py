"""What the build asks of the machine, with the compilers' commands recorded and not run."""

import os
import subprocess
import sys

import pytest

from paper_2608_22883_gb300 import _build


@pytest.fixture
def made(tmp_path, monkeypatch):
    """build() into an empty folder: the commands that it runs, each of which makes its output."""
    for name, path in (("BUILD", "b"), ("LIBDIR", "l"), ("LIB", "l/libfovea.so"), ("BINDING", "l/fovea_binding.so")):
        monkeypatch.setattr(_build, name, str(tmp_path / path))
    commands = []

    def run(cmd, **kw):
        assert all(isinstance(word, str) for word in cmd), cmd
        commands.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("x")
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(_build.subprocess, "run", run)
    return commands


def outputs(commands):
    names = [os.path.basename(cmd[cmd.index("-o") + 1]) for cmd in commands]
    commands.clear()
    return names


def test_everything_is_made_once(made):
    _build.build()
    first = outputs(made)
    assert {"binding.o", "libfovea.so", "fovea_binding.so"} < set(first) and len(first) == len(_build.sources()) + 3
    _build.build()
    assert outputs(made) == []


def test_the_library_needs_no_torch(made, monkeypatch):
    """libfovea is for C programs too: without torch it is made, and the Python module is not."""
    monkeypatch.setitem(sys.modules, "torch", None)
    assert _build.build() == _build.LIB and os.path.exists(_build.LIB)
    names = outputs(made)
    assert "libfovea.so" in names and len(names) == len(_build.sources()) + 1
    assert not os.path.exists(_build.BINDING)


def test_a_missing_compiler_is_named(made, monkeypatch):
    monkeypatch.delenv("CXX", raising=False)
    which = _build.shutil.which
    monkeypatch.setattr(_build.shutil, "which", lambda name: None if name == "g++" else which(name))
    with pytest.raises(RuntimeError, match="g\\+\\+"):
        _build.build()
    assert outputs(made) == []
    monkeypatch.setenv("CXX", "some-c++")
    _build.build()
    assert sum(cmd[0] == "some-c++" for cmd in made) == 2


def test_another_torch_makes_the_module_again(made, monkeypatch, tmp_path):
    """The module goes with the torch that it was compiled against, whatever the files' times."""
    homes = []
    for version in ("1", "2"):
        home = tmp_path / version
        home.mkdir()
        (home / "version.py").write_text(f"__version__ = '{version}'")
        os.utime(home / "version.py", (1, 1))
        homes.append(str(home))
    monkeypatch.setattr(_build, "torch_home", lambda: homes[0])
    _build.build()
    outputs(made)
    _build.build()
    assert outputs(made) == []
    monkeypatch.setattr(_build, "torch_home", lambda: homes[1])
    _build.build()
    assert {"binding.o", "fovea_binding.so"} <= set(outputs(made))
    with open(os.path.join(homes[1], "version.py"), "w") as f:      # replaced in its place
        f.write("__version__ = '3'")
    os.utime(os.path.join(homes[1], "version.py"), (1, 1))
    _build.build()
    assert {"binding.o", "fovea_binding.so"} <= set(outputs(made))
    _build.build()
    assert outputs(made) == []
