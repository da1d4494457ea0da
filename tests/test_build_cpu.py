"""What the build compiles again, and what it does without: a copy of its output places, with compilers that
only record their commands."""
import os
import subprocess
from types import SimpleNamespace

import pytest

import __graft_entry__


@pytest.fixture
def build(monkeypatch, tmp_path):
    b = __graft_entry__._build_module()
    monkeypatch.setattr(b, "OBJDIR", str(tmp_path / "_build"))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libress.so"))
    monkeypatch.setattr(b, "TENSORS", str(tmp_path / "_tensors.so"))
    b.commands = []

    def run(cmd, **kw):
        b.commands.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(b.subprocess, "run", run)

    def outputs():
        """Names of what one build compiled and linked."""
        b.commands.clear()
        b.build()
        return sorted(os.path.basename(c[c.index("-o") + 1]) for c in b.commands)

    b.outputs = outputs
    return b


def torch_at(folder, version):
    os.makedirs(folder, exist_ok=True)
    for name, text in (("__init__.py", ""), ("version.py", f"__version__ = '{version}'\n")):
        path = os.path.join(folder, name)
        with open(path, "w") as f:
            f.write(text)
        os.utime(path, (1, 1))  # as old as a wheel's files are
    return SimpleNamespace(origin=os.path.join(folder, "__init__.py"))


def test_tensors_are_compiled_again_for_another_torch_or_python(build, monkeypatch, tmp_path):
    spec = torch_at(str(tmp_path / "a" / "torch"), "2.9.1")
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: spec)
    assert len(build.outputs()) == len(build.SOURCES) + 2  # everything
    assert build.outputs() == []
    torch_at(str(tmp_path / "a" / "torch"), "2.11.0")  # another version in the same place
    assert build.outputs() == ["_tensors.so"]
    assert build.outputs() == []
    spec.origin = torch_at(str(tmp_path / "b" / "torch"), "2.11.0").origin  # the same one in another place
    assert build.outputs() == ["_tensors.so"]
    variables = build.sysconfig.get_config_var
    monkeypatch.setattr(build.sysconfig, "get_config_var", lambda n: "cpython-399" if n == "SOABI" else variables(n))
    assert build.outputs() == ["_tensors.so"]
    assert build.outputs() == []


def test_library_is_built_without_torch(build, monkeypatch, capsys):
    """libress.so and the calls on raw pointers need no torch."""
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    want = sorted([os.path.basename(build.LIB)] + [s.replace(".cu", ".o") for s in build.SOURCES])
    assert build.outputs() == want
    assert "torch" in capsys.readouterr().out
    assert build.outputs() == []


def test_tensors_follow_once_torch_is_there(build, monkeypatch, tmp_path):
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    build.outputs()
    spec = torch_at(str(tmp_path / "torch"), "2.11.0")
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: spec)
    assert build.outputs() == ["_tensors.so"]
