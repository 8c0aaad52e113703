"""What a build leaves behind where parts of it cannot be built (no GPU, no compiler needed: the
compilers here write a file that says who made it)."""
import importlib.util
import os
import stat
import subprocess
import sys
import sysconfig
import types

import pytest

COMPILER = """#!{python}
import sys
if {fails} and any({fails} in a for a in sys.argv):
    sys.stderr.write("no such thing")
    sys.exit(1)
open(sys.argv[sys.argv.index("-o") + 1], "w").write("new")
"""


@pytest.fixture
def place(tmp_path, monkeypatch):
    """The build module, building into a folder of its own that holds an earlier build."""
    from paper_2205_13542_amd import build
    for name in ("LIB_PATH", "FLOOR_LIB_PATH", "TORCH_LIB_PATH"):
        path = tmp_path / os.path.basename(getattr(build, name))
        path.write_text("old")
        monkeypatch.setattr(build, name, str(path))

    def compiler(name, fails=""):
        path = tmp_path / name
        path.write_text(COMPILER.format(python=sys.executable, fails=repr(fails)))
        path.chmod(path.stat().st_mode | stat.S_IXUSR)
        return str(path)

    def torch(rocm=True):
        root = tmp_path / "torch"
        (root / "lib").mkdir(parents=True)
        if rocm:
            (root / "lib" / "libtorch_hip.so").write_text("")
        monkeypatch.setattr(importlib.util, "find_spec",
                            lambda name: types.SimpleNamespace(origin=str(root / "__init__.py")))

    def held():
        return [open(p).read() if os.path.exists(p) else None
                for p in (build.LIB_PATH, build.FLOOR_LIB_PATH, build.TORCH_LIB_PATH)]

    python = tmp_path / "python"
    python.mkdir()
    (python / "Python.h").write_text("")
    monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": str(python)})
    monkeypatch.setattr(build, "HIPCC", compiler("hipcc"))
    monkeypatch.setattr(build, "CXX", compiler("c++"))
    return types.SimpleNamespace(build=build, compiler=compiler, torch=torch, held=held, headers=python)


def test_everything_is_built(place):
    place.torch()
    assert place.build.build() == place.build.LIB_PATH
    assert place.held() == ["new", "new", "new"]


def test_no_torch_builds_the_library_and_leaves_no_old_module(place, monkeypatch):
    monkeypatch.setattr(importlib.util, "find_spec", lambda name: None)
    place.build.build()
    assert place.held() == ["new", "new", None]


def test_another_torch_builds_the_library(place, monkeypatch):
    """Beside a torch that is no ROCm build the module is not tried."""
    place.torch(rocm=False)
    monkeypatch.setattr(place.build, "CXX", place.compiler("broken", "layer_torch"))
    place.build.build()
    assert place.held() == ["new", "new", None]


def test_no_compiler_or_headers_of_the_module(place, monkeypatch):
    place.torch()
    with monkeypatch.context() as m:
        m.setattr(place.build, "CXX", str(place.headers / "none"))
        with pytest.warns(UserWarning, match="none.*layer_ops"):
            place.build.build()
    assert place.held() == ["new", "new", None]
    (place.headers / "Python.h").unlink()
    with pytest.warns(UserWarning, match="Python.h.*layer_ops"):
        place.build.build()
    assert place.held() == ["new", "new", None]


@pytest.mark.parametrize("fails", ["layer_torch.cpp", "-shared"])
def test_a_module_that_fails_is_raised_beside_the_new_library(place, monkeypatch, fails):
    place.torch()
    monkeypatch.setattr(place.build, "CXX", place.compiler("broken", fails))
    with pytest.raises(subprocess.CalledProcessError) as failed:
        place.build.build()
    assert failed.value.stderr == "no such thing"
    assert place.held() == ["new", "new", None]


@pytest.mark.parametrize("fails", ["norm.hip", "floor.hip", "libbevpool.so"])
def test_a_library_that_fails_changes_nothing(place, monkeypatch, fails):
    place.torch()
    monkeypatch.setattr(place.build, "HIPCC", place.compiler("broken", fails))
    with pytest.raises(subprocess.CalledProcessError):
        place.build.build()
    assert place.held() == ["old", "old", "old"]
