"""What is compiled and linked, and for whom, without compiling: the library needs neither PyTorch nor Python, the module that reads tensors is for one of each."""
import sys
import sysconfig

import pytest

from paper_2409_02208_amd import binding, build


@pytest.fixture
def commands(monkeypatch):
    """The commands that a build would run."""
    ran = []
    monkeypatch.setattr(build, "_run", ran.append)
    return ran


def _links(commands, path):
    return [c for c in commands if "-shared" in c and path in c]


def _module_compiles(commands):
    return [c for c in commands if any(a.endswith(build.CALLS_SOURCE) for a in c)]


def test_the_library_is_built_without_pytorch(commands, monkeypatch, capsys):
    for name in [m for m in sys.modules if m == "torch" or m.startswith("torch.")]:
        monkeypatch.setitem(sys.modules, name, None)  # (importing it raises ImportError)
    assert build.build() == build.LIB
    assert len(_links(commands, build.LIB)) == 1 and not _module_compiles(commands) and not _links(commands, build.CALLS)
    assert "PyTorch" in capsys.readouterr().err


def test_the_library_is_built_where_the_module_is_not(monkeypatch):
    ran = []

    def run(cmd):
        ran.append(cmd)
        if any(a.endswith(build.CALLS_SOURCE) for a in cmd):
            raise RuntimeError("build failed: headers of another PyTorch")

    monkeypatch.setattr(build, "_run", run)
    with pytest.raises(RuntimeError, match="another PyTorch"):
        build.build()
    assert len(_links(ran, build.LIB)) == 1 and not _links(ran, build.CALLS)


def test_both_are_built_with_pytorch(commands):
    build.build()
    library, module = _links(commands, build.LIB), _links(commands, build.CALLS)
    assert len(library) == len(module) == 1 and commands.index(library[0]) < commands.index(module[0])
    assert len(_module_compiles(commands)) == 1 and not any("torch" in a for c in commands if c not in _module_compiles(commands) + module for a in c)


def test_the_module_is_for_this_interpreter_and_this_pytorch(monkeypatch):
    assert build.CALLS.endswith("_calls" + sysconfig.get_config_var("EXT_SUFFIX"))
    import torch

    module = binding._calls()
    assert module.__file__ == build.CALLS and module.torch_version == torch.__version__.split("+")[0]
    monkeypatch.setattr(module, "torch_version", "1.0.0")
    monkeypatch.setattr(binding, "_CALLS", None)
    with pytest.raises(RuntimeError, match="1.0.0"):
        binding._calls()
