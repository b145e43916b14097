"""Building the library without what only the Python module needs, and modules of another Python or torch.  No compiler is run."""
import os

import pytest

from paper_2410_15352_b200 import block, build


@pytest.fixture()
def elsewhere(tmp_path, monkeypatch):
    """A place without a module; the library is up to date."""
    build.build_library()
    monkeypatch.setattr(build, "MODULE_PATH", str(tmp_path / "_block_py.so"))
    return build.MODULE_PATH


def test_the_library_needs_no_host_compiler(elsewhere, monkeypatch):
    monkeypatch.setenv("CXX", "/nonexistent/g++")
    with pytest.warns(RuntimeWarning, match="Python module"):
        assert build.build_library() == build.LIB_PATH
    assert os.listdir(os.path.dirname(elsewhere)) == []
    with pytest.raises(OSError):
        build.build_module()


def test_the_library_needs_no_torch_headers(elsewhere, monkeypatch):
    monkeypatch.setattr(build, "_module_command", lambda out: ["sh", "-c", "echo no such file: ATen/ATen.h >&2; exit 1"])
    with pytest.warns(RuntimeWarning, match="ATen/ATen.h"):
        assert build.build_library() == build.LIB_PATH
    with pytest.raises(RuntimeError, match="ATen/ATen.h"):
        build.build_module()

    def no_torch():
        raise ImportError("No module named 'torch'")

    monkeypatch.setattr(build, "module_tag", no_torch)
    with open(elsewhere, "wb") as f:
        f.write(b"built for [something]")
    with pytest.warns(RuntimeWarning, match="torch"):
        assert build.build_library() == build.LIB_PATH


def test_a_module_of_another_torch_is_built_again(elsewhere, monkeypatch):
    built = []

    def command(out):
        built.append(out)
        return ["sh", "-c", f"printf 'built for [%s]' '{build.module_tag()}' > '{out}'"]

    monkeypatch.setattr(build, "_module_command", command)
    with open(elsewhere, "wb") as f:
        f.write(b"built for [python 2, torch 0.1, abi 0]")
    assert not build.module_fits()
    build.build_module()
    assert len(built) == 1 and build.module_fits()
    build.build_module()
    assert len(built) == 1                                     # up to date now
    monkeypatch.setattr(build, "module_tag", lambda: "python 3, torch 99, abi 1")
    assert not build.module_fits()
    build.build_module()
    assert len(built) == 2 and build.module_fits()
    assert os.listdir(os.path.dirname(elsewhere)) == ["_block_py.so"]


def test_operators_refuse_a_module_that_does_not_fit(monkeypatch):
    build.build_library()
    assert build.module_fits() and block._module() is not None
    monkeypatch.setattr(block, "_mod", None)
    monkeypatch.setattr(block, "module_fits", lambda: False)
    with pytest.raises(ImportError, match="build_module"):
        block.Rotary(64)
