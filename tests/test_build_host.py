"""The library is built where PyTorch's headers or a host compiler are not: only the binding's look at lists of tensors needs them."""
import os
import subprocess
import sys

import pytest


@pytest.fixture
def build(monkeypatch, tmp_path):
    """The module with its outputs in a folder of its own and the kernels' compiler replaced by notes of what it is asked for."""
    from paper_2512_06547_amd import build as module
    lib, tensors, asked = tmp_path / "liba3po.so", tmp_path / "a3po_tensors.so", []
    monkeypatch.setattr(module, "LIB", str(lib))
    monkeypatch.setattr(module, "TENSORS", str(tensors))
    monkeypatch.setattr(module, "OBJ", str(tmp_path / "obj"))
    run = subprocess.check_call
    def check_call(command, *args, **kw):
        if command[0] != module.HIPCC:
            return run(command, *args, **kw)
        asked.append(os.path.basename(command[command.index("-o") + 1]))
        open(command[command.index("-o") + 1], "w").write("built")
    monkeypatch.setattr(module.subprocess, "check_call", check_call)
    module.asked = asked
    yield module
    del module.asked


@pytest.mark.parametrize("missing", ["torch", "compiler", "failing compiler"])
def test_library_without_what_the_binding_needs(build, monkeypatch, capfd, missing):
    open(build.TENSORS, "w").write("of an earlier build")
    if missing == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        monkeypatch.setenv("CXX", "/nonexistent/g++" if missing == "compiler" else "false")
    assert build.build(force=True) == build.LIB
    assert build.asked[-1] == "liba3po.so" and len(build.asked) == len(build.SOURCES) + 1
    assert not os.path.exists(build.TENSORS), "one that does not match the sources is not left"
    said = capfd.readouterr().err
    assert "a3po_tensors.so" in said and "adamw_step" in said and "grad_norm" in said


def test_only_what_is_out_of_date_is_built(build, monkeypatch):
    made = []
    monkeypatch.setattr(build, "_compile_tensors", lambda: (made.append(1), open(build.TENSORS, "w").write("built"))[0])
    build.build(force=True)
    assert made == [1]
    n = len(build.asked)
    build.build(force=False)
    assert len(build.asked) == n and made == [1]
    os.remove(build.TENSORS)
    build.build(force=False)
    assert len(build.asked) == n and made == [1, 1]
    os.utime(build.LIB, (0, 0))
    build.build(force=False)
    assert len(build.asked) == 2 * n and made == [1, 1]


def test_kernels_that_do_not_compile_fail_the_build(build, monkeypatch):
    monkeypatch.setattr(build, "_compile_tensors", lambda: None)
    def refuse(src):
        raise subprocess.CalledProcessError(1, [src])
    monkeypatch.setattr(build, "_compile", refuse)
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)
