"""The build where PyTorch's or Python's headers are missing: the C library is built
alone, and only the 8-bit operators' Python calls raise."""

import pytest

from paper_2607_27842_gb300 import build, featfix as ff


@pytest.fixture
def small(tmp_path, monkeypatch):
    """The build in a folder of its own, from the one source that compiles fast."""
    monkeypatch.setattr(build, "SOURCES", ["ff_noalloc.cu"])
    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path / "build"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libfeatfix.so"))
    monkeypatch.setattr(build, "BINDING_LIB", str(tmp_path / "_ops8.so"))
    return tmp_path


@pytest.mark.parametrize("missing", ["torch", "Python.h", "g++"])
def test_library_is_built_without_the_binding(small, monkeypatch, capsys, missing):
    if missing == "torch":
        real = build.importlib.util.find_spec
        monkeypatch.setattr(build.importlib.util, "find_spec", lambda n, *a: None if n == "torch" else real(n, *a))
    elif missing == "Python.h":
        paths = dict(build.sysconfig.get_paths(), include=str(small))
        monkeypatch.setattr(build.sysconfig, "get_paths", lambda *a, **k: paths)
    else:
        which = build.shutil.which
        monkeypatch.setattr(build.shutil, "which", lambda n, *a, **k: None if n == "g++" else which(n, *a, **k))
    (small / "_ops8.so").write_bytes(b"of an earlier build")
    assert build.build() == str(small / "libfeatfix.so")
    assert (small / "libfeatfix.so").stat().st_size > 0 and not (small / "_ops8.so").exists()
    assert "_ops8.so is not built" in capsys.readouterr().err


def test_a_binding_that_does_not_compile_is_an_error(small, monkeypatch):
    """Only what is missing is left out: with everything there, a failure is one."""
    def fails():
        raise RuntimeError("g++ on py_ops8.cpp failed")
    monkeypatch.setattr(build, "_compile_binding", fails)
    with pytest.raises(RuntimeError):
        build.build()


def test_calls_without_the_binding_raise(monkeypatch):
    import sys
    import torch
    if not build.os.path.exists(ff.LIB_PATH):
        build.build()
    monkeypatch.setattr(ff, "_ops8", None)
    monkeypatch.setitem(sys.modules, ff.__package__ + "._ops8", None)
    monkeypatch.delattr(sys.modules[ff.__package__], "_ops8", raising=False)
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    with pytest.raises(ff.FeatFixError) as e:
        ff.featfix_op_rms_norm("bf16", x, None, 1e-6, out=x)
    assert e.value.status == ff.ERR_UNSUPPORTED and "_ops8" in str(e.value)
