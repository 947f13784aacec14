"""Building without what only the Python module of the calls around a block's linears needs (a host compiler, torch's and Python's headers):
the library is built all the same, and a module that is older than it does not stay."""
import pytest

from paper_2503_06564_amd import build, trdq


@pytest.fixture
def module(tmp_path):
    """A module of an earlier build."""
    out = tmp_path / "_trdq_calls.so"
    out.write_bytes(b"old")
    return out


def test_without_a_host_compiler(module, monkeypatch, capsys):
    monkeypatch.setattr(build.shutil, "which", lambda name: None)
    assert build.build_calls(str(module)) is None
    assert not module.exists() and "g++" in capsys.readouterr().err


def test_without_headers(module, monkeypatch, capsys, tmp_path):
    monkeypatch.setattr(build, "_calls_headers", lambda: [str(tmp_path)])
    assert build.build_calls(str(module)) is None
    assert not module.exists() and "Python.h" in capsys.readouterr().err


def test_an_error_in_the_source_is_one(module, monkeypatch, tmp_path):
    (tmp_path / "block_calls.cpp").write_text("#error wrong\n")
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    with pytest.raises(RuntimeError, match="wrong"):
        build.build_calls(str(module))
    assert not module.exists()


def test_calls_say_that_the_module_is_missing(monkeypatch):
    import builtins
    real = builtins.__import__

    def without(name, globals=None, locals=None, fromlist=(), level=0):
        if fromlist and "_trdq_calls" in fromlist:
            raise ImportError("no module")
        return real(name, globals, locals, fromlist, level)

    monkeypatch.setattr(trdq, "_block_calls", None)
    monkeypatch.setattr(builtins, "__import__", without)
    with pytest.raises(RuntimeError, match="_trdq_calls"):
        trdq.fp8_quant(None, None, None)
