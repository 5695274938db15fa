"""The library is built where the headers of the module over torch are missing; the module's own errors still show."""
import sysconfig

import pytest

torch = pytest.importorskip("torch")

from paper_2408_04323_amd import _native  # noqa: E402
from paper_2408_04323_amd import build as b  # noqa: E402


def _no_python_headers(monkeypatch, tmp_path):
    monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: {"include": str(tmp_path)})


def _no_torch_headers(monkeypatch, tmp_path):
    monkeypatch.setattr(torch, "__file__", str(tmp_path / "__init__.py"))


def _no_torch(monkeypatch, tmp_path):
    monkeypatch.setitem(__import__("sys").modules, "torch", None)


@pytest.mark.parametrize("lacking", [_no_python_headers, _no_torch_headers, _no_torch])
def test_the_library_without_the_module(monkeypatch, tmp_path, capsys, lacking):
    lib, module = tmp_path / "libscoot.so", tmp_path / "_kv_torch.so"
    module.write_bytes(b"stale")
    monkeypatch.setattr(b, "LIB", str(lib))
    monkeypatch.setattr(b, "MODULE", str(module))
    monkeypatch.setattr(b, "OUT_DIR", str(tmp_path / "obj"))
    monkeypatch.setattr(b, "_hipcc", lambda: "/bin/true")  # the link is stood in for
    monkeypatch.setattr(b, "_compile", lambda src, hipcc: src)
    (tmp_path / "libscoot.so.tmp").write_bytes(b"linked")
    lacking(monkeypatch, tmp_path)
    b.build(verbose=True)
    assert lib.read_bytes() == b"linked" and not module.exists()
    assert "missing" in capsys.readouterr().err


def test_a_module_that_does_not_compile_is_an_error(monkeypatch, tmp_path):
    monkeypatch.setattr(b, "MODULE", str(tmp_path / "_kv_torch.so"))
    monkeypatch.setattr(b, "HERE", str(tmp_path))  # no source there
    with pytest.raises(RuntimeError, match="compile failed"):
        b._build_module()


def test_calls_without_the_module_say_so(monkeypatch, tmp_path):
    _native.lib()
    monkeypatch.setattr(_native, "HERE", str(tmp_path))
    with pytest.raises(RuntimeError, match="is missing: build it"):
        _native.kv_module(None)
