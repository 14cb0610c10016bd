"""The C library does not need the Python module of the forward point's operators, nor torch: where the one cannot be
built the other is, and a module built from other sources does not stay."""
import os

import pytest

from paper_2609_38095_gb300 import build as B


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """Output paths of their own, and one small source in place of the library's."""
    for name in ("LIB", "BINDING", "STAMP"):
        monkeypatch.setattr(B, name, str(tmp_path / os.path.basename(getattr(B, name))))
    monkeypatch.setattr(B, "BUILD", str(tmp_path / "objects"))
    (tmp_path / "src").mkdir()
    (tmp_path / "src" / "one.cu").write_text('extern "C" int one() { return 1; }\n')
    monkeypatch.setattr(B, "CSRC", str(tmp_path / "src"))
    monkeypatch.setattr(B, "SOURCES", ["one.cu"])
    monkeypatch.setattr(B, "HEADERS", [])
    return tmp_path


def test_a_module_that_does_not_compile(elsewhere):
    (elsewhere / "src" / "zo_binding.cpp").write_text("#error no torch\n")
    (elsewhere / "_binding.so").write_text("of other sources")
    with pytest.warns(UserWarning, match="not built"):
        lib = B.build()
    assert os.path.exists(lib) and not os.path.exists(B.BINDING)
    with pytest.raises(RuntimeError, match="compiler failed"):
        B.build_binding()


def test_no_torch(elsewhere, monkeypatch):
    def none():
        raise ModuleNotFoundError("torch")
    monkeypatch.setattr(B, "_torch_version", none)
    with pytest.warns(UserWarning, match="not built"):
        assert os.path.exists(B.build())


def test_the_module_follows_both_headers(elsewhere, monkeypatch):
    """zo_forward.h includes zo.h: a module older than either is built again."""
    (elsewhere / "src" / "zo_binding.cpp").write_text("int one() { return 1; }\n")
    include = elsewhere / "include"
    include.mkdir()
    for h in ("zo.h", "zo_forward.h"):
        (include / h).write_text("")
    monkeypatch.setattr(B, "INCLUDE", str(include))
    B.build_binding()
    for h in ("zo.h", "zo_forward.h"):
        first = os.stat(B.BINDING).st_mtime_ns
        B.build_binding()
        assert os.stat(B.BINDING).st_mtime_ns == first
        after = os.path.getmtime(B.BINDING) + 10
        os.utime(include / h, (after, after))
        B.build_binding()
        assert os.stat(B.BINDING).st_mtime_ns != first
        os.utime(include / h, (0, 0))
