"""The extension behind the calls on 8-bit matrices: it is there, and says so where it is not."""
import pytest

from paper_1905_10138_amd import fp8


def test_the_extension_loads():
    native = fp8._load()
    assert all(callable(getattr(native, name)) for name in ("quant", "norm", "gate", "matmul", "moe"))
    for name, count in (("quant", 2), ("norm", 6), ("gate", 1), ("matmul", 6), ("moe", 9)):
        with pytest.raises(TypeError, match=f"{count} arguments"):
            getattr(native, name)()


def test_a_missing_extension_is_an_error(monkeypatch):
    monkeypatch.setattr(fp8, "_native", None)
    monkeypatch.setattr(fp8, "library_path", lambda: "/nonexistent/libxorenc.so")
    with pytest.raises(RuntimeError, match="build it"):
        fp8.quant_fp8(None)
