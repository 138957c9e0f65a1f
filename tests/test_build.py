"""The build: libquartz.so needs hipcc alone, whatever becomes of the compiled binding."""
import ctypes
import os

import pytest

from paper_2509_26436_amd import build


@pytest.mark.parametrize("broken", ["torch", "compiler"])
def test_library_without_the_binding(broken, monkeypatch, tmp_path):
    """A plain C library: it is linked where torch is missing, or the binding does not compile, which
    the build then says."""
    if not os.path.exists(build.hipcc()):
        pytest.skip("no hipcc")
    lib, binding = str(tmp_path / "lib.so"), str(tmp_path / "binding.so")
    monkeypatch.setattr(build, "LIB", lib)
    monkeypatch.setattr(build, "BINDING", binding)
    monkeypatch.setattr(build, "SOURCES", ["w4a4_gemm_plain.hip"])
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    (tmp_path / "w4a4_gemm_plain.hip").write_text('extern "C" int answer() { return 42; }\n')
    (tmp_path / build.BINDING_SOURCE).write_text("no C++\n" if broken == "compiler" else "int x;\n")

    def no_torch():
        raise ModuleNotFoundError("No module named 'torch'")
    monkeypatch.setattr(build, "binding_flags", no_torch if broken == "torch" else lambda: ([], []))
    with pytest.raises(ModuleNotFoundError if broken == "torch" else RuntimeError, match="torch|binding"):
        build.build()
    assert ctypes.CDLL(lib).answer() == 42
    assert not os.path.exists(binding)
