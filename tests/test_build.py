"""A build whose torch module does not compile (no torch headers, another compiler) still leaves the library, and says
what failed."""

import os
import shutil

import pytest

from paper_2605_20863_amd import build as B


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_library_without_the_module(tmp_path, monkeypatch):
    src = tmp_path / "csrc"
    src.mkdir()
    (src / "one.cpp").write_text('extern "C" int one(void) { return 1; }\n')
    monkeypatch.setattr(B, "CSRC", str(src))
    monkeypatch.setattr(B, "SOURCES", ["one.cpp"])
    monkeypatch.setattr(B, "LIB", str(tmp_path / "libpda.so"))
    monkeypatch.setattr(B, "MODULE", str(tmp_path / "_pda_torch.so"))
    monkeypatch.setattr(B, "module_command", lambda out: ["g++", "-c", str(src / "none.cpp"), "-o", out])
    with pytest.raises(RuntimeError, match="g\\+\\+ failed"):
        B.build()
    assert os.path.exists(B.LIB) and not os.path.exists(B.MODULE)
    assert sorted(os.listdir(tmp_path)) == ["csrc", "libpda.so"]
