"""The binding without its torch module (not built, or for another torch): it loads, says so, and every call goes
through its own checks to the same library."""

import os
import shutil
import subprocess
import sys

import pytest

from paper_2605_20863_amd import _lib as L

USE = """
import warnings
with warnings.catch_warnings(record=True) as seen:
    warnings.simplefilter("always")
    from paper_2605_20863_amd import _lib as L
assert any("_pda_torch" in str(w.message) for w in seen), seen
import torch
assert L.version() >= 1
t = torch.zeros
for call in (lambda: L.token_logprobs(t(2, 10), t(2, dtype=torch.int64), t(2)),
             lambda: L.qk_norm_rope(t(2, 4, 64), t(2, 2, 64), None, None, t(8, 64), t(2, dtype=torch.int32), t(2, 4, 64), t(2, 2, 64))):
    try:
        call()
    except ValueError as e:
        assert "HIP device" in str(e), e
    else:
        raise AssertionError("host tensors were accepted")
print("loaded", L._pda_torch)
"""


@pytest.mark.parametrize("module", ["missing", "broken"])
def test_import(tmp_path, module):
    src, pkg = os.path.dirname(L.__file__), tmp_path / "paper_2605_20863_amd"
    pkg.mkdir()
    for name in os.listdir(src):
        if name.endswith(".py"):
            shutil.copy(os.path.join(src, name), pkg / name)
    if module == "broken":
        (pkg / "_pda_torch.so").write_bytes(b"\x7fELF no module")
    run = subprocess.run([sys.executable, "-c", USE], cwd=tmp_path, capture_output=True, text=True,
                         env=dict(os.environ, PDA_LIBRARY=L.LIB_PATH, PYTHONPATH=str(tmp_path)))
    assert run.returncode == 0 and "loaded None" in run.stdout, run.stdout + run.stderr


@pytest.mark.gpu
def test_same_results(monkeypatch):
    import torch

    z = torch.randn((5, 1000), generator=torch.Generator().manual_seed(1)).to("cuda")
    y, a, b = torch.arange(5, device="cuda"), torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda")
    L.token_logprobs(z, y, a)
    monkeypatch.setattr(L, "_calls", {})
    L.token_logprobs(z, y, b)
    assert torch.equal(a, b) and (a < 0).all()
