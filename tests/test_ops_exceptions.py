"""What is thrown below a C entry of include/pda_ops.h becomes an error code with a text, whatever it is: the host code
built over the note-taking HIP runtime, with launchers that throw."""

import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2605_20863_amd import _lib as L
from tests import test_ops_abi as A

ROOT, CSRC, ROCM = A.ROOT, A.CSRC, A.ROCM
THROWN = {"memory": ("std::bad_alloc()", L.ENOMEM), "failed": ('std::runtime_error("lock")', L.EHIP), "number": ("1", L.EHIP)}


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM, "include", "hip")),
                    reason="needs g++ and the ROCm headers")
@pytest.mark.parametrize("what", THROWN)
def test_thrown(tmp_path, what):
    thrown, code = THROWN[what]
    stubs = tmp_path / "throw.cpp"
    stubs.write_text('#include "pda_ops_internal.h"\n#include <new>\n#include <stdexcept>\nnamespace pda {\n' + "".join(
        f"hipError_t {n}(const {a}&{k}, hipStream_t) {{ throw {thrown}; }}\n" for n, a, k in (
            ("launch_rope_append", "RopeArgs", ", KvType"), ("launch_rope", "RopeArgs", ""), ("launch_rope_backward", "RopeArgs", ""),
            ("launch_token_logprobs", "LogitsArgs", ""), ("launch_policy_loss", "LogitsArgs", ""))) + "}\n")
    lib = str(tmp_path / "libpda_throw.so")
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-I",
                          os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                          os.path.join(CSRC, "pda_host.cpp"), os.path.join(CSRC, "pda_ops_host.cpp"), str(stubs),
                          os.path.join(ROOT, "tests", "hostsim", "fake_hip.cpp"), "-o", lib], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    # in a process of its own: what is not caught ends it
    run = subprocess.run(["python3", "-c", USE, lib], capture_output=True, text=True, cwd=ROOT)
    assert run.returncode == 0, run.stdout + run.stderr
    for line in run.stdout.splitlines():
        name, rc, text = line.split("|")
        assert int(rc) == code and text, line
    assert len(run.stdout.splitlines()) == 10


USE = """
import ctypes, sys
from tests import test_ops_abi as A
L = A.L
lib = L._lib = ctypes.CDLL(sys.argv[1])
lib.pda_last_error.restype = ctypes.c_char_p
stream, P = ctypes.c_void_p(0x1000), ctypes.c_void_p(A.P)
b = ctypes.byref
for turn in range(2):  # the workspace is free again after the first
    for name, n, structs in (("paged_qk_norm_rope_append", 14, (A.rope(), A.cache())), ("qk_norm_rope", 8, (A.rope(),)),
                             ("qk_norm_rope_backward", 12, (A.rope(),)), ("token_logprobs", 4, (A.logits(),)),
                             ("policy_loss", 10, (A.logits(), A.options()))):
        rc = getattr(lib, "pdaops_" + name)(*[P] * n, *[b(s) for s in structs], stream)
        print(name, rc, lib.pda_last_error().decode(), sep="|", flush=True)
"""
