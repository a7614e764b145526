"""The host side of include/pda_lm.h: what the library exports, the structs' layout, the refusal of bad arguments before
any HIP call, and what is thrown below an entry (no GPU needed)."""

import ctypes
import os
import shutil
import subprocess
import sys

import pytest

from paper_2605_20863_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_20863_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
P = 0x10000  # a pointer that is never read
INF, NAN = float("inf"), float("nan")
NAMES = ["pdalm_add_rms_norm", "pdalm_add_rms_norm_backward", "pdalm_distill_loss", "pdalm_top_logprobs"]
LAUNCHERS = (("launch_norm", "NormArgs"), ("launch_norm_backward", "NormArgs"), ("launch_top_logprobs", "TopArgs"),
             ("launch_distill_loss", "DistillArgs"))
needs_gxx = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM, "include", "hip")),
                               reason="needs g++ and the ROCm headers")


def test_exports_every_declared_symbol():
    assert L.lm_header_symbols() == NAMES
    nm = subprocess.run(["nm", "-D", "--defined-only", L.LIB_PATH], capture_output=True, text=True).stdout
    exported = {line.split()[-1] for line in nm.splitlines() if " T " in line}
    assert {s for s in exported if s.startswith("pdalm_")} == set(NAMES)


def test_struct_layouts_match_the_header(tmp_path):
    structs = {"pdalm_norm_problem": L.NormProblem, "pdalm_distill_options": L.DistillOptions}
    lines = [f'printf("PDALM_MAX_TOP %d\\n", PDALM_MAX_TOP);']
    for name, t in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in t._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "pda_lm.h"\nint main(void) {\n' + "\n".join(lines)
                   + "\nreturn 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROCM, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    got = dict(line.rsplit(" ", 1) for line in out.splitlines())
    assert int(got["PDALM_MAX_TOP"]) == L.MAX_TOP
    for name, t in structs.items():
        assert int(got[name]) == ctypes.sizeof(t), name
        for f, _ in t._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(t, f).offset, f"{name}.{f}"


def norm(**kw):
    base = dict(num_tokens=4, width=1024, dtype=L.BF16, out_dtype=L.BF16, weight_dtype=L.BF16, scale_group=0, eps=1e-6)
    return L.NormProblem(**{**base, **kw})


def logits(**kw):
    base = dict(num_tokens=4, vocab=1000, row_stride=0, dtype=L.BF16, targets_int64=1, temperature=1.0)
    return L.LogitsProblem(**{**base, **kw})


def options(**kw):
    base = dict(num_listed=8, rest=1, reverse=0.0, grad_scale=1.0, dlogits_stride=0)
    return L.DistillOptions(**{**base, **kw})


def ref(x):
    return None if x is None else ctypes.byref(x)


def pick(names, ptr, **default):
    return [ptr.get(n, default.get(n, P)) for n in names]


def forward(pr, **ptr):
    return L._lib.pdalm_add_rms_norm(*pick(("x", "res", "w", "sum", "out", "scales"), ptr, scales=None), ref(pr), None)


def backward(pr, **ptr):
    return L._lib.pdalm_add_rms_norm_backward(*pick(("h", "w", "g", "q", "dh", "dw"), ptr), ref(pr), None)


def top(pr, K=8, **ptr):
    return L._lib.pdalm_top_logprobs(*pick(("z", "y", "ids", "tops", "lp", "ent"), ptr), ref(pr), K, None)


def distill(pr, op, **ptr):
    return L._lib.pdalm_distill_loss(*pick(("z", "ids", "tau", "w", "stats", "losses", "dz"), ptr), ref(pr), ref(op), None)


@pytest.mark.parametrize("change,code", [
    (dict(num_tokens=-1), L.EINVAL), (dict(num_tokens=2 ** 22 + 1), L.EINVAL), (dict(width=0), L.EINVAL), (dict(width=-8), L.EINVAL),
    (dict(width=1001), L.EUNSUPPORTED), (dict(width=32776), L.EUNSUPPORTED), (dict(dtype=L.FP8_E4M3), L.EINVAL),
    (dict(dtype=5), L.EINVAL), (dict(weight_dtype=L.FP8_E4M3), L.EINVAL), (dict(eps=-1.0), L.EINVAL), (dict(eps=NAN), L.EINVAL),
    (dict(eps=INF), L.EINVAL), (dict(x_stride=1016), L.EINVAL), (dict(x_stride=1028), L.EINVAL), (dict(x_stride=-1024), L.EINVAL),
    (dict(x_stride=2 ** 62), L.EINVAL), (dict(residual_stride=8), L.EINVAL), (dict(sum_stride=1025), L.EINVAL),
    (dict(out_stride=1025), L.EINVAL)])
def test_norm_refusals(change, code):
    assert forward(norm(**change)) == code and L.last_error()
    assert backward(norm(**change)) == code and L.last_error()


@pytest.mark.parametrize("change,code", [
    (dict(out_dtype=9), L.EINVAL), (dict(out_dtype=L.FP8_E4M3, scale_group=32), L.EUNSUPPORTED),
    (dict(out_dtype=L.FP8_E4M3, scale_group=-1), L.EUNSUPPORTED), (dict(out_dtype=L.FP8_E4M3, scale_group=128, width=1032), L.EUNSUPPORTED),
    (dict(out_dtype=L.FP8_E4M3, out_stride=1028), L.EINVAL)])
def test_norm_out_refusals(change, code):
    assert forward(norm(**change), scales=P) == code and L.last_error()


def test_norm_pointers():
    assert forward(None) == L.EINVAL and backward(None) == L.EINVAL
    for n in ("x", "w", "out"):
        assert forward(norm(), **{n: None}) == L.EINVAL and L.last_error().endswith("is NULL")
    for n in ("x", "res", "w", "sum", "out"):
        assert forward(norm(), **{n: P + 8}) == L.EINVAL and "aligned" in L.last_error()
    assert forward(norm(), res=None) == L.EINVAL and "residual" in L.last_error()  # nothing to keep
    assert forward(norm(), scales=P) == L.EINVAL and "scales" in L.last_error()
    fp8 = norm(out_dtype=L.FP8_E4M3)
    assert forward(fp8) == L.EINVAL and L.last_error() == "scales is NULL"
    assert forward(fp8, scales=P + 2) == L.EINVAL and forward(fp8, scales=P, out=P + 4) == L.EINVAL
    for n in ("h", "w", "g", "dh"):
        assert backward(norm(), **{n: None}) == L.EINVAL
    for n in ("h", "w", "g", "q", "dh"):
        assert backward(norm(), **{n: P + 8}) == L.EINVAL
    assert backward(norm(), dw=P + 2) == L.EINVAL
    assert forward(norm(num_tokens=0), x=None, out=None) == L.OK
    assert backward(norm(num_tokens=0), h=None, g=None, dh=None, w=None, dw=None) == L.OK


LOGITS = [dict(num_tokens=-1), dict(vocab=0), dict(vocab=2 ** 30 + 1), dict(row_stride=999), dict(row_stride=-1000),
          dict(row_stride=2 ** 62), dict(dtype=L.FP8_E4M3), dict(targets_int64=2), dict(temperature=0.0), dict(temperature=-1.0),
          dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-45)]


@pytest.mark.parametrize("change", LOGITS)
def test_logits_refusals(change):
    assert top(logits(**change)) == L.EINVAL and L.last_error()
    assert distill(logits(**change), options()) == L.EINVAL and L.last_error()


def test_top_refusals():
    for K in (0, -1, 257, 2 ** 31 - 1):
        assert top(logits(), K) == L.EINVAL and "num_top" in L.last_error()
    assert top(None) == L.EINVAL
    for n in ("z", "ids", "tops"):
        assert top(logits(), **{n: None}) == L.EINVAL and L.last_error().endswith("is NULL")
    for n, off in (("z", 1), ("y", 4), ("ids", 2), ("tops", 2), ("lp", 2), ("ent", 2)):
        assert top(logits(), **{n: P + off}) == L.EINVAL and "aligned" in L.last_error()
    assert top(logits(), y=None) == L.EINVAL and "targets" in L.last_error()
    assert top(logits(num_tokens=2 ** 22 + 1)) == L.EINVAL
    assert top(logits(num_tokens=0), z=None, y=None, ids=None, tops=None, lp=None) == L.OK


@pytest.mark.parametrize("change", [
    dict(num_listed=0), dict(num_listed=257), dict(num_listed=-5), dict(rest=2), dict(rest=-1), dict(reverse=-0.1), dict(reverse=1.1),
    dict(reverse=NAN), dict(grad_scale=NAN), dict(grad_scale=INF), dict(dlogits_stride=999), dict(dlogits_stride=-1000),
    dict(dlogits_stride=2 ** 62)])
def test_distill_refusals(change):
    assert distill(logits(), options(**change)) == L.EINVAL and L.last_error()


def test_distill_pointers():
    assert distill(None, options()) == L.EINVAL and distill(logits(), None) == L.EINVAL
    for n in ("z", "ids", "tau", "w", "stats"):
        assert distill(logits(), options(), **{n: None}) == L.EINVAL and L.last_error().endswith("is NULL")
    for n, off in (("z", 1), ("ids", 2), ("tau", 2), ("w", 2), ("stats", 2), ("losses", 2), ("dz", 1)):
        assert distill(logits(), options(), **{n: P + off}) == L.EINVAL and "aligned" in L.last_error()
    assert distill(logits(num_tokens=2 ** 20 + 1), options()) == L.EINVAL
    assert distill(logits(num_tokens=0), options(), stats=None) == L.EINVAL


def test_binding_refuses_host_tensors():
    import torch

    z = torch.zeros
    ids = z((2, 3), dtype=torch.int32)
    for call in (lambda: L.add_rms_norm(z(2, 64), z(64), z(2, 64)), lambda: L.add_rms_norm_backward(z(2, 64), z(64), z(2, 64), z(2, 64)),
                 lambda: L.top_logprobs(z(2, 9), ids, z(2, 3)), lambda: L.distill_loss(z(2, 9), ids, z(2, 3), z(2), z(6))):
        with pytest.raises(ValueError, match="HIP device"):
            call()


def host_build(out, stubs, *more):
    return subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I",
                           os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                           os.path.join(CSRC, "pda_host.cpp"), os.path.join(CSRC, "pda_lm_host.cpp"), str(stubs), *more, "-o", out],
                          capture_output=True, text=True)


@needs_gxx
def test_host_code_under_sanitizers(tmp_path):
    """pda_lm_host.cpp with the code it shares, built for the host alone, under these refusal tests."""
    if "asan" in os.environ.get("LD_PRELOAD", ""):
        pytest.skip("already the instrumented build")
    stubs = tmp_path / "stubs.cpp"
    stubs.write_text('#include "pda_lm_internal.h"\nnamespace pda {\n' + "".join(
        f"hipError_t {n}(const {a}&, hipStream_t) {{ return hipErrorInvalidValue; }}\n" for n, a in LAUNCHERS) + "}\n")
    lib = str(tmp_path / "libpda_host_sanitized.so")
    res = host_build(lib, stubs, "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
                     os.path.join(ROOT, "tests", "sanitize", "kernel_stubs.cpp"), "-L", os.path.join(ROCM, "lib"),
                     f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}", "-lamdhip64")
    assert res.returncode == 0, res.stderr[-4000:]
    rt = [subprocess.run(["g++", f"-print-file-name={n}"], capture_output=True, text=True).stdout.strip()
          for n in ("libasan.so", "libubsan.so")]
    env = dict(os.environ, PDA_LIBRARY=lib, LD_PRELOAD=" ".join(p for p in rt if os.path.isabs(p)),
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    run = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", os.path.abspath(__file__)],
                         capture_output=True, text=True, env=env, cwd=ROOT, timeout=600)
    out = run.stdout + run.stderr
    assert run.returncode == 0, out[-6000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out and " passed" in out, out[-6000:]


THROWN = {"memory": ("std::bad_alloc()", L.ENOMEM), "failed": ('std::runtime_error("lock")', L.EHIP), "number": ("1", L.EHIP)}
USE = """
import ctypes, sys
from tests import test_lm_abi as A
lib = ctypes.CDLL(sys.argv[1])
lib.pda_last_error.restype = ctypes.c_char_p
stream, P = ctypes.c_void_p(0x1000), ctypes.c_void_p(A.P)
b = ctypes.byref
for turn in range(2):  # the workspace is free again after the first
    for name, args in (("add_rms_norm", [P] * 5 + [None, b(A.norm())]), ("add_rms_norm_backward", [P] * 6 + [b(A.norm())]),
                       ("top_logprobs", [P] * 6 + [b(A.logits()), 8]), ("distill_loss", [P] * 7 + [b(A.logits()), b(A.options())])):
        rc = getattr(lib, "pdalm_" + name)(*args, stream)
        print(name, rc, lib.pda_last_error().decode(), sep="|", flush=True)
"""


@needs_gxx
@pytest.mark.parametrize("what", THROWN)
def test_thrown(tmp_path, what):
    """What is thrown below an entry becomes an error code with a text."""
    thrown, code = THROWN[what]
    stubs = tmp_path / "throw.cpp"
    stubs.write_text('#include "pda_lm_internal.h"\n#include <new>\n#include <stdexcept>\nnamespace pda {\n' + "".join(
        f"hipError_t {n}(const {a}&, hipStream_t) {{ throw {thrown}; }}\n" for n, a in LAUNCHERS) + "}\n")
    lib = str(tmp_path / "libpda_throw.so")
    res = host_build(lib, stubs, "-Wl,-Bsymbolic", os.path.join(ROOT, "tests", "hostsim", "fake_hip.cpp"))
    assert res.returncode == 0, res.stderr[-4000:]
    # in a process of its own: what is not caught ends it
    run = subprocess.run([sys.executable, "-c", USE, lib], capture_output=True, text=True, cwd=ROOT)
    assert run.returncode == 0, run.stdout + run.stderr
    lines = run.stdout.splitlines()
    assert len(lines) == 8
    for line in lines:
        _, rc, text = line.split("|")
        assert int(rc) == code and text, line
