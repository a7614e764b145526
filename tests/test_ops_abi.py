"""The host side of include/pda_ops.h: what the library exports, the structs'
layout, and the refusal of bad arguments before any HIP call (no GPU needed)."""

import ctypes
import os
import shutil
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2605_20863_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_20863_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
P = 0x10000  # a pointer that is never read


def test_exports_every_declared_symbol():
    declared = L.ops_header_symbols()
    assert set(declared) == {"pdaops_paged_qk_norm_rope_append", "pdaops_qk_norm_rope", "pdaops_qk_norm_rope_backward",
                             "pdaops_token_logprobs", "pdaops_policy_loss"}
    nm = subprocess.run(["nm", "-D", "--defined-only", L.LIB_PATH], capture_output=True, text=True).stdout
    exported = {line.split()[-1] for line in nm.splitlines() if " T " in line}
    assert {s for s in exported if s.startswith("pdaops_")} == set(declared)


def test_struct_layouts_match_the_header(tmp_path):
    structs = {"pdaops_rope_problem": L.RopeProblem, "pdaops_cache": L.Cache, "pdaops_logits_problem": L.LogitsProblem,
               "pdaops_policy_options": L.PolicyOptions}
    lines = []
    for name, t in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in t._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "pda_ops.h"\nint main(void) {\n' + "\n".join(lines)
                   + "\nreturn 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROCM, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    got = dict(line.rsplit(" ", 1) for line in out.splitlines())
    for name, t in structs.items():
        assert int(got[name]) == ctypes.sizeof(t), name
        for f, _ in t._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(t, f).offset, f"{name}.{f}"


def rope(**kw):
    base = dict(num_tokens=8, num_q_heads=8, num_kv_heads=2, head_dim=128, rotary_dim=128, max_positions=64, interleaved=0,
                dtype=L.BF16, out_dtype=L.BF16, weight_dtype=L.BF16, eps=1e-6)
    base.update(kw)
    return L.RopeProblem(**base)


def cache(**kw):
    base = dict(num_seqs=4, block_size=16, max_blocks_per_seq=8, max_seq_len=0, num_blocks=64, kv_dtype=L.BF16)
    base.update(kw)
    return L.Cache(**base)


def logits(**kw):
    base = dict(num_tokens=4, vocab=1000, row_stride=0, dtype=L.BF16, targets_int64=1, temperature=1.0)
    base.update(kw)
    return L.LogitsProblem(**base)


def options(**kw):
    base = dict(clip_low=0.2, clip_high=0.2, dual_clip=0.0, kl_coef=0.0, entropy_coef=0.0, grad_scale=1.0, dlogits_stride=0)
    base.update(kw)
    return L.PolicyOptions(**base)


def ref(x):
    return None if x is None else ctypes.byref(x)


def append(pr, ca, **ptr):
    names = ("q", "k", "v", "wq", "wk", "cs", "pos", "off", "qo", "kc", "vc", "sc", "bt", "sl")
    p = [ptr.get(n, P) for n in names]
    return L._lib.pdaops_paged_qk_norm_rope_append(*p, ref(pr), ref(ca), None)


def forward(pr, **ptr):
    return L._lib.pdaops_qk_norm_rope(*[ptr.get(n, P) for n in ("q", "k", "wq", "wk", "cs", "pos", "qo", "ko")], ref(pr), None)


def backward(pr, **ptr):
    names = ("q", "k", "wq", "wk", "cs", "pos", "gq", "gk", "dq", "dk", "dwq", "dwk")
    return L._lib.pdaops_qk_norm_rope_backward(*[ptr.get(n, P) for n in names], ref(pr), None)


def logprobs(pr, **ptr):
    return L._lib.pdaops_token_logprobs(*[ptr.get(n, P) for n in ("z", "y", "lp", "h")], ref(pr), None)


def policy(pr, op, **ptr):
    names = ("z", "y", "old", "ref", "adv", "w", "stats", "dz", "lp", "h")
    return L._lib.pdaops_policy_loss(*[ptr.get(n, P) for n in names], ref(pr), ref(op), None)


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("change,code", [
    (dict(num_tokens=-1), L.EINVAL), (dict(num_q_heads=0), L.EINVAL), (dict(num_kv_heads=0), L.EINVAL),
    (dict(num_q_heads=70000), L.EINVAL), (dict(head_dim=96), L.EUNSUPPORTED), (dict(head_dim=256), L.EUNSUPPORTED),
    (dict(rotary_dim=0), L.EINVAL), (dict(rotary_dim=144), L.EINVAL), (dict(rotary_dim=24), L.EUNSUPPORTED),
    (dict(max_positions=0), L.EINVAL), (dict(interleaved=2), L.EINVAL), (dict(dtype=L.FP8_E4M3), L.EINVAL),
    (dict(out_dtype=7), L.EINVAL), (dict(weight_dtype=-1), L.EINVAL), (dict(eps=-1.0), L.EINVAL), (dict(eps=NAN), L.EINVAL),
    (dict(eps=INF), L.EINVAL), (dict(q_stride=8 * 128 - 8), L.EINVAL), (dict(k_stride=2 * 128 + 4), L.EINVAL),
    (dict(k_stride=-256), L.EINVAL), (dict(q_stride=2 ** 62), L.EINVAL), (dict(q_out_stride=8), L.EINVAL),
    (dict(k_out_stride=257), L.EINVAL), (dict(num_tokens=2 ** 30), L.EINVAL)])
def test_rope_refusals(change, code):
    pr = rope(**change)
    assert forward(pr) == code and L.last_error()
    assert backward(pr) == code and append(pr, cache()) == code


def test_rope_pointers():
    assert forward(None) == backward(None) == append(None, cache()) == append(rope(), None) == L.EINVAL
    for n in ("q", "k", "cs", "pos", "qo", "ko"):
        assert forward(rope(), **{n: None}) == L.EINVAL and L.last_error().endswith("is NULL")
    for n in ("q", "k", "cs", "pos", "gq", "gk", "dq", "dk", "dwq", "dwk"):
        assert backward(rope(), **{n: None}) == L.EINVAL and L.last_error().endswith("is NULL")
    for n in ("q", "k", "v", "cs", "qo", "kc", "vc", "bt", "sl"):
        assert append(rope(), cache(), **{n: None}) == L.EINVAL and L.last_error().endswith("is NULL")
    for n in ("q", "k", "wq", "wk", "cs", "qo", "ko"):
        assert forward(rope(), **{n: P + 8}) == L.EINVAL and "16-byte" in L.last_error()
    for n in ("v", "kc", "vc"):
        assert append(rope(), cache(), **{n: P + 8}) == L.EINVAL and "16-byte" in L.last_error()
    for n in ("pos", "off", "sc", "bt", "sl"):
        assert append(rope(), cache(), **{n: P + 2}) == L.EINVAL and "4-byte" in L.last_error()
    assert append(rope(), cache(kv_dtype=L.FP8_E4M3), sc=None) == L.EINVAL
    for call in (forward, backward, lambda pr, **k: append(pr, cache(), **k)):
        assert call(rope(), wq=None) == L.EINVAL and "both or neither" in L.last_error()
    assert backward(rope(out_dtype=L.F32)) == L.EINVAL
    # nothing to do: no pointer is needed, nothing is launched
    none = dict.fromkeys(("q", "k", "v", "wq", "wk", "cs", "pos", "qo", "ko", "gq", "gk", "dq", "dk", "dwq", "dwk", "kc", "vc",
                          "sc", "bt", "sl"))
    assert forward(rope(num_tokens=0), **none) == backward(rope(num_tokens=0), **none) == L.OK
    assert append(rope(num_tokens=0), cache(), **none) == L.OK


@pytest.mark.parametrize("change,code", [
    (dict(num_seqs=-1), L.EINVAL), (dict(block_size=32), L.EUNSUPPORTED), (dict(max_blocks_per_seq=0), L.EINVAL),
    (dict(max_blocks_per_seq=2 ** 28), L.EINVAL), (dict(num_blocks=0), L.EINVAL), (dict(num_blocks=2 ** 60), L.EINVAL),
    (dict(max_seq_len=129), L.EINVAL), (dict(max_seq_len=-1), L.EINVAL), (dict(kv_dtype=3), L.EINVAL),
    (dict(num_seqs=2 ** 30), L.EINVAL)])
def test_cache_refusals(change, code):
    assert append(rope(), cache(**change)) == code and L.last_error()


def test_tokens_without_offsets():
    assert append(rope(num_tokens=9), cache(), off=None) == L.EINVAL and "multiple of num_seqs" in L.last_error()
    assert append(rope(num_tokens=8), cache(num_seqs=0), off=None) == L.EINVAL
    assert append(rope(num_tokens=0), cache(num_seqs=0), off=None) == L.OK


@pytest.mark.parametrize("change", [
    dict(num_tokens=-1), dict(vocab=0), dict(vocab=2 ** 31 - 1), dict(dtype=L.FP8_E4M3), dict(targets_int64=2),
    dict(row_stride=999), dict(row_stride=-1000), dict(row_stride=2 ** 61), dict(temperature=0.0), dict(temperature=-1.0),
    dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-45), dict(num_tokens=2 ** 30)])
def test_logits_refusals(change):
    pr = logits(**change)
    assert logprobs(pr) == L.EINVAL and L.last_error()
    assert policy(pr, options()) == L.EINVAL


@pytest.mark.parametrize("change", [
    dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-0.1), dict(clip_high=INF), dict(clip_low=NAN), dict(dual_clip=1.0),
    dict(dual_clip=-2.0), dict(dual_clip=INF), dict(kl_coef=-1.0), dict(kl_coef=NAN), dict(entropy_coef=-1.0),
    dict(entropy_coef=INF), dict(grad_scale=NAN), dict(dlogits_stride=999), dict(dlogits_stride=-1)])
def test_policy_refusals(change):
    assert policy(logits(), options(**change)) == L.EINVAL and L.last_error()


def test_logits_pointers():
    assert logprobs(None) == policy(None, options()) == policy(logits(), None) == L.EINVAL
    for n in ("z", "y", "lp"):
        assert logprobs(logits(), **{n: None}) == L.EINVAL
    for n in ("z", "y", "old", "adv", "w", "stats"):
        assert policy(logits(), options(), **{n: None}) == L.EINVAL
    assert policy(logits(), options(kl_coef=0.1), ref=None) == L.EINVAL and "ref_logprobs" in L.last_error()
    assert logprobs(logits(), z=P + 1) == L.EINVAL and "2-byte" in L.last_error()
    assert logprobs(logits(dtype=L.F32), z=P + 2) == L.EINVAL and "4-byte" in L.last_error()
    assert logprobs(logits(), y=P + 4) == L.EINVAL and "8-byte" in L.last_error()
    assert logprobs(logits(num_tokens=0), z=None, y=None, lp=None) == L.OK


def test_binding_refuses_host_tensors_and_wrong_shapes():
    t = torch.zeros
    with pytest.raises(ValueError, match="HIP device"):
        L.qk_norm_rope(t(2, 4, 64), t(2, 2, 64), None, None, t(8, 64), t(2, dtype=torch.int32), t(2, 4, 64), t(2, 2, 64))
    with pytest.raises(ValueError, match="HIP device"):
        L.token_logprobs(t(2, 10), t(2, dtype=torch.int64), t(2))
    # the checks of shapes do not look at the device
    for bad in (t(2, 4, 64).transpose(0, 1), t(2, 8, 64)[:, ::2], t(2, 64, 4).transpose(1, 2), t(1, 4, 64).expand(2, 4, 64), t(2, 4)):
        with pytest.raises(ValueError):
            L._heads(bad, "q", torch.Size((2, 4, 64)))
    assert L._heads(t(3, 9, 64)[:, 2:6], "q") == 9 * 64
    for bad in (t(1, 10).expand(2, 10), t(10, 2).t(), t(2, 20)[:, ::2]):
        with pytest.raises(ValueError):
            L._logits_problem(bad, t(2, dtype=torch.int64), 1.0)
    with pytest.raises(ValueError):
        L._logits_problem(t(2, 10), t(2), 1.0)


@pytest.mark.parametrize("seed", range(20))
def test_numbering_of_cache_tiles(seed):
    """The append kernel's tile numbers with ragged offsets (a model of its search): every tile that a
    sequence's new tokens touch has a number below the grid's bound, and no two the same."""
    rng = np.random.default_rng(seed)
    B = int(rng.integers(1, 300))
    counts = rng.choice([0, 0, 1, 2, 15, 16, 17, 40, 333], B)
    lens = counts + rng.integers(0, 100, B)
    off = np.concatenate([[rng.integers(0, 50)], counts]).cumsum()
    T = int(off[-1] + rng.integers(0, 50))
    total, seen = T // 16 + 2 * B, {}
    key = off[:-1] // 16 + 2 * np.arange(B)
    for i in range(total):
        lo, size = 0, B
        while size > 1:  # 64 keys a round
            step = (size + 63) // 64
            k = sum(1 for j in range(0, size, step) if key[lo + j] <= i) - 1
            if k < 0:
                break
            lo, size = lo + k * step, min(step, size - k * step)
        jt = i - key[lo]
        start = lens[lo] - counts[lo]
        if 0 <= jt < (lens[lo] + 15) // 16 - start // 16 and counts[lo]:
            assert seen.setdefault((lo, start // 16 + jt), i) == i
    want = {(b, j) for b in range(B) if counts[b] for j in range((lens[b] - counts[b]) // 16, (lens[b] + 15) // 16)}
    assert set(seen) == want


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM, "include", "hip")),
                    reason="needs g++ and the ROCm headers")
def test_host_code_under_sanitizers(tmp_path):
    """pda_ops_host.cpp with the code it shares, built for the host alone, under these refusal tests."""
    if "asan" in os.environ.get("LD_PRELOAD", ""):
        pytest.skip("already the instrumented build")
    stubs = tmp_path / "ops_stubs.cpp"
    stubs.write_text('#include "pda_ops_internal.h"\nnamespace pda {\n'
                     + "".join(f"hipError_t {n}(const {a}&{k}, hipStream_t) {{ return hipErrorInvalidValue; }}\n" for n, a, k in (
                         ("launch_rope_append", "RopeArgs", ", KvType"), ("launch_rope", "RopeArgs", ""),
                         ("launch_rope_backward", "RopeArgs", ""), ("launch_token_logprobs", "LogitsArgs", ""),
                         ("launch_policy_loss", "LogitsArgs", ""))) + "}\n")
    lib = str(tmp_path / "libpda_host_sanitized.so")
    build = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fPIC", "-shared", "-fsanitize=address,undefined",
             "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I",
             os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(CSRC, "pda_host.cpp"),
             os.path.join(CSRC, "pda_ops_host.cpp"), str(stubs), os.path.join(ROOT, "tests", "sanitize", "kernel_stubs.cpp"),
             "-L", os.path.join(ROCM, "lib"), f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}", "-lamdhip64", "-o", lib]
    res = subprocess.run(build, capture_output=True, text=True)
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
