"""Lanes of a wave that hand each other keys or vectors through LDS: in the kernels' device code (LLVM's intermediate form, from
the library's source and flags) no path leads from such a write to another lane's read, or from a read to the write over it, without
a barrier of the wave or the workgroup, across which the compiler moves no access. Host-only."""

import os
import re
import subprocess

import pytest

from paper_2605_20863_amd import build as B

# Two of the helpers by themselves, with the accesses around them that their callers make.
PROBES = """#include "pda_top.hip"
namespace pda { namespace {
__global__ void probe_thin(int* kept, int n, uint32_t least) {
  extern __shared__ char lds[];
  kept[threadIdx.x] = thin(*reinterpret_cast<Pool*>(lds), n, least);
}
__global__ void probe_gather(const uint64_t* key, int* kept, int n, uint32_t least) {
  extern __shared__ char lds[];
  Pool& b = *reinterpret_cast<Pool*>(lds);
  b.keys[wave_id() * kRegion + (kept[threadIdx.x] & 63)] = key[threadIdx.x];
  kept[threadIdx.x] = gather(b, n, least);
}
void* probes[] = {(void*)&probe_thin, (void*)&probe_gather};
} }
void* pda_probe(int i) { return pda::probes[i]; }
"""
BARRIER = re.compile(r"call void @llvm\.amdgcn\.(wave\.barrier|s\.barrier)\(")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: {block: [lines]}}, the entry first."""
    try:
        hipcc = B.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("ir")
    (d / "probes.hip").write_text(PROBES)
    cmd = [hipcc, f"--offload-arch={B.ARCH}", "-O3", "-std=c++17", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC,
           *B.HIP_FLAGS, "--cuda-device-only", "-S", "-emit-llvm", str(d / "probes.hip"), "-o", str(d / "probes.ll")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    out = {}
    for name, body in re.findall(r"^define [^\n]*amdgpu_kernel [^\n]*?@(\w+)\([^\n]*\{\n(.*?)^\}", (d / "probes.ll").read_text(), re.S | re.M):
        blocks, at = {}, "entry"
        for line in body.splitlines():
            label = re.match(r"^([\w.$-]+):", line)
            if label:
                at = label.group(1)
            elif line.strip():
                blocks.setdefault(at, []).append(line)
        out[name] = blocks
    return out


def unguarded(blocks, start, end):
    """(a line that matches `start`, one that matches `end` and can follow it without a barrier in between), or None."""
    follows = {b: re.findall(r"label %([\w.$-]+)", lines[-1] if "switch" not in " ".join(lines) else " ".join(lines))
               for b, lines in blocks.items()}
    for b, lines in blocks.items():
        for i, line in enumerate(lines):
            if not start.search(line):
                continue
            seen, todo = set(), [(b, i + 1)]
            while todo:
                block, j = todo.pop()
                for other in blocks[block][j:]:
                    if BARRIER.search(other):
                        break
                    if end.search(other):
                        return line.strip(), other.strip()
                else:
                    for n in follows[block]:
                        if n not in seen:
                            seen.add(n)
                            todo.append((n, 0))
    return None


def access(kind, of):
    word = {"load": rf"= load (?:volatile )?{of}, ptr addrspace\(3\)", "store": rf"store {of} [^,]+, ptr addrspace\(3\)"}[kind]
    return re.compile(word)


KEY, VECTOR = "i64", "<4 x (?:i32|float)>"


def named(kernels, what, n):
    found = {k: v for k, v in kernels.items() if what in k}
    assert len(found) == n, sorted(kernels)
    return found.items()


def present(blocks, pattern):
    return any(pattern.search(line) for lines in blocks.values() for line in lines)


def test_vectors_that_wait_to_be_looked_through(kernels):
    for name, blocks in named(kernels, "10top_kernel", 4):
        write, read = access("store", VECTOR), access("load", VECTOR)
        assert present(blocks, write) and present(blocks, read), name
        assert unguarded(blocks, write, read) is None, name
        assert unguarded(blocks, read, write) is None, name


def test_keys_of_a_short_row(kernels):
    for name, blocks in named(kernels, "15top_rows_kernel", 4):
        write, read = access("store", KEY), access("load", KEY)
        assert present(blocks, write) and present(blocks, read), name
        assert unguarded(blocks, write, read) is None, name


def test_keys_that_move_to_the_front(kernels):
    for name, blocks in named(kernels, "10probe_thin", 1):
        write, read = access("store", KEY), access("load", KEY)
        assert present(blocks, write) and present(blocks, read), name
        assert unguarded(blocks, read, write) is None, name


def test_keys_that_are_gathered(kernels):
    for name, blocks in named(kernels, "12probe_gather", 1):
        write, read = access("store", KEY), access("load", KEY)
        assert present(blocks, write) and present(blocks, read), name
        assert unguarded(blocks, write, read) is None, name
        assert unguarded(blocks, read, write) is None, name
