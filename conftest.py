"""Fixes glibc's threshold for blocks with a mapping of their own, which otherwise grows with the blocks that the process
has freed: the host-side tests over a note-taking HIP runtime compare addresses of allocations, and a big one
that has been freed must not give its address to a small one."""

import ctypes
import sys

if sys.platform == "linux":
    M_MMAP_THRESHOLD = -3
    ctypes.CDLL(None).mallopt(M_MMAP_THRESHOLD, 128 << 10)
