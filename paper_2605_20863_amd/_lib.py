"""ctypes binding of the C interface in include/pda.h, include/pda_ops.h and include/pda_lm.h.

Argument marshalling only: every step of the decode attention, KV append,
prefill and the operators around them runs in the HIP library ``libpda.so``. Importing this module fails loudly when the
library has not been built; there is no fallback.

torch is used for device memory and streams: tensors provide device pointers
(``data_ptr()``) and the current HIP stream (``torch.cuda.current_stream()``).
"""

from __future__ import annotations

import ctypes
import os
import re
import warnings

_PKG = os.path.dirname(os.path.abspath(__file__))
# PDA_LIBRARY may point at another build of the same library (same C interface)
LIB_PATH = os.environ.get("PDA_LIBRARY") or os.path.join(_PKG, "libpda.so")
HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "pda.h")
OPS_HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "pda_ops.h")
LM_HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "pda_lm.h")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build the HIP library first "
        "(python -m paper_2605_20863_amd.build); there is no CPU fallback")

# Map PyTorch's bundled HIP runtime before the library: libpda.so then binds to
# that already-loaded runtime (same SONAME), so torch and the library share one
# HIP runtime instead of each bringing up its own (a second runtime in the
# process does not see the device).
try:
    import torch as _torch_rt  # noqa: F401
except ImportError:  # pure C-ABI use without torch: the ROCm installation's runtime
    _torch_rt = None

_lib = ctypes.CDLL(LIB_PATH)

# The torch module only saves host time: without it every call goes through the
# checks below, to the same kernels.
_pda_torch = None
if _torch_rt is not None:
    try:
        from . import _pda_torch
    except ImportError as e:  # not built, or for a torch of another ABI
        warnings.warn(f"_pda_torch does not load ({e}); calls of include/pda_ops.h and pda_lm.h take some "
                      "microseconds more host time each until python -m paper_2605_20863_amd.build has built it", RuntimeWarning)

# pda_dtype / pda_status / pda_variant
F32, BF16, FP8_E4M3 = 0, 1, 2
OK, EINVAL, EUNSUPPORTED, EHIP, ENOMEM = 0, -1, -2, -3, -4
VARIANT_AUTO, VARIANT_VECTOR, VARIANT_MFMA = 0, 1, 2
_VARIANTS = {"auto": VARIANT_AUTO, "vector": VARIANT_VECTOR, "mfma": VARIANT_MFMA}
STATUS_LEN_CLAMPED, STATUS_BAD_BLOCK, STATUS_PREFIX_SHORTENED, STATUS_BAD_OFFSETS = 1, 2, 4, 8
STATUS_HALF_RANGE = 16
STATUS_BAD_POSITION, STATUS_BAD_TARGET, STATUS_TWICE = 32, 64, 128
# "old_kl" is e^-d - 1 + d of the log ratio d: include/pda_ops.h says what its mean estimates.
POLICY_STATS = ("loss", "policy", "kl", "entropy", "clipped", "ratio", "old_kl", "weight")
# Sums over rows of weights times these; the masses are the list's under the teacher and under the student.
DISTILL_STATS = ("loss", "forward", "reverse", "teacher_mass", "student_mass", "weight")
MAX_TOP = 256   # PDALM_MAX_TOP
NOALLOC_SCRATCH_BYTES = 32 << 20   # PDA_NOALLOC_SCRATCH_BYTES


class Problem(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("block_size", ctypes.c_int32),
        ("max_blocks_per_seq", ctypes.c_int32),
        ("num_blocks", ctypes.c_int64),
        ("max_seq_len", ctypes.c_int32),
        ("q_dtype", ctypes.c_int32),
        ("kv_dtype", ctypes.c_int32),
        ("out_dtype", ctypes.c_int32),
        ("q_tokens", ctypes.c_int32),
    ]


class Options(ctypes.Structure):
    _fields_ = [
        ("variant", ctypes.c_int32),
        ("waves_per_cu", ctypes.c_int32),
        ("min_blocks_per_wave", ctypes.c_int32),
        ("chunks_per_wave", ctypes.c_int32),
        ("min_blocks_per_chunk", ctypes.c_int32),
    ]


class PlanInfo(ctypes.Structure):
    _fields_ = [
        ("variant", ctypes.c_int32),
        ("waves", ctypes.c_int32),
        ("group_size", ctypes.c_int32),
        ("chunks_max", ctypes.c_int32),
        ("workspace_bytes", ctypes.c_int64),
    ]


class AppendProblem(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("block_size", ctypes.c_int32),
        ("max_blocks_per_seq", ctypes.c_int32),
        ("num_blocks", ctypes.c_int64),
        ("new_dtype", ctypes.c_int32),
        ("kv_dtype", ctypes.c_int32),
    ]


class PrefillProblem(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("num_tokens", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("block_size", ctypes.c_int32),
        ("max_blocks_per_seq", ctypes.c_int32),
        ("num_blocks", ctypes.c_int64),
        ("max_seq_len", ctypes.c_int32),
        ("q_dtype", ctypes.c_int32),
        ("kv_dtype", ctypes.c_int32),
        ("out_dtype", ctypes.c_int32),
    ]


class RopeProblem(ctypes.Structure):
    _fields_ = [
        ("num_tokens", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("rotary_dim", ctypes.c_int32),
        ("max_positions", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("out_dtype", ctypes.c_int32),
        ("weight_dtype", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("q_stride", ctypes.c_int64),
        ("k_stride", ctypes.c_int64),
        ("v_stride", ctypes.c_int64),
        ("q_out_stride", ctypes.c_int64),
        ("k_out_stride", ctypes.c_int64),
        ("grad_q_stride", ctypes.c_int64),
        ("grad_k_stride", ctypes.c_int64),
    ]


class Cache(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("block_size", ctypes.c_int32),
        ("max_blocks_per_seq", ctypes.c_int32),
        ("max_seq_len", ctypes.c_int32),
        ("num_blocks", ctypes.c_int64),
        ("kv_dtype", ctypes.c_int32),
    ]


class LogitsProblem(ctypes.Structure):
    _fields_ = [
        ("num_tokens", ctypes.c_int32),
        ("vocab", ctypes.c_int32),
        ("row_stride", ctypes.c_int64),
        ("dtype", ctypes.c_int32),
        ("targets_int64", ctypes.c_int32),
        ("temperature", ctypes.c_float),
    ]


class PolicyOptions(ctypes.Structure):
    _fields_ = [
        ("clip_low", ctypes.c_float),
        ("clip_high", ctypes.c_float),
        ("dual_clip", ctypes.c_float),
        ("kl_coef", ctypes.c_float),
        ("entropy_coef", ctypes.c_float),
        ("grad_scale", ctypes.c_float),
        ("dlogits_stride", ctypes.c_int64),
    ]


class NormProblem(ctypes.Structure):
    _fields_ = [
        ("num_tokens", ctypes.c_int32),
        ("width", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("out_dtype", ctypes.c_int32),
        ("weight_dtype", ctypes.c_int32),
        ("scale_group", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("x_stride", ctypes.c_int64),
        ("residual_stride", ctypes.c_int64),
        ("sum_stride", ctypes.c_int64),
        ("out_stride", ctypes.c_int64),
    ]


class DistillOptions(ctypes.Structure):
    _fields_ = [
        ("num_listed", ctypes.c_int32),
        ("rest", ctypes.c_int32),
        ("reverse", ctypes.c_float),
        ("grad_scale", ctypes.c_float),
        ("dlogits_stride", ctypes.c_int64),
    ]


_vp = ctypes.c_void_p
_lib.pda_paged_decode_attention.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float,
                                            ctypes.POINTER(Problem), ctypes.POINTER(Options), _vp]
_lib.pda_paged_decode_attention.restype = ctypes.c_int
_lib.pda_paged_decode_attention_noalloc.argtypes = _lib.pda_paged_decode_attention.argtypes
_lib.pda_paged_decode_attention_noalloc.restype = ctypes.c_int
_lib.pda_query_plan.argtypes = [ctypes.POINTER(Problem), ctypes.POINTER(Options), ctypes.c_float,
                                ctypes.c_int32, ctypes.POINTER(PlanInfo)]
_lib.pda_query_plan.restype = ctypes.c_int
_lib.pda_paged_decode_attention_shared_prefix.argtypes = [
    _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float, ctypes.c_int32, _vp,
    ctypes.POINTER(Problem), ctypes.POINTER(Options), _vp]
_lib.pda_paged_decode_attention_shared_prefix.restype = ctypes.c_int
_lib.pda_query_plan_shared_prefix.argtypes = [ctypes.POINTER(Problem), ctypes.POINTER(Options), ctypes.c_float,
                                              ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(PlanInfo)]
_lib.pda_query_plan_shared_prefix.restype = ctypes.c_int
_lib.pda_paged_kv_append.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.POINTER(AppendProblem), _vp]
_lib.pda_paged_kv_append.restype = ctypes.c_int
_lib.pda_paged_prefill_attention.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float,
                                             ctypes.POINTER(PrefillProblem), _vp]
_lib.pda_paged_prefill_attention.restype = ctypes.c_int
_lib.pda_read_device_status.argtypes = [_vp]
_lib.pda_read_device_status.restype = ctypes.c_int
_lib.pda_release_workspaces.argtypes = []
_lib.pda_release_workspaces.restype = ctypes.c_int
_lib.pda_last_error.argtypes = []
_lib.pda_last_error.restype = ctypes.c_char_p
_lib.pda_version.argtypes = []
_lib.pda_version.restype = ctypes.c_int
# include/pda_ops.h and include/pda_lm.h. PDA_LIBRARY may name a build of the host code behind
# pda.h alone; a call of one of these then fails for want of its symbol.
_rope, _logits, _norm = ctypes.POINTER(RopeProblem), ctypes.POINTER(LogitsProblem), ctypes.POINTER(NormProblem)
for _name, _args in (
        ("pdaops_paged_qk_norm_rope_append", [_vp] * 14 + [_rope, ctypes.POINTER(Cache), _vp]),
        ("pdaops_qk_norm_rope", [_vp] * 8 + [_rope, _vp]),
        ("pdaops_qk_norm_rope_backward", [_vp] * 12 + [_rope, _vp]),
        ("pdaops_token_logprobs", [_vp] * 4 + [_logits, _vp]),
        ("pdaops_policy_loss", [_vp] * 10 + [_logits, ctypes.POINTER(PolicyOptions), _vp]),
        ("pdalm_add_rms_norm", [_vp] * 6 + [_norm, _vp]),
        ("pdalm_add_rms_norm_backward", [_vp] * 6 + [_norm, _vp]),
        ("pdalm_top_logprobs", [_vp] * 6 + [_logits, ctypes.c_int32, _vp]),
        ("pdalm_distill_loss", [_vp] * 7 + [_logits, ctypes.POINTER(DistillOptions), _vp])):
    if hasattr(_lib, _name):
        getattr(_lib, _name).argtypes = _args
        getattr(_lib, _name).restype = ctypes.c_int
# The torch module's functions with the addresses of their entries.
_calls = {n: (getattr(_pda_torch, n), ctypes.cast(getattr(_lib, p + n), _vp).value) for p, n in (
    ("pdaops_", "paged_qk_norm_rope_append"), ("pdaops_", "qk_norm_rope"), ("pdaops_", "qk_norm_rope_backward"),
    ("pdaops_", "token_logprobs"), ("pdaops_", "policy_loss"), ("pdalm_", "add_rms_norm"),
    ("pdalm_", "add_rms_norm_backward"), ("pdalm_", "top_logprobs"), ("pdalm_", "distill_loss"))
    if hasattr(_pda_torch, n) and hasattr(_lib, p + n)}


class PdaError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"pda error {code}: {message}")
        self.code = code


def last_error() -> str:
    return (_lib.pda_last_error() or b"").decode()


def version() -> int:
    return _lib.pda_version()


def header_symbols():
    """Names of the functions include/pda.h declares."""
    text = open(HEADER_PATH).read()
    return sorted(set(re.findall(r"^\s*(?:const\s+)?\w+\*?\s+\*?(pda_\w+)\s*\(", text, re.M)))


def ops_header_symbols():
    """Names of the functions include/pda_ops.h declares."""
    return sorted(set(re.findall(r"^int (pdaops_\w+)\s*\(", open(OPS_HEADER_PATH).read(), re.M)))


def lm_header_symbols():
    """Names of the functions include/pda_lm.h declares."""
    return sorted(set(re.findall(r"^int (pdalm_\w+)\s*\(", open(LM_HEADER_PATH).read(), re.M)))


def _check(rc):
    if rc != OK:
        raise PdaError(rc, last_error())
    return rc


def make_options(variant="auto", waves_per_cu=0, min_blocks_per_wave=0, chunks_per_wave=0,
                 min_blocks_per_chunk=0) -> Options:
    v = _VARIANTS[variant] if isinstance(variant, str) else int(variant)
    return Options(v, int(waves_per_cu), int(min_blocks_per_wave), int(chunks_per_wave),
                   int(min_blocks_per_chunk))


def raw_call(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, softmax_scale,
             problem: Problem, options: Options | None = None, stream=None) -> int:
    """pda_paged_decode_attention with integer pointers; returns the status code."""
    return _lib.pda_paged_decode_attention(
        q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, ctypes.c_float(softmax_scale),
        ctypes.byref(problem), ctypes.byref(options) if options is not None else None, stream)


def raw_call_noalloc(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, softmax_scale,
                     problem: Problem, options: Options | None = None, stream=None) -> int:
    """pda_paged_decode_attention_noalloc with integer pointers; returns the status code."""
    return _lib.pda_paged_decode_attention_noalloc(
        q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, ctypes.c_float(softmax_scale),
        ctypes.byref(problem), ctypes.byref(options) if options is not None else None, stream)


def raw_call_shared_prefix(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, softmax_scale,
                           group_size, shared_blocks, problem: Problem, options: Options | None = None,
                           stream=None) -> int:
    """pda_paged_decode_attention_shared_prefix with integer pointers; returns the status code."""
    return _lib.pda_paged_decode_attention_shared_prefix(
        q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, ctypes.c_float(softmax_scale),
        int(group_size), shared_blocks, ctypes.byref(problem),
        ctypes.byref(options) if options is not None else None, stream)


def raw_kv_append(k_new, v_new, k_cache, v_cache, kv_scales, block_table, positions, problem: AppendProblem,
                  stream=None) -> int:
    """pda_paged_kv_append with integer pointers; returns the status code."""
    return _lib.pda_paged_kv_append(k_new, v_new, k_cache, v_cache, kv_scales, block_table, positions,
                                    ctypes.byref(problem), stream)


def raw_prefill(q, q_offsets, k_cache, v_cache, block_table, seq_lens, kv_scales, out, softmax_scale,
                problem: PrefillProblem, stream=None) -> int:
    """pda_paged_prefill_attention with integer pointers; returns the status code."""
    return _lib.pda_paged_prefill_attention(q, q_offsets, k_cache, v_cache, block_table, seq_lens, kv_scales, out,
                                            ctypes.c_float(softmax_scale), ctypes.byref(problem), stream)


def query_plan_shared_prefix(problem: Problem, group_size: int, options: Options | None = None,
                             softmax_scale: float = 1.0, num_compute_units: int = 256) -> PlanInfo:
    info = PlanInfo()
    _check(_lib.pda_query_plan_shared_prefix(ctypes.byref(problem),
                                             ctypes.byref(options) if options is not None else None,
                                             ctypes.c_float(softmax_scale), int(group_size),
                                             int(num_compute_units), ctypes.byref(info)))
    return info


def query_plan(problem: Problem, options: Options | None = None, softmax_scale: float = 1.0,
               num_compute_units: int = 256) -> PlanInfo:
    info = PlanInfo()
    _check(_lib.pda_query_plan(ctypes.byref(problem),
                               ctypes.byref(options) if options is not None else None,
                               ctypes.c_float(softmax_scale), int(num_compute_units), ctypes.byref(info)))
    return info


# ------------------------------------------------------------------ torch front end
#
# A small call's kernels take 3-5 us, so what is done per call here counts:
# checks are one pass over the tensors (the error to raise is worked out only
# when one fails), the device is switched only when it is not the current one,
# and default options are passed as NULL. Nothing is remembered between calls.

def _torch():
    if _torch_rt is None:
        raise ImportError("the torch front end needs torch")
    return _torch_rt


if _torch_rt is not None:
    _DTYPES = {_torch_rt.float32: F32, _torch_rt.bfloat16: BF16, _torch_rt.uint8: FP8_E4M3,
               _torch_rt.float8_e4m3fn: FP8_E4M3}
    _INT32, _FLOAT32 = _torch_rt.int32, _torch_rt.float32
    # the current stream's handle without a Stream object around it
    _raw_stream = getattr(_torch_rt._C, "_cuda_getCurrentRawStream", None)


def _dtype_code(t, what):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: unsupported dtype {t.dtype}")
    return code


def _stream_handle(stream, device):
    if stream is None:
        stream = _torch().cuda.current_stream(device)
    return stream.cuda_stream


def _check_tensors(tensors):
    """Every tensor contiguous on the first one's HIP device (its index is returned)."""
    first = next(iter(tensors.values()))
    index = first.get_device()
    if first.is_cuda:
        for t in tensors.values():
            if t.get_device() != index or not t.is_contiguous():
                break
        else:
            return index
    dev = first.device
    for name, t in tensors.items():
        if not t.is_cuda or t.device != dev:
            raise ValueError(f"{name} must be on {dev}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    return index


def _launch(fn, index, stream, *args):
    """fn(*args, stream) with device ``index`` current; raises on an error code."""
    cuda = _torch_rt.cuda
    if stream is None and _raw_stream is not None:
        handle = _raw_stream(index)
    else:
        handle = _stream_handle(stream, index)
    if index == cuda.current_device():
        rc = fn(*args, handle)
    else:
        with cuda.device(index):
            rc = fn(*args, handle)
    if rc != OK:
        _check(rc)


def problem_for(q, k_cache, v_cache, block_table, seq_lens, max_seq_len=0, out=None) -> Problem:
    """Problem descriptor from tensor shapes and dtypes (checks they agree).
    q is [num_seqs, num_q_heads, head_dim], or [num_seqs, q_tokens, num_q_heads,
    head_dim] for several query tokens per sequence."""
    qs, ks, bts = q.shape, k_cache.shape, block_table.shape
    if len(qs) == 4:
        B, ntok, hq, d = qs
    elif len(qs) == 3:
        (B, hq, d), ntok = qs, 1
    else:
        raise ValueError("q must be [num_seqs, num_q_heads, head_dim] or [num_seqs, q_tokens, num_q_heads, head_dim]")
    if len(ks) != 4 or v_cache.dim() != 4:
        raise ValueError("k_cache must be [NB, Hkv, 16, D] and v_cache [NB, Hkv, D, 16]")
    nb, hkv, bs, dk = ks
    if v_cache.shape != (nb, hkv, dk, bs):
        raise ValueError(f"v_cache shape {tuple(v_cache.shape)} != {(nb, hkv, dk, bs)} (dim-major tiles)")
    if dk != d:
        raise ValueError(f"head_dim mismatch: q {d}, cache {dk}")
    if len(bts) != 2 or bts[0] != B:
        raise ValueError("block_table must be [num_seqs, max_blocks_per_seq]")
    if seq_lens.shape != (B,):
        raise ValueError("seq_lens must be [num_seqs]")
    kv_dt = _dtype_code(k_cache, "k_cache")
    if _dtype_code(v_cache, "v_cache") != kv_dt:
        raise TypeError("k_cache and v_cache dtypes differ")
    q_dt = _dtype_code(q, "q")
    out_dt = _dtype_code(out, "out") if out is not None else q_dt
    return Problem(B, hq, hkv, d, bs, bts[1], nb, int(max_seq_len), q_dt, kv_dt, out_dt, ntok)


def paged_decode_attention(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out,
                           softmax_scale, max_seq_len=0, stream=None, variant="auto",
                           waves_per_cu=0, min_blocks_per_wave=0, chunks_per_wave=0,
                           min_blocks_per_chunk=0):
    """Enqueue one decode-attention step on ``stream`` (default: torch's current stream).

    All tensors live on the same HIP device and are contiguous; layouts and
    dtypes are those of include/pda.h (k_cache [NB, Hkv, 16, D], v_cache
    [NB, Hkv, D, 16], fp8 caches as uint8 or float8_e4m3fn codes plus
    kv_scales [2, NB, Hkv] fp32). ``out`` has q's shape and q's dtype or float32.
    """
    prob, opts, index = _prepare(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, max_seq_len,
                                 variant, waves_per_cu, min_blocks_per_wave, chunks_per_wave, min_blocks_per_chunk)
    _launch(_lib.pda_paged_decode_attention, index, stream, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
            block_table.data_ptr(), seq_lens.data_ptr(), kv_scales.data_ptr() if kv_scales is not None else None,
            out.data_ptr(), float(softmax_scale), prob, opts)
    return out


def paged_decode_attention_noalloc(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out,
                                   softmax_scale, max_seq_len=0, stream=None, variant="auto",
                                   waves_per_cu=0, min_blocks_per_wave=0, chunks_per_wave=0,
                                   min_blocks_per_chunk=0):
    """paged_decode_attention through the entry point that allocates nothing:
    its workspace is the library's fixed per-device scratch array
    (NOALLOC_SCRATCH_BYTES), shared by every call on the device."""
    prob, opts, index = _prepare(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, max_seq_len,
                                 variant, waves_per_cu, min_blocks_per_wave, chunks_per_wave, min_blocks_per_chunk)
    _launch(_lib.pda_paged_decode_attention_noalloc, index, stream, q.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
            kv_scales.data_ptr() if kv_scales is not None else None, out.data_ptr(), float(softmax_scale), prob, opts)
    return out


def paged_decode_attention_shared_prefix(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out,
                                         softmax_scale, group_size, shared_blocks, max_seq_len=0, stream=None,
                                         variant="auto", waves_per_cu=0, min_blocks_per_wave=0,
                                         chunks_per_wave=0, min_blocks_per_chunk=0):
    """The same step for groups of ``group_size`` consecutive sequences whose
    block tables share leading blocks; ``shared_blocks`` is an int32 device
    tensor [num_seqs / group_size] bounding each group's shared blocks (the
    library checks the bound against the block tables)."""
    prob, opts, index = _prepare(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, max_seq_len,
                                 variant, waves_per_cu, min_blocks_per_wave, chunks_per_wave, min_blocks_per_chunk)
    if shared_blocks.device != q.device or not shared_blocks.is_contiguous() or shared_blocks.dtype != _INT32:
        raise ValueError(f"shared_blocks must be a contiguous int32 tensor on {q.device}")
    if group_size < 1 or q.shape[0] % group_size or shared_blocks.numel() != q.shape[0] // group_size:
        raise ValueError("shared_blocks must have num_seqs / group_size entries")
    _launch(_lib.pda_paged_decode_attention_shared_prefix, index, stream, q.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
            kv_scales.data_ptr() if kv_scales is not None else None, out.data_ptr(), float(softmax_scale),
            int(group_size), shared_blocks.data_ptr(), prob, opts)
    return out


def _prepare(q, k_cache, v_cache, block_table, seq_lens, kv_scales, out, max_seq_len, variant, waves_per_cu,
             min_blocks_per_wave, chunks_per_wave, min_blocks_per_chunk):
    """(problem, options or None for the defaults, device index) of a decode call, checked."""
    tensors = {"q": q, "k_cache": k_cache, "v_cache": v_cache, "block_table": block_table,
               "seq_lens": seq_lens, "out": out}
    if kv_scales is not None:
        tensors["kv_scales"] = kv_scales
    index = _check_tensors(tensors)
    if block_table.dtype != _INT32 or seq_lens.dtype != _INT32:
        raise TypeError("block_table and seq_lens must be int32")
    if kv_scales is not None and kv_scales.dtype != _FLOAT32:
        raise TypeError("kv_scales must be float32")
    if out.shape != q.shape or (out.dtype != q.dtype and out.dtype != _FLOAT32):
        raise ValueError("out must have q's shape, and q's dtype or float32")
    prob = problem_for(q, k_cache, v_cache, block_table, seq_lens, max_seq_len, out)
    if kv_scales is not None and kv_scales.shape != (2, prob.num_blocks, prob.num_kv_heads):
        raise ValueError("kv_scales must be [2, num_blocks, num_kv_heads]")
    if variant == "auto" and waves_per_cu == min_blocks_per_wave == chunks_per_wave == min_blocks_per_chunk == 0:
        return prob, None, index
    return prob, make_options(variant, waves_per_cu, min_blocks_per_wave, chunks_per_wave,
                              min_blocks_per_chunk), index


def paged_kv_append(k_new, v_new, k_cache, v_cache, kv_scales, block_table, positions, stream=None):
    """Enqueue the write of one decode step's new keys / values ([B, Hkv, D],
    float32 or bfloat16) into the paged cache at ``positions`` (int32 [B]);
    layouts as for paged_decode_attention. fp8 caches update ``kv_scales``."""
    # Shapes first: the kernel reads block_table[b, :] for every b < B, so a
    # table with fewer rows (or a flat one) would be read past its end.
    ns, ks, bts = k_new.shape, k_cache.shape, block_table.shape
    if len(ns) != 3 or v_new.shape != ns or v_new.dtype != k_new.dtype:
        raise ValueError("k_new and v_new must both be [B, Hkv, D] with one dtype")
    B, hkv, d = ns
    if len(ks) != 4 or v_cache.dim() != 4:
        raise ValueError("k_cache must be [NB, Hkv, 16, D] and v_cache [NB, Hkv, D, 16]")
    nb, hkv2, bs, d2 = ks
    if hkv2 != hkv or d2 != d or v_cache.shape != (nb, hkv, d, bs) or positions.shape != (B,):
        raise ValueError("shapes: k_cache [NB, Hkv, 16, D], v_cache [NB, Hkv, D, 16], positions [B]")
    if len(bts) != 2 or bts[0] != B:
        raise ValueError(f"block_table must be [B, max_blocks_per_seq] with B = {B} rows (one per new token), "
                         f"got {tuple(bts)}")
    tensors = {"k_new": k_new, "v_new": v_new, "k_cache": k_cache, "v_cache": v_cache,
               "block_table": block_table, "positions": positions}
    if kv_scales is not None:
        tensors["kv_scales"] = kv_scales
    index = _check_tensors(tensors)
    if block_table.dtype != _INT32 or positions.dtype != _INT32:
        raise TypeError("block_table and positions must be int32")
    kv_dt = _dtype_code(k_cache, "k_cache")
    if kv_dt == FP8_E4M3 and (kv_scales is None or kv_scales.shape != (2, nb, hkv)
                              or kv_scales.dtype != _FLOAT32):
        raise ValueError("an fp8 cache needs float32 kv_scales [2, num_blocks, num_kv_heads]")
    prob = AppendProblem(B, hkv, d, bs, bts[1], nb, _dtype_code(k_new, "k_new"), kv_dt)
    _launch(_lib.pda_paged_kv_append, index, stream, k_new.data_ptr(), v_new.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), kv_scales.data_ptr() if kv_scales is not None else None, block_table.data_ptr(),
            positions.data_ptr(), prob)


def paged_prefill_attention(q, q_offsets, k_cache, v_cache, block_table, seq_lens, kv_scales, out,
                            softmax_scale, max_seq_len=0, stream=None):
    """Enqueue the causal attention of packed query tokens over the paged cache.

    q and out are [T, Hq, D] (q bfloat16; out bfloat16 or float32); rows
    q_offsets[b] .. q_offsets[b + 1] - 1 (int32 [B + 1]) are the last tokens of
    sequence b, whose cache holds seq_lens[b] tokens; cache layouts as for
    paged_decode_attention. A call of at least PDA_PREFILL_IMAGE_MIN_TILES
    (default 5, 8 for fp8; 10 and 13 for lengths bounded by 1,024) tiles of 256 / G
    query tokens per sequence on average converts
    the cache tiles it reads into an image in the stream's workspace (V as fp16,
    an fp8 cache's K as bf16; NB * Hkv * 16 * D * 2 bytes, twice that for fp8)
    unless that exceeds PDA_PREFILL_IMAGE_MAX_MB (default 8192); with fewer on
    average but 100 in all it does so for the sequences that have that many;
    otherwise the kernel converts tiles in registers. The results are the same
    bit for bit.
    """
    tensors = {"q": q, "q_offsets": q_offsets, "k_cache": k_cache, "v_cache": v_cache,
               "block_table": block_table, "seq_lens": seq_lens, "out": out}
    if kv_scales is not None:
        tensors["kv_scales"] = kv_scales
    index = _check_tensors(tensors)
    if q.dim() != 3:
        raise ValueError("q must be [num_tokens, num_q_heads, head_dim]")
    T, hq, d = q.shape
    if k_cache.dim() != 4 or v_cache.dim() != 4:
        raise ValueError("k_cache must be [NB, Hkv, 16, D] and v_cache [NB, Hkv, D, 16]")
    nb, hkv, bs, dk = k_cache.shape
    if tuple(v_cache.shape) != (nb, hkv, dk, bs) or dk != d:
        raise ValueError("cache shapes must be k [NB, Hkv, 16, D], v [NB, Hkv, D, 16] with q's D")
    if block_table.dim() != 2 or seq_lens.dim() != 1 or block_table.shape[0] != seq_lens.shape[0]:
        raise ValueError("block_table must be [num_seqs, max_blocks_per_seq] and seq_lens [num_seqs]")
    B = seq_lens.shape[0]
    if q_offsets.shape != (B + 1,):
        raise ValueError("q_offsets must be [num_seqs + 1]")
    if any(t.dtype != _INT32 for t in (q_offsets, block_table, seq_lens)):
        raise TypeError("q_offsets, block_table and seq_lens must be int32")
    if out.shape != q.shape:
        raise ValueError("out must have q's shape")
    kv_dt = _dtype_code(k_cache, "k_cache")
    if _dtype_code(v_cache, "v_cache") != kv_dt:
        raise TypeError("k_cache and v_cache dtypes differ")
    if kv_scales is not None and (tuple(kv_scales.shape) != (2, nb, hkv) or kv_scales.dtype != _FLOAT32):
        raise ValueError("kv_scales must be float32 [2, num_blocks, num_kv_heads]")
    prob = PrefillProblem(B, T, hq, hkv, d, bs, block_table.shape[1], nb, int(max_seq_len),
                          _dtype_code(q, "q"), kv_dt, _dtype_code(out, "out"))
    _launch(_lib.pda_paged_prefill_attention, index, stream, q.data_ptr(), q_offsets.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
            kv_scales.data_ptr() if kv_scales is not None else None, out.data_ptr(), float(softmax_scale), prob)
    return out


# ------------------------------------------------------------------ around attention
#
# _pda_torch reads the tensors and makes the call where every argument is as it
# has to be, and the device is the current one. For any other the code here works out
# what to raise, or makes the call (host time of a call: 2.7 - 7.4 us from here, below
# 1.5 us so, and 2.5 us for each kernel's launch).

if _torch_rt is not None:
    _FLOATS = {_torch_rt.float32: F32, _torch_rt.bfloat16: BF16}
    _TARGETS = {_torch_rt.int64: 1, _torch_rt.int32: 0}
    _current_device = getattr(_torch_rt._C, "_cuda_getDevice", _torch_rt.cuda.current_device)


def _direct(name, first, stream, *args):
    """The call's code from _pda_torch, or None: not made."""
    index = first.get_device()
    if index < 0 or index != _current_device() or _raw_stream is None or name not in _calls:
        return None
    call, entry = _calls[name]
    rc = call(entry, _raw_stream(index) if stream is None else stream.cuda_stream, *args)
    if rc:
        _check(rc)
    return rc


def _refuse(index, strided, packed):
    """Raise what keeps the tensors of a call from being on HIP device ``index``, or ``packed`` ones contiguous."""
    if index < 0:
        raise ValueError(f"{next(iter(strided))} must be on a HIP device")
    for name, t in {**strided, **packed}.items():
        if t is not None and t.get_device() != index:
            raise ValueError(f"{name} must be on HIP device {index}")
    for name, t in packed.items():
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _apart(index, strided, packed):
    """Whether some tensor is off HIP device ``index``, or one of ``packed`` not contiguous (None passes)."""
    if index < 0:
        return True
    for t in strided:
        if t is not None and t.get_device() != index:
            return True
    for t in packed:
        if t is not None and (t.get_device() != index or not t.is_contiguous()):
            return True
    return False


def _heads(t, name, shape=None, dtype=None):
    """Elements between the tokens of t [T, H, D], whose heads must be contiguous (0: one token)."""
    s = t.shape
    if len(s) != 3 or (shape is not None and s != shape):
        raise ValueError(f"{name} must be {'[tokens, heads, head_dim]' if shape is None else tuple(shape)}, got {tuple(s)}")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    step, head, one = t.stride()
    if one == 1 and head == s[2] and step >= s[1] * head and s[0] > 1:
        return step
    if (one != 1 and s[2] > 1) or (head != s[2] and s[1] > 1):
        raise ValueError(f"{name}: a token's heads must be contiguous")
    if s[0] <= 1:
        return 0
    if step < s[1] * s[2]:
        raise ValueError(f"{name}: tokens must not overlap (an expanded tensor needs .contiguous())")
    return step


def _ptr(t):
    return None if t is None else t.data_ptr()


def _float_code(t, name):
    code = _FLOATS.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return code


def _rope_problem(q, k, q_weight, k_weight, cos_sin, positions, out_code, eps, interleaved, q_stride, k_stride, v_stride,
                  q_out_stride, k_out_stride, grad_q_stride=0, grad_k_stride=0):
    T, hq, d = q.shape
    Tk, hkv, dk = k.shape
    if Tk != T or dk != d:
        raise ValueError(f"k {tuple(k.shape)} must have q's tokens and head_dim {tuple(q.shape)}")
    if cos_sin.dtype is not _FLOAT32 or cos_sin.dim() != 2:
        raise ValueError("cos_sin must be float32 [max_positions, rotary_dim]")
    P, rot = cos_sin.shape
    if positions is not None and (positions.dtype is not _INT32 or positions.shape != (T,)):
        raise ValueError("positions must be int32 [tokens]")
    w = F32
    if q_weight is not None:
        if k_weight is None or q_weight.shape != (d,) or k_weight.shape != (d,) or q_weight.dtype is not k_weight.dtype:
            raise ValueError("q_weight and k_weight must both be [head_dim], of one dtype, or both None")
        w = _float_code(q_weight, "q_weight")
    elif k_weight is not None:
        raise ValueError("q_weight and k_weight must both be given, or both None")
    return RopeProblem(T, hq, hkv, d, rot, P, 1 if interleaved else 0, _float_code(q, "q"), out_code, w, eps, q_stride,
                       k_stride, v_stride, q_out_stride, k_out_stride, grad_q_stride, grad_k_stride)


def paged_qk_norm_rope_append(q, k, v, q_weight, k_weight, cos_sin, q_offsets, k_cache, v_cache, kv_scales,
                              block_table, seq_lens, q_out, eps=1e-6, interleaved=False, positions=None,
                              max_seq_len=0, stream=None):
    """Enqueue the norm and rotation of new tokens' queries and keys and the write
    of their keys and values into the paged cache, in one launch.

    q [T, Hq, D], k and v [T, Hkv, D] (float32 or bfloat16; views of a packed
    projection need no copy); rows q_offsets[b] .. q_offsets[b + 1] - 1 (int32 [B +
    1], or None: T / B tokens each) are the last tokens of sequence b, whose length
    with them is seq_lens[b]. q_weight, k_weight [D], or both None: rotation alone.
    cos_sin [max_positions, rotary_dim] float32 holds each position's cosines, then
    its sines; ``positions`` [T] int32 names rows of it other than the tokens' places.
    The rotated queries go to q_out [T, Hq, D]; cache layouts and fp8 scales as for
    paged_kv_append.
    """
    if _direct("paged_qk_norm_rope_append", q, stream, q, k, v, q_weight, k_weight, cos_sin,
               q_offsets, k_cache, v_cache, kv_scales, block_table, seq_lens, q_out, eps, interleaved, positions,
               max_seq_len) == OK:
        return q_out
    index = q.get_device()
    if _apart(index, (q, k, v, q_out), (cos_sin, k_cache, v_cache, block_table, seq_lens, q_weight, k_weight, q_offsets,
                                        kv_scales, positions)):
        _refuse(index, {"q": q, "k": k, "v": v, "q_out": q_out},
                {"cos_sin": cos_sin, "k_cache": k_cache, "v_cache": v_cache, "block_table": block_table,
                 "seq_lens": seq_lens, "q_weight": q_weight, "k_weight": k_weight, "q_offsets": q_offsets,
                 "kv_scales": kv_scales, "positions": positions})
    dt, ks = q.dtype, k.shape
    qs = _heads(q, "q")
    pr = _rope_problem(q, k, q_weight, k_weight, cos_sin, positions, _float_code(q_out, "q_out"), eps, interleaved, qs,
                       _heads(k, "k", None, dt), _heads(v, "v", ks, dt), _heads(q_out, "q_out", q.shape), 0)
    shape, bts = k_cache.shape, block_table.shape
    if len(shape) != 4 or shape[1] != ks[1] or shape[3] != ks[2] or v_cache.shape != (shape[0], shape[1], shape[3], shape[2]):
        raise ValueError("shapes: k_cache [NB, Hkv, 16, D], v_cache [NB, Hkv, D, 16]")
    if len(bts) != 2 or seq_lens.shape != bts[:1]:
        raise ValueError("block_table must be [num_seqs, max_blocks_per_seq] and seq_lens [num_seqs]")
    if block_table.dtype is not _INT32 or seq_lens.dtype is not _INT32:
        raise TypeError("block_table and seq_lens must be int32")
    if q_offsets is not None and (q_offsets.shape != (bts[0] + 1,) or q_offsets.dtype is not _INT32):
        raise ValueError("q_offsets must be int32 [num_seqs + 1]")
    kv_dt = _dtype_code(k_cache, "k_cache")
    if _dtype_code(v_cache, "v_cache") != kv_dt:
        raise TypeError("k_cache and v_cache dtypes differ")
    if kv_dt == FP8_E4M3 and (kv_scales is None or kv_scales.shape != (2, shape[0], shape[1]) or kv_scales.dtype is not _FLOAT32):
        raise ValueError("an fp8 cache needs float32 kv_scales [2, num_blocks, num_kv_heads]")
    _launch(_lib.pdaops_paged_qk_norm_rope_append, index, stream, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(q_weight),
            _ptr(k_weight), cos_sin.data_ptr(), _ptr(positions), _ptr(q_offsets), q_out.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), _ptr(kv_scales), block_table.data_ptr(), seq_lens.data_ptr(), pr,
            Cache(bts[0], shape[2], bts[1], max_seq_len, shape[0], kv_dt))
    return q_out


def qk_norm_rope(q, k, q_weight, k_weight, cos_sin, positions, q_out, k_out, eps=1e-6, interleaved=False, stream=None):
    """Enqueue the norm and rotation of q [T, Hq, D] and k [T, Hkv, D] (as for
    paged_qk_norm_rope_append) at ``positions`` [T] int32 into q_out and k_out."""
    if _direct("qk_norm_rope", q, stream, q, k, q_weight, k_weight, cos_sin, positions,
               q_out, k_out, eps, interleaved) == OK:
        return q_out, k_out
    index = q.get_device()
    if _apart(index, (q, k, q_out, k_out), (cos_sin, positions, q_weight, k_weight)):
        _refuse(index, {"q": q, "k": k, "q_out": q_out, "k_out": k_out},
                {"cos_sin": cos_sin, "positions": positions, "q_weight": q_weight, "k_weight": k_weight})
    qs = _heads(q, "q")
    pr = _rope_problem(q, k, q_weight, k_weight, cos_sin, positions, _float_code(q_out, "q_out"), eps, interleaved, qs,
                       _heads(k, "k", None, q.dtype), 0, _heads(q_out, "q_out", q.shape),
                       _heads(k_out, "k_out", k.shape, q_out.dtype))
    _launch(_lib.pdaops_qk_norm_rope, index, stream, q.data_ptr(), k.data_ptr(), _ptr(q_weight), _ptr(k_weight),
            cos_sin.data_ptr(), positions.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), pr)
    return q_out, k_out


def qk_norm_rope_backward(q, k, q_weight, k_weight, cos_sin, positions, grad_q_out, grad_k_out, grad_q, grad_k,
                          grad_q_weight=None, grad_k_weight=None, eps=1e-6, interleaved=False, stream=None):
    """Enqueue the gradient of qk_norm_rope: grad_q, grad_k (q's dtype) from
    grad_q_out, grad_k_out, and with weights grad_q_weight, grad_k_weight [D]
    float32, which are written, not added to."""
    if _direct("qk_norm_rope_backward", q, stream, q, k, q_weight, k_weight,
               cos_sin, positions, grad_q_out, grad_k_out, grad_q, grad_k, grad_q_weight, grad_k_weight, eps, interleaved) == OK:
        return grad_q, grad_k
    index = q.get_device()
    if _apart(index, (q, k, grad_q_out, grad_k_out, grad_q, grad_k),
              (cos_sin, positions, q_weight, k_weight, grad_q_weight, grad_k_weight)):
        _refuse(index, {"q": q, "k": k, "grad_q_out": grad_q_out, "grad_k_out": grad_k_out, "grad_q": grad_q,
                        "grad_k": grad_k},
                {"cos_sin": cos_sin, "positions": positions, "q_weight": q_weight, "k_weight": k_weight,
                 "grad_q_weight": grad_q_weight, "grad_k_weight": grad_k_weight})
    dt, qs, ks = q.dtype, q.shape, k.shape
    code, step = _float_code(q, "q"), _heads(q, "q")
    pr = _rope_problem(q, k, q_weight, k_weight, cos_sin, positions, code, eps, interleaved, step, _heads(k, "k", None, dt), 0,
                       _heads(grad_q_out, "grad_q_out", qs, dt), _heads(grad_k_out, "grad_k_out", ks, dt),
                       _heads(grad_q, "grad_q", qs, dt), _heads(grad_k, "grad_k", ks, dt))
    if q_weight is not None:
        for name, t in (("grad_q_weight", grad_q_weight), ("grad_k_weight", grad_k_weight)):
            if t is None or t.dtype is not _FLOAT32 or t.shape != q_weight.shape:
                raise ValueError(f"{name} must be float32 [head_dim]")
    _launch(_lib.pdaops_qk_norm_rope_backward, index, stream, q.data_ptr(), k.data_ptr(), _ptr(q_weight), _ptr(k_weight),
            cos_sin.data_ptr(), positions.data_ptr(), grad_q_out.data_ptr(), grad_k_out.data_ptr(), grad_q.data_ptr(),
            grad_k.data_ptr(), _ptr(grad_q_weight), _ptr(grad_k_weight), pr)
    return grad_q, grad_k


def _row_step(t, name):
    """Elements between the rows of t [T, V], whose words must be contiguous (0: one row)."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be [tokens, vocab]")
    T, V = t.shape
    step, one = t.stride()
    if one != 1 and V > 1:
        raise ValueError(f"{name}: rows must be contiguous")
    if T <= 1:
        return 0
    if step < V:
        raise ValueError(f"{name}: rows must not overlap (an expanded tensor needs .contiguous())")
    return step


def _logits_problem(logits, targets, temperature):
    step = _row_step(logits, "logits")
    T, V = logits.shape
    kind = _TARGETS.get(targets.dtype)
    if kind is None or targets.shape != (T,):
        raise ValueError("targets must be int64 or int32 [tokens]")
    return LogitsProblem(T, V, step, _float_code(logits, "logits"), kind, temperature)


def _rows(T, tensors):
    for t in tensors:
        if t is not None and (t.dtype is not _FLOAT32 or t.shape != (T,)):
            raise ValueError("log-probabilities, entropies, advantages and weights must be float32 [tokens]")


def token_logprobs(logits, targets, logprobs, entropy=None, temperature=1.0, stream=None):
    """Enqueue the log-probabilities of ``targets`` (int64 or int32 [T]; negative:
    a row that takes no part) under logits [T, V] / temperature, and the rows'
    entropies, into float32 [T] tensors. Rows of logits may be apart."""
    if _direct("token_logprobs", logits, stream, logits, targets, logprobs,
               entropy, temperature) == OK:
        return logprobs
    index = logits.get_device()
    if _apart(index, (logits,), (targets, logprobs, entropy)):
        _refuse(index, {"logits": logits}, {"targets": targets, "logprobs": logprobs, "entropy": entropy})
    pr = _logits_problem(logits, targets, temperature)
    _rows(pr.num_tokens, (logprobs, entropy))
    _launch(_lib.pdaops_token_logprobs, index, stream, logits.data_ptr(), targets.data_ptr(), logprobs.data_ptr(),
            _ptr(entropy), pr)
    return logprobs


def policy_loss(logits, targets, old_logprobs, advantages, weights, stats, dlogits=None, logprobs=None, entropy=None,
                ref_logprobs=None, clip_low=0.2, clip_high=0.2, dual_clip=0.0, kl_coef=0.0, entropy_coef=0.0,
                temperature=1.0, grad_scale=1.0, stream=None):
    """Enqueue the clipped policy loss with its KL and entropy terms and its
    gradient at the logits.

    old_logprobs, advantages, weights (and ref_logprobs) are float32 [T]; ``stats``
    float32 [8] gets the weighted sums named in POLICY_STATS, the loss first;
    ``dlogits`` [T, V] of the logits' dtype (may be ``logits``; None: the loss alone)
    grad_scale times its gradient; ``logprobs`` and ``entropy`` the rows' values.
    """
    if _direct("policy_loss", logits, stream, logits, targets, old_logprobs, advantages,
               weights, stats, dlogits, logprobs, entropy, ref_logprobs, clip_low, clip_high, dual_clip, kl_coef, entropy_coef,
               temperature, grad_scale) == OK:
        return stats
    index = logits.get_device()
    if _apart(index, (logits, dlogits), (targets, old_logprobs, advantages, weights, stats, logprobs, entropy, ref_logprobs)):
        _refuse(index, {"logits": logits, "dlogits": dlogits},
                {"targets": targets, "old_logprobs": old_logprobs, "advantages": advantages, "weights": weights,
                 "stats": stats, "logprobs": logprobs, "entropy": entropy, "ref_logprobs": ref_logprobs})
    pr = _logits_problem(logits, targets, temperature)
    _rows(pr.num_tokens, (old_logprobs, advantages, weights, logprobs, entropy, ref_logprobs))
    if stats.shape != (8,) or stats.dtype is not _FLOAT32:
        raise ValueError("stats must be float32 [8]")
    step = 0
    if dlogits is not None:
        if dlogits.shape != logits.shape or dlogits.dtype is not logits.dtype:
            raise ValueError("dlogits must have the logits' shape and dtype")
        step = _row_step(dlogits, "dlogits")
    _launch(_lib.pdaops_policy_loss, index, stream, logits.data_ptr(), targets.data_ptr(), old_logprobs.data_ptr(),
            _ptr(ref_logprobs), advantages.data_ptr(), weights.data_ptr(), stats.data_ptr(), _ptr(dlogits), _ptr(logprobs),
            _ptr(entropy), pr,
            PolicyOptions(clip_low, clip_high, dual_clip, kl_coef, entropy_coef, grad_scale, step))
    return stats


def _wide(t, name, shape=None, dtype=None):
    """Elements between the rows of t [T, H], whose elements must be contiguous (0: one row)."""
    s = t.shape
    if len(s) != 2 or (shape is not None and s != shape):
        raise ValueError(f"{name} must be {'[tokens, width]' if shape is None else tuple(shape)}, got {tuple(s)}")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    step, one = t.stride()
    if one != 1 and s[1] > 1:
        raise ValueError(f"{name}: rows must be contiguous")
    if s[0] <= 1:
        return 0
    if step < s[1]:
        raise ValueError(f"{name}: rows must not overlap (an expanded tensor needs .contiguous())")
    return step


def add_rms_norm(x, weight, out, residual=None, residual_out=None, scales=None, eps=1e-6, stream=None):
    """Enqueue the residual stream's root-mean-square norm.

    x [T, H] (and ``residual`` [T, H], added to it first) float32 or bfloat16; the sum,
    rounded to x's dtype, goes to ``residual_out`` [T, H] unless None (x or residual
    itself will do); ``weight`` [H] float32 or bfloat16. ``out`` [T, H] is float32,
    bfloat16, or float8_e4m3fn (or uint8) with ``scales`` float32 [T, H / 64], [T, H / 128], or
    [T] or [T, 1]: one scale for each group of neighbours, or each row; out * scales
    stands for the norm. Rows of all but weight and scales may be apart.
    """
    if _direct("add_rms_norm", x, stream, x, weight, out, residual, residual_out, scales, eps) == OK:
        return out
    index = x.get_device()
    strided = {"x": x, "out": out, "residual": residual, "residual_out": residual_out}
    packed = {"weight": weight, "scales": scales}
    if _apart(index, strided.values(), packed.values()):
        _refuse(index, strided, packed)
    steps = [_wide(x, "x")]
    T, H = x.shape
    for name, t in (("residual", residual), ("residual_out", residual_out)):
        steps.append(0 if t is None else _wide(t, name, x.shape, x.dtype))
    steps.append(_wide(out, "out", x.shape))
    if weight.shape != (H,):
        raise ValueError("weight must be [width]")
    code, group = _dtype_code(out, "out"), 0
    if code == FP8_E4M3:
        if scales is None or scales.dtype is not _FLOAT32 or scales.dim() not in (1, 2) or scales.shape[0] != T:
            raise ValueError("an fp8 out needs float32 scales [tokens] or [tokens, groups]")
        n = scales.shape[1] if scales.dim() == 2 else 1
        if n < 1 or H % n:
            raise ValueError(f"scales: {n} groups do not divide the width {H}")
        group = H // n if n > 1 else 0
    elif scales is not None:
        raise ValueError("scales are for an fp8 out")
    _launch(_lib.pdalm_add_rms_norm, index, stream, x.data_ptr(), _ptr(residual), weight.data_ptr(), _ptr(residual_out),
            out.data_ptr(), _ptr(scales),
            NormProblem(T, H, _float_code(x, "x"), code, _float_code(weight, "weight"), group, eps, *steps))
    return out


def add_rms_norm_backward(h, weight, grad_out, grad_h, grad_weight=None, grad_residual=None, eps=1e-6, stream=None):
    """Enqueue the gradient of add_rms_norm at ``h`` [T, H] (its residual_out, or its x
    without residual): ``grad_h`` (the gradient of x and of residual alike; h's dtype)
    from ``grad_out`` and, unless None, ``grad_residual``, that of residual_out; and
    ``grad_weight`` [H] float32 unless None, which is written, not added to."""
    if _direct("add_rms_norm_backward", h, stream, h, weight, grad_out, grad_h, grad_weight, grad_residual, eps) == OK:
        return grad_h
    index = h.get_device()
    strided = {"h": h, "grad_out": grad_out, "grad_h": grad_h, "grad_residual": grad_residual}
    packed = {"weight": weight, "grad_weight": grad_weight}
    if _apart(index, strided.values(), packed.values()):
        _refuse(index, strided, packed)
    step = _wide(h, "h")
    (T, H), dt = h.shape, h.dtype
    steps = [0 if t is None else _wide(t, name, h.shape, dt) for name, t in
             (("grad_residual", grad_residual), ("grad_h", grad_h), ("grad_out", grad_out))]
    if weight.shape != (H,):
        raise ValueError("weight must be [width]")
    if grad_weight is not None and (grad_weight.shape != (H,) or grad_weight.dtype is not _FLOAT32):
        raise ValueError("grad_weight must be float32 [width]")
    code = _float_code(h, "h")
    _launch(_lib.pdalm_add_rms_norm_backward, index, stream, h.data_ptr(), weight.data_ptr(), grad_out.data_ptr(),
            _ptr(grad_residual), grad_h.data_ptr(), _ptr(grad_weight),
            NormProblem(T, H, code, code, _float_code(weight, "weight"), 0, eps, step, *steps))
    return grad_h


def _lists(ids, logprobs, T, names):
    """Places of the lists ids int32 and logprobs float32, both [T, K]."""
    if ids.dim() != 2 or ids.shape[0] != T or ids.dtype is not _INT32:
        raise ValueError(f"{names[0]} must be int32 [tokens, places]")
    if logprobs.shape != ids.shape or logprobs.dtype is not _FLOAT32:
        raise ValueError(f"{names[1]} must be float32, of {names[0]}' shape")
    return ids.shape[1]


def top_logprobs(logits, top_ids, top_logprobs, targets=None, logprobs=None, entropy=None, temperature=1.0, stream=None):
    """Enqueue the most likely words of every row of logits [T, V] / temperature, the
    likeliest first: ``top_ids`` int32 [T, K] and ``top_logprobs`` float32 [T, K], K up to
    MAX_TOP (equal logits in the order of their words; -1 and -inf where no word is
    left); and as token_logprobs the log-probabilities of ``targets`` [T] (negative: a
    row that takes no part) and the rows' entropies, float32 [T], each unless None."""
    if _direct("top_logprobs", logits, stream, logits, top_ids, top_logprobs, targets, logprobs, entropy, temperature) == OK:
        return top_ids, top_logprobs
    index = logits.get_device()
    packed = {"top_ids": top_ids, "top_logprobs": top_logprobs, "targets": targets, "logprobs": logprobs, "entropy": entropy}
    if _apart(index, (logits,), packed.values()):
        _refuse(index, {"logits": logits}, packed)
    if targets is not None:
        pr = _logits_problem(logits, targets, temperature)
    elif logprobs is not None:
        raise ValueError("logprobs are of targets")
    else:
        step = _row_step(logits, "logits")
        pr = LogitsProblem(*logits.shape, step, _float_code(logits, "logits"), 0, temperature)
    places = _lists(top_ids, top_logprobs, pr.num_tokens, ("top_ids", "top_logprobs"))
    _rows(pr.num_tokens, (logprobs, entropy))
    _launch(_lib.pdalm_top_logprobs, index, stream, logits.data_ptr(), _ptr(targets), top_ids.data_ptr(),
            top_logprobs.data_ptr(), _ptr(logprobs), _ptr(entropy), pr, places)
    return top_ids, top_logprobs


def distill_loss(logits, teacher_ids, teacher_logprobs, weights, stats, dlogits=None, losses=None, reverse=0.0, rest=True,
                 temperature=1.0, grad_scale=1.0, stream=None):
    """Enqueue the distillation loss of the student's logits [T, V] from a teacher's
    lists (as top_logprobs writes them: teacher_ids int32 [T, K], -1 an empty place, and
    teacher_logprobs float32 [T, K]) and its gradient at the logits.

    A row's loss is (1 - reverse) KL(teacher || student) + reverse KL(student || teacher)
    over the listed words and, with ``rest``, all others as one outcome; without, the
    sums are over the listed words alone. ``weights`` float32 [T] carry the mask and the
    mean; ``stats`` float32 [6] gets the weighted sums named in DISTILL_STATS, the loss
    first; ``dlogits`` [T, V] of the logits' dtype (may be ``logits``; None: the loss
    alone) grad_scale times its gradient; ``losses`` float32 [T] the rows'.
    """
    if _direct("distill_loss", logits, stream, logits, teacher_ids, teacher_logprobs, weights, stats, dlogits, losses, reverse,
               rest, temperature, grad_scale) == OK:
        return stats
    index = logits.get_device()
    packed = {"teacher_ids": teacher_ids, "teacher_logprobs": teacher_logprobs, "weights": weights, "stats": stats, "losses": losses}
    if _apart(index, (logits, dlogits), packed.values()):
        _refuse(index, {"logits": logits, "dlogits": dlogits}, packed)
    step = _row_step(logits, "logits")
    pr = LogitsProblem(*logits.shape, step, _float_code(logits, "logits"), 0, temperature)
    places = _lists(teacher_ids, teacher_logprobs, pr.num_tokens, ("teacher_ids", "teacher_logprobs"))
    _rows(pr.num_tokens, (weights, losses))
    if stats.shape != (6,) or stats.dtype is not _FLOAT32:
        raise ValueError("stats must be float32 [6]")
    step = 0
    if dlogits is not None:
        if dlogits.shape != logits.shape or dlogits.dtype is not logits.dtype:
            raise ValueError("dlogits must have the logits' shape and dtype")
        step = _row_step(dlogits, "dlogits")
    _launch(_lib.pdalm_distill_loss, index, stream, logits.data_ptr(), teacher_ids.data_ptr(), teacher_logprobs.data_ptr(),
            weights.data_ptr(), stats.data_ptr(), _ptr(losses), _ptr(dlogits), pr,
            DistillOptions(places, 1 if rest else 0, reverse, grad_scale, step))
    return stats


def read_device_status(stream=None, device=None) -> int:
    torch = _torch()
    device = device if device is not None else torch.cuda.current_device()
    with torch.cuda.device(device):
        rc = _lib.pda_read_device_status(_stream_handle(stream, device))
    if rc < 0:
        raise PdaError(rc, last_error())
    return rc


def release_workspaces() -> None:
    _check(_lib.pda_release_workspaces())
