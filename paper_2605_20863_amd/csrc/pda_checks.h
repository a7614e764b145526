// What the host code of the operators around attention shares (pda_ops_host.cpp,
// pda_lm_host.cpp): checks of pointers and of logits, the cut of their rows into parts,
// arrival counts, and the C entries' way to make exceptions into codes.
#pragma once

#include "pda_ops.h"
#include "pda_host.h"
#include "pda_ops_internal.h"

#include <cmath>
#include <initializer_list>
#include <new>

namespace pda {

constexpr int64_t kMaxWaves = 1 << 26;  // a launch has below 2^32 threads
constexpr int64_t kHeader = 256;        // bytes of the workspace's header
static_assert(kHdrWords * 4 <= kHeader, "header");

struct Ptr {
  const void* p;
  uintptr_t align;
  const char* name;
  bool required;
};

inline int check_pointers(std::initializer_list<Ptr> ptrs) {
  for (const Ptr& x : ptrs) {
    if (x.required && !x.p) return host_fail(PDA_EINVAL, "%s is NULL", x.name);
    if (reinterpret_cast<uintptr_t>(x.p) % x.align)
      return host_fail(PDA_EINVAL, "%s is not %d-byte aligned", x.name, (int)x.align);
  }
  return PDA_OK;
}

inline bool float_type(int t) { return t == PDA_DTYPE_F32 || t == PDA_DTYPE_BF16; }
inline int size_of(int t) { return t == PDA_DTYPE_F32 ? 4 : 2; }

// Arrival counts for the call, unless it is captured.
template <typename Args>
int count(hipStream_t s, const HeldWorkspace& ws, Args* a) {
  Counts c;
  const int rc = take_counts(s, ws, &c);
  a->counts = c.words;
  a->epoch = c.epoch;
  return rc;
}

inline int32_t* status_word(char* base) { return reinterpret_cast<int32_t*>(base) + kHdrStatus; }

inline int check_logits(const pdaops_logits_problem* pr, LogitsArgs* a) {
  if (!pr) return host_fail(PDA_EINVAL, "problem is NULL");
  if (pr->num_tokens < 0) return host_fail(PDA_EINVAL, "num_tokens = %d < 0", pr->num_tokens);
  if (pr->vocab < 1 || pr->vocab > (1 << 30)) return host_fail(PDA_EINVAL, "vocab = %d (1 .. 2^30)", pr->vocab);
  if (!float_type(pr->dtype)) return host_fail(PDA_EINVAL, "dtype = %d (supported: F32, BF16)", pr->dtype);
  if (pr->targets_int64 != 0 && pr->targets_int64 != 1) return host_fail(PDA_EINVAL, "targets_int64 = %d (0 or 1)", pr->targets_int64);
  a->stride = pr->row_stride ? pr->row_stride : pr->vocab;
  if (a->stride < pr->vocab || a->stride > INT64_MAX / 8 / (pr->num_tokens + 1ll))
    return host_fail(PDA_EINVAL, "row_stride = %lld", (long long)pr->row_stride);
  if (!(pr->temperature > 0.f) || !std::isfinite(pr->temperature) || !std::isfinite(1.f / pr->temperature))
    return host_fail(PDA_EINVAL, "temperature must be positive and finite");
  a->T = pr->num_tokens;
  a->V = pr->vocab;
  a->bf16 = pr->dtype == PDA_DTYPE_BF16;
  a->targets64 = pr->targets_int64;
  a->inv_temp = 1.f / pr->temperature;
  return PDA_OK;
}

// Whole 16-byte vectors of a row.
inline int vectors_of(const LogitsArgs& a) { return a.bf16 ? a.V / 8 : a.V / 4; }

// Parts per row: enough workgroups for the compute units, of at least 512 vectors
// (two for each thread) each. Half or twice as many workgroups, or least vectors, are
// within 10% on every size tried (1 to 3,000 rows of 8,000 to 150,000 words) but for
// rows of 8,000 words, which 256 vectors a part cut in two: 5.3 - 9.3 us per call, 4.2 - 7.1 whole.
inline void split_rows(LogitsArgs* a, int64_t least = 512) {
  constexpr int64_t kWgs = 1024;
  const int64_t v = vectors_of(*a);
  int64_t s = (kWgs + a->T - 1) / a->T;
  if (s > v / least) s = v / least;
  if (s > kMaxSplits) s = kMaxSplits;
  if (s < 1) s = 1;
  a->chunk = (int32_t)((v + s - 1) / s);
  if (a->chunk < 1) a->chunk = 1;
  a->splits = (int32_t)((v + a->chunk - 1) / a->chunk);
  if (a->splits < 1) a->splits = 1;
}

// A C entry: what is thrown below it (no memory for the workspace's record, a
// failed lock) becomes an error code with a text, of at most 15 characters: a
// std::string holds these without memory of its own.
template <typename F>
int entry(F run) {
  try {
    return run();
  } catch (const std::bad_alloc&) {
    return host_fail(PDA_ENOMEM, "no host memory");
  } catch (...) {
    return host_fail(PDA_EHIP, "host exception");
  }
}

}  // namespace pda
