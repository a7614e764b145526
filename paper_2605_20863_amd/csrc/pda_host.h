// What pda_host.cpp offers the host code of further entry points
// (pda_ops_host.cpp): the calling thread's error text, and the stream's workspace.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <mutex>

namespace pda {

// Sets the text of pda_last_error() and returns `code`.
__attribute__((format(printf, 2, 3))) int host_fail(int code, const char* fmt, ...);
int host_fail_hip(hipError_t e, const char* what);
void host_clear_error();

// The (current device, stream) workspace, grown to at least the asked bytes and
// held by `lock` until the call's launches are enqueued. `base` starts with the
// header (kHdrWords words, the status word among them).
struct HeldWorkspace {
  std::unique_lock<std::mutex> lock;
  char* base = nullptr;
  int cus = 0;
  void* record = nullptr;
};
int hold_workspace(hipStream_t s, int64_t bytes, HeldWorkspace* out);

// Arrival counts for one call on a held workspace: kShortUnits words,
// kShortCountStride apart, and the epoch that this call counts from. `words` stays
// null while the stream is captured, whose replays would all have one epoch.
struct Counts {
  uint64_t* words = nullptr;
  uint32_t epoch = 0;
};
int take_counts(hipStream_t s, const HeldWorkspace& ws, Counts* out);

}  // namespace pda
