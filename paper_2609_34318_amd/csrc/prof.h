// Optional per-launch event timing used by hydra_profile_start / hydra_profile_stop.
#pragma once
#include <hip/hip_runtime.h>

namespace hydra {
// Every launch calls these, on paths that end at the C interface, which no exception may cross: a launch that finds
// no memory for its record is not timed.
// Returns a token (or -1 when not recording) after recording a start event on `stream`.
int prof_begin(const char* kernel, hipStream_t stream) noexcept;
// Records the end event for `token` on `stream` (no-op for -1).
void prof_end(int token, hipStream_t stream) noexcept;
}  // namespace hydra
