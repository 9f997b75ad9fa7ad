// What the entry points of several source files share about workspaces (defined in hetis_attn.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>

namespace hetis {

// Arrival counters of a decode workspace: they follow the control words and sit at the same place
// whatever the shape.  Partial results of any call start behind them, so that calls of different kinds
// can share one workspace.
constexpr size_t kArrivalSlots = (size_t)1 << 18;
constexpr size_t kArrivalBytes = kArrivalSlots * sizeof(unsigned int);
constexpr size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// HETIS_OK, NULL or WORKSPACE (too small, misaligned).
int check_workspace(const void *ws, size_t have, size_t need);
// The library-owned workspace of the current device, at least `need` bytes large.
int owned_workspace(size_t need, hipStream_t st, bool may_be_capturing, void **out);
// Compute units of the current device; 0: HIP reported an error.
int device_cu_count();

}  // namespace hetis
