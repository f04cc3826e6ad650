// What the translation units of libheinsen_scan share on the host: error text, device check, counters.
#pragma once
#include <cuda_runtime.h>

#include "../../include/heinsen_scan.h"

namespace hs_internal {
#pragma GCC visibility push(hidden)
// Records the message that heinsen_scan_strerror(HS_ERR_CUDA) returns on this thread; returns HS_ERR_CUDA.
hs_status cuda_fail(const char* what, cudaError_t e);
// HS_OK on an sm_100 device, with its number of SMs; HS_ERR_UNSUPPORTED_DEVICE or HS_ERR_CUDA otherwise.
hs_status current_device(int* sm_count);
void count_launches(int n);
// Identifies one call in a workspace header; never 0, not repeated within a process.
unsigned long long call_id();
// What heinsen_scan_debug_config has set: polls of a bounded wait, and the tile (chunk) that is to be left unannounced, or -1.
unsigned int spin_limit();
long long mute_tile();
#pragma GCC visibility pop
}  // namespace hs_internal
