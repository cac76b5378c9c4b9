// What the translation units of libdaspmm.so share on the host.
#pragma once
#include <hip/hip_runtime.h>

namespace daspmm {

// Keeps `text` for da_spmm_last_error() of this thread; returns `code`.
int set_error(int code, const char* text) noexcept;
int set_hip_error(hipError_t e, const char* where) noexcept;

// Compute units of the current device.
int compute_units() noexcept;

}  // namespace daspmm
