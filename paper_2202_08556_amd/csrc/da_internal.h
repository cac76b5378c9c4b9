// What the translation units of libdaspmm.so share on the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

namespace daspmm {

// Keeps `text` for da_spmm_last_error() of this thread; returns `code`.
int set_error(int code, const char* text) noexcept;
int set_hip_error(hipError_t e, const char* where) noexcept;

// Compute units of the current device.
int compute_units() noexcept;

// Kernel may be launched with up to `bytes` of dynamic LDS on the current device, always the same `bytes` for a kernel.  The kernel itself,
// and not its type, is the template's argument: kernels of one signature have flags of their own.
template <auto Kernel> void allow_lds(int bytes) noexcept {
    static std::atomic<uint64_t> allowed{0};                 // devices that know
    int device = 0;
    (void)hipGetDevice(&device);
    const uint64_t bit = 1ull << (device & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit) &&
        hipFuncSetAttribute(reinterpret_cast<const void*>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess)
        allowed.fetch_or(bit, std::memory_order_relaxed);
}

}  // namespace daspmm
