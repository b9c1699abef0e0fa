// More dynamic LDS than a launch may have by default: the limit is a kernel's and a device's, and has to be raised on every device that launches it.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include <atomic>

namespace drf {

// Raises the limit of `kern` on the current device to `bytes`, once: bit i of `done`, which belongs to this kernel alone, says that device i has it.
// Two threads may both find it missing and raise it, to the same.  (Devices from the 64th on are asked every time.)
inline hipError_t allow_lds(const void* kern, int bytes, std::atomic<uint64_t>& done)
{
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    if (done.load(std::memory_order_acquire) & bit) return hipSuccess;
    e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

}  // namespace drf
