// Launch attributes that are set once per kernel and device.
#pragma once
#include <hip/hip_runtime.h>
#include <mutex>

#include "../../include/moe_sb.h"

namespace moe {

// Guards the launch-attribute caches: calls may come from several host threads.
inline std::mutex g_attr_lock;

// The large-LDS attribute of a kernel is set once per device (bit d of *done: device d, d < 64).
inline int ensure_lds_attr(const void* fn, int lds, unsigned long long* done) {
    std::lock_guard<std::mutex> hold(g_attr_lock);
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return MOE_ERR_HIP;
    const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
    if (bit && (*done & bit)) return MOE_OK;
    if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return MOE_ERR_HIP;
    *done |= bit;
    return MOE_OK;
}

}  // namespace moe
