// Shared by the launchers of kernels with more LDS than the default limit.
#pragma once
#include "internal.h"

namespace tabed {

// The limit of a kernel's LDS is raised once for each device.
template <typename K>
inline hipError_t raise_on_device(K kernel, size_t lds, std::once_flag (&once)[kMaxDevices], hipError_t (&rc)[kMaxDevices]) {
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
    return raise_lds_limit(kernel, lds, once[dev], rc[dev]);
}

}  // namespace tabed
