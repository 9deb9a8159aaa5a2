// What the entry points of the C ABI share: alignment, the current device, CUDA errors as a status.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ada.h"

namespace ada {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct DeviceGuard {
    int prev = -1;
    explicit DeviceGuard(int dev) {
        cudaGetDevice(&prev);
        if (prev != dev) cudaSetDevice(dev);
        else prev = -1;
    }
    ~DeviceGuard() {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

}  // namespace ada

#define CU(x)                                  \
    do {                                       \
        cudaError_t e__ = (x);                 \
        if (e__ != cudaSuccess) {              \
            cudaGetLastError(); /* reported by the status; the next launcher that asks must not find it */ \
            return ADA_ERR_CUDA;               \
        }                                      \
    } while (0)
