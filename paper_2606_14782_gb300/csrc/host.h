// Host-side helpers of the C ABI: the calling thread's last message, argument
// checks and the device of a call.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <string>

#include "bacon.h"

namespace bacon {

extern thread_local std::string g_last_error;

// Records the message for bacon_last_error and returns the status.
bacon_status fail(bacon_status st, const char* fmt, ...);
bacon_status cuda_fail(cudaError_t e, const char* what);

#define BACON_CUDA(call, what)                         \
    do {                                               \
        cudaError_t e_ = (call);                       \
        if (e_ != cudaSuccess) return cuda_fail(e_, what); \
    } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Makes the context's device current for the duration of a call.
struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        if (prev != dev) ok = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard()
    {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

}  // namespace bacon
