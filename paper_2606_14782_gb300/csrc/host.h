// Host-side helpers of the C ABI: the calling thread's last message, argument
// checks, the device of a call and words that kernels of any stream rely on.
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

// Zeros `bytes` bytes of the current device's memory before it returns, without
// waiting for other work: on a stream of its own, since the default stream has
// whatever the caller put there, and what it runs late is late for every stream
// that does not wait for it.
inline cudaError_t clear_now(void* p, size_t bytes)
{
    cudaStream_t own;
    cudaError_t e = cudaStreamCreateWithFlags(&own, cudaStreamNonBlocking);
    if (e != cudaSuccess) return e;
    e = cudaMemsetAsync(p, 0, bytes, own);
    if (e == cudaSuccess) e = cudaStreamSynchronize(own);
    const cudaError_t d = cudaStreamDestroy(own);
    return e != cudaSuccess ? e : d;
}

}  // namespace bacon
