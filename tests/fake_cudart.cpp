// A CUDA runtime on the host, for tests of the library's host code: two
// devices, "device" memory from malloc, streams as queues of the operations
// that wait to run.  An operation runs when its stream, or the device, is
// waited for, never earlier, so that whatever a call leaves unordered stays
// undone; every stream is ordered by itself alone, the default one too.  A
// kernel is not run: a launch is checked against the attributes that its
// function has on the current device, and counted.
#include <cuda.h>
#include <cuda_runtime_api.h>

#include <cstdlib>
#include <cstring>
#include <deque>
#include <functional>
#include <map>
#include <utility>

namespace {

constexpr int kDevices = 2, kSms = 152;
constexpr size_t kPlainShared = 48 * 1024;  // dynamic shared memory without an attribute

int g_device = 0;
std::map<cudaStream_t, std::deque<std::function<void()>>> g_streams;
std::map<std::pair<int, const void*>, size_t> g_shared;  // (device, function): its limit
std::map<void*, std::pair<size_t, int>> g_memory;        // size, device
void* g_last = nullptr;
int g_launches[kDevices];
int g_attribute_failures = 0, g_malloc_failures = 0;
cudaError_t g_error = cudaSuccess;

cudaError_t result(cudaError_t e)
{
    if (e != cudaSuccess) g_error = e;
    return e;
}
void run(cudaStream_t s)
{
    auto& q = g_streams[s];
    while (!q.empty()) {
        q.front()();
        q.pop_front();
    }
}
void run_all()
{
    for (auto& s : g_streams) run(s.first);
}

CUresult encode(...) { return CUDA_SUCCESS; }

}  // namespace

extern "C" {

// ---- for the tests
int fake_pending()
{
    size_t n = 0;
    for (auto& s : g_streams) n += s.second.size();
    return (int)n;
}
void* fake_last_allocation(size_t* bytes)
{
    *bytes = g_last ? g_memory[g_last].first : 0;
    return g_last;
}
// The only allocation of this size; null when there is none or several.
void* fake_allocation_of(size_t bytes)
{
    void* found = nullptr;
    for (auto& m : g_memory)
        if (m.second.first == bytes) {
            if (found) return nullptr;
            found = m.first;
        }
    return found;
}
int fake_launches(int device) { return g_launches[device]; }
void fake_fail_attributes(int calls) { g_attribute_failures = calls; }
void fake_fail_allocations(int calls) { g_malloc_failures = calls; }
void fake_device_work(cudaStream_t s, int* word, int value)
{
    g_streams[s].push_back([=] { *word = value; });
}

// ---- the runtime
cudaError_t cudaGetDevice(int* d) { return *d = g_device, cudaSuccess; }
cudaError_t cudaSetDevice(int d)
{
    if (d < 0 || d >= kDevices) return result(cudaErrorInvalidDevice);
    return g_device = d, cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int)
{
    return *v = a == cudaDevAttrMultiProcessorCount ? kSms : 0, cudaSuccess;
}
cudaError_t cudaDeviceSynchronize() { return run_all(), cudaSuccess; }
cudaError_t cudaMalloc(void** p, size_t n)
{
    if (g_malloc_failures > 0 && g_malloc_failures--) return result(cudaErrorMemoryAllocation);
    *p = g_last = std::malloc(n);
    std::memset(*p, 0xAB, n);
    g_memory[*p] = {n, g_device};
    return cudaSuccess;
}
cudaError_t cudaFree(void* p)
{
    run_all();
    g_memory.erase(p);
    std::free(p);
    return cudaSuccess;
}
cudaError_t cudaHostAlloc(void** p, size_t n, unsigned) { return *p = std::malloc(n), cudaSuccess; }
cudaError_t cudaFreeHost(void* p) { return std::free(p), cudaSuccess; }
// (returns before it has run, as for device memory)
cudaError_t cudaMemset(void* p, int v, size_t n)
{
    g_streams[nullptr].push_back([=] { std::memset(p, v, n); });
    return cudaSuccess;
}
cudaError_t cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t s)
{
    g_streams[s].push_back([=] { std::memset(p, v, n); });
    return cudaSuccess;
}
cudaError_t cudaMemcpy(void* to, const void* from, size_t n, cudaMemcpyKind)
{
    run(nullptr);
    std::memcpy(to, from, n);
    return cudaSuccess;
}
cudaError_t cudaMemcpyAsync(void* to, const void* from, size_t n, cudaMemcpyKind, cudaStream_t s)
{
    g_streams[s].push_back([=] { std::memcpy(to, from, n); });
    return cudaSuccess;
}
cudaError_t cudaStreamCreateWithFlags(cudaStream_t* s, unsigned)
{
    return *s = static_cast<cudaStream_t>(std::malloc(1)), cudaSuccess;
}
cudaError_t cudaStreamDestroy(cudaStream_t s)
{
    if (g_streams[s].empty()) g_streams.erase(s);  // else its work runs some time later
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t s) { return run(s), cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t, cudaEvent_t, unsigned) { return cudaSuccess; }
cudaError_t cudaEventCreate(cudaEvent_t* e) { return *e = nullptr, cudaSuccess; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t* e, unsigned) { return *e = nullptr, cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventElapsedTime(float* ms, cudaEvent_t, cudaEvent_t) { return *ms = 0, cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void* f, cudaFuncAttribute a, int v)
{
    if (g_attribute_failures > 0 && g_attribute_failures--) return result(cudaErrorUnknown);
    if (a == cudaFuncAttributeMaxDynamicSharedMemorySize) g_shared[{g_device, f}] = v;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void**)
{
    size_t limit = kPlainShared;
    auto it = g_shared.find({g_device, f});
    if (it != g_shared.end() && it->second > limit) limit = it->second;
    if (c->dynamicSmemBytes > limit) return result(cudaErrorInvalidValue);
    ++g_launches[g_device];
    return cudaSuccess;
}
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** fn, unsigned, unsigned long long,
                                             cudaDriverEntryPointQueryResult* q)
{
    *fn = reinterpret_cast<void*>(encode);
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
const char* cudaGetErrorString(cudaError_t) { return "an error of the runtime"; }
cudaError_t cudaGetLastError()
{
    const cudaError_t e = g_error;
    return g_error = cudaSuccess, e;
}
cudaError_t cudaPeekAtLastError() { return g_error; }
cudaError_t cudaGetSymbolAddress(void**, const void*) { return cudaErrorInvalidSymbol; }
cudaError_t cudaPointerGetAttributes(cudaPointerAttributes*, const void*)
{
    return cudaErrorInvalidValue;
}

// ---- what compiled host code registers itself with
void** __cudaRegisterFatBinary(void*) { return nullptr; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, void*, void*, void*, void*,
                            int*)
{
}
void __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
cudaError_t __cudaGetKernel(cudaKernel_t*, const void*) { return cudaErrorUnknown; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void**, size_t, cudaStream_t)
{
    return cudaErrorUnknown;
}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaErrorUnknown; }

}  // extern "C"
