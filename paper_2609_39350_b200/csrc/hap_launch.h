// Host side that the operators' files share: launches and their status, the current device, checks of arguments.
#pragma once
#include "../../include/hap.h"

#include <atomic>
#include <cuda_runtime.h>

// The status of a CUDA call.  A failed one also leaves its error behind, for whoever asks for the last error next: it is taken back.
static inline hap_status status_of(cudaError_t e) { return e == cudaSuccess ? HAP_OK : (cudaGetLastError(), HAP_E_CUDA); }
// Launches, and says whether this launch was made, not whether any call so far left an error behind.  Arguments of the kernel's own
// types are passed where they are, without a copy.
template <typename T> struct Same { using type = T; };
template <typename... P> static hap_status start(void (*kernel)(P...), const cudaLaunchConfig_t &c, const typename Same<P>::type &...args)
{
    void *at[] = {(void *)&args...};
    return status_of(cudaLaunchKernelExC(&c, (const void *)kernel, at));
}
static inline cudaLaunchConfig_t shape_of(int64_t grid, int threads, int smem, cudaStream_t stream)
{
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)grid), c.blockDim = dim3((unsigned)threads), c.dynamicSmemBytes = (size_t)smem, c.stream = stream;
    return c;
}

// The current device and its multiprocessors; 0 of them: no device.  What does not change is asked once for each device.
struct Device { int id = 0, sms = 0; };
constexpr int DEVICES = 64;

static inline Device device()
{
    static std::atomic<int> known[DEVICES];
    Device d;
    if (status_of(cudaGetDevice(&d.id)) != HAP_OK || d.id < 0) return d;
    if (d.id < DEVICES) d.sms = known[d.id].load(std::memory_order_relaxed);
    if (d.sms) return d;
    if (status_of(cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, d.id)) != HAP_OK) d.sms = 0;
    if (d.id < DEVICES) known[d.id].store(d.sms, std::memory_order_relaxed);
    return d;
}

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Launches a kernel that may start while its predecessor in the stream still ends: its setup (barriers, tensor memory, maps) and the
// launch itself then cost nothing (loss of 129 rows: 28.7 -> 25.3 us).  The kernel waits for the predecessor before it reads.
template <typename... P> static hap_status launch_next(void (*kernel)(P...), int64_t grid, int threads, int smem, int cluster, cudaStream_t stream, const typename Same<P>::type &...args)
{
    cudaLaunchConfig_t c = shape_of(grid, threads, smem, stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization, attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension, attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    c.attrs = attr, c.numAttrs = cluster > 1 ? 2 : 1;
    return start(kernel, c, args...);
}

static inline bool dtype16(int32_t t) { return t == HAP_BF16 || t == HAP_FP16; }
static inline int64_t size_of(int32_t t) { return t == HAP_FP32 ? 4 : 2; }
static inline bool aligned(const void *p, int64_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
static inline uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }
