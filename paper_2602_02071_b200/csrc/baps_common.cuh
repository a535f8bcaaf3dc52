// Shared host/device plumbing of the BAPS CUDA library: status word, launch counter, checks.
#pragma once
#include <atomic>
#include <cstdint>
#include <cstdio>
#include <mutex>
#include <cuda_runtime.h>
#include "../../include/baps.h"
#include "baps_register_split.cuh"

namespace baps {

// Device-side status word: 0 = fine; non-zero = a bounded wait expired (the value encodes
// which role gave up).  Read and cleared by baps_poll_async_error().  Each translation unit has its own.
static __device__ int g_async_status = 0;

// Reads and clears the word of the translation unit it is called in (the caller has waited for the stream).
static inline baps_status take_async_status()
{
    int host = 0;
    if (cudaMemcpyFromSymbol(&host, g_async_status, sizeof(int)) != cudaSuccess) return BAPS_ERR_CUDA;
    if (host == 0) return BAPS_OK;
    const int zero = 0;
    return cudaMemcpyToSymbol(g_async_status, &zero, sizeof(int)) == cudaSuccess ? BAPS_ERR_TIMEOUT : BAPS_ERR_CUDA;
}
baps_status take_serving_status();       // that of baps_serving.cu

// Host-side count of kernel launches issued by this library.
inline std::atomic<int64_t> g_launches{0};

// Serialises the one-time, per-device set-up steps (table builds, symbol look-ups) when several
// host threads make their first call at the same time.
inline std::mutex g_setup_mutex;

constexpr float kLog2e = 1.4426950408889634074f;

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline baps_status launch_status()
{
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return BAPS_ERR_CUDA;
    ++g_launches;
    return BAPS_OK;
}

// Programmatic dependent launch.  Every kernel of the library is launched with the attribute that lets it start
// before the kernel ahead of it in the stream has ended, does what needs no caller memory (tables, barriers,
// tensor memory), and waits for that kernel -- its completion, whatever it is -- before it touches any.  The wait
// hands the pointer through, so that no load from it, not even one the compiler takes for invariant, can
// move ahead of the wait.  The allow call is made by every CTA when it starts (attention_d64_kernel: when it has its
// tensor memory): the next kernel then comes in as this one's last CTAs drain.
__device__ __forceinline__ void allow_next_kernel() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void await_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename T>
__device__ __forceinline__ T *await_previous_kernel(T *p)
{
    asm volatile("griddepcontrol.wait;" : "+l"(p) :: "memory");
    return p;
}

// cluster: CTAs per cluster, along x; 0: what the kernel itself says, if anything.
template <typename... P, typename... A>
inline baps_status launch_clusters(void (*kernel)(P...), dim3 grid, unsigned cluster, int threads, size_t smem, cudaStream_t stream, A... args)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = cluster ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return BAPS_ERR_CUDA;
    }
    return launch_status();
}
template <typename... P, typename... A>
inline baps_status launch_kernel(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, A... args)
{
    return launch_clusters(kernel, grid, 0, threads, smem, stream, args...);
}

// Whether the compiled kernel has the registers that its roles share out (see split_fits); asked once per kernel, the
// answer is part of the module image.
template <auto kernel>
static inline bool has_registers_for(const RegisterSplit &split)
{
    static std::atomic<bool> yes{false};
    if (yes.load(std::memory_order_relaxed)) return true;
    cudaFuncAttributes a;
    if (cudaFuncGetAttributes(&a, kernel) != cudaSuccess) { (void)cudaGetLastError(); return false; }
    if (!split_fits(split, a.numRegs)) return false;
    yes.store(true, std::memory_order_relaxed);
    return true;
}

inline bool have_device()
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev >= 0;
}

// Streaming multiprocessors of the current device.
inline int num_sms()
{
    static int cached[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    if (cached[dev] == 0) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
            n = 148;
        cached[dev] = n;
    }
    return cached[dev];
}

inline cudaStream_t as_stream(baps_stream s) { return reinterpret_cast<cudaStream_t>(s); }

} // namespace baps
