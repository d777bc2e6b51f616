// Launching kernels.
#pragma once

#include <atomic>
#include <utility>

#include "dg4_internal.h"

// How many blocks of a kernel the current device holds at once, asked of the runtime once per kernel and device (the
// question costs about 2 us, a quarter of a small call).
template <auto kKernel>
dg4_status dg4i_resident_blocks(int threads, int* out) {
    static std::atomic<int> known[64];         // 0 = not asked yet
    int dev = 0;
    DG4_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) DG4_FAIL(DG4_ERR_UNSUPPORTED, "device ordinal %d is out of range", dev);
    int blocks = known[dev].load(std::memory_order_relaxed);
    if (blocks == 0) {
        int sms = 0, per_sm = 0;
        DG4_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        DG4_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kKernel, threads, 0));
        blocks = sms * (per_sm > 0 ? per_sm : 1);
        known[dev].store(blocks, std::memory_order_relaxed);
    }
    *out = blocks;
    return DG4_OK;
}

// Launches a kernel.  `early`: it may begin while the kernel enqueued before it on the stream is still running, once all of
// that one's CTAs have called let_next_begin() (a kernel that does not call it lets the next begin when it has ended).  All
// its threads call wait_for_previous() before they touch global memory, which leaves the launch and the set-up to overlap: a
// few us of a small call.  A kernel that needs nothing of the one before may call it later, but before it ends, so that the
// stream's order holds for whatever comes behind; that one lets it begin behind its own wait.
template <class... Params, class... Args>
dg4_status dg4i_launch_clusters(void (*kernel)(Params...), dim3 grid, int cluster, int threads, int smem, cudaStream_t st, bool early, Args&&... args) {
    cudaLaunchConfig_t c = {};
    c.gridDim = grid; c.blockDim = dim3((unsigned)threads); c.dynamicSmemBytes = (size_t)smem; c.stream = st;
    cudaLaunchAttribute at[2] = {};
    c.attrs = at;
    if (early) {
        at[c.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[c.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        at[c.numAttrs].id = cudaLaunchAttributeClusterDimension;
        at[c.numAttrs].val.clusterDim.x = (unsigned)cluster;
        at[c.numAttrs].val.clusterDim.y = at[c.numAttrs].val.clusterDim.z = 1;
        ++c.numAttrs;
    }
    DG4_CUDA_TRY(cudaLaunchKernelEx(&c, kernel, std::forward<Args>(args)...));
    dg4i_count_launch();
    return DG4_OK;
}
template <class... Params, class... Args>
dg4_status dg4i_launch(void (*kernel)(Params...), dim3 grid, int threads, int smem, cudaStream_t st, bool early, Args&&... args) {
    return dg4i_launch_clusters(kernel, grid, 1, threads, smem, st, early, std::forward<Args>(args)...);
}
// How many clusters of a size the current device holds at once, asked once per kernel, size (a power of two up to 8) and device.
template <auto kKernel>
dg4_status dg4i_resident_clusters(int cluster, int threads, int smem, int* out) {
    static std::atomic<int> known[64][4];
    int dev = 0, size = 0;
    while ((2 << size) <= cluster) ++size;
    DG4_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64 || size > 3) DG4_FAIL(DG4_ERR_UNSUPPORTED, "device ordinal %d or cluster size %d is out of range", dev, cluster);
    int n = known[dev][size].load(std::memory_order_relaxed) - 1;
    if (n < 0) {
        cudaLaunchConfig_t c = {};
        c.gridDim = dim3((unsigned)cluster); c.blockDim = dim3((unsigned)threads); c.dynamicSmemBytes = (size_t)smem;
        cudaLaunchAttribute at = {};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = (unsigned)cluster; at.val.clusterDim.y = at.val.clusterDim.z = 1;
        c.attrs = &at; c.numAttrs = 1;
        n = 0;
        DG4_CUDA_TRY(cudaOccupancyMaxActiveClusters(&n, kKernel, &c));
        known[dev][size].store(n + 1, std::memory_order_relaxed);
    }
    *out = n;
    return DG4_OK;
}
#ifdef __CUDACC__
__device__ __forceinline__ void let_next_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
#endif
