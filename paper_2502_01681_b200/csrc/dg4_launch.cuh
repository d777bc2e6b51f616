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
dg4_status dg4i_launch(void (*kernel)(Params...), dim3 grid, int threads, int smem, cudaStream_t st, bool early, Args&&... args) {
    cudaLaunchConfig_t c = {};
    c.gridDim = grid; c.blockDim = dim3((unsigned)threads); c.dynamicSmemBytes = (size_t)smem; c.stream = st;
    cudaLaunchAttribute at = {};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &at; c.numAttrs = early ? 1 : 0;
    DG4_CUDA_TRY(cudaLaunchKernelEx(&c, kernel, std::forward<Args>(args)...));
    dg4i_count_launch();
    return DG4_OK;
}
#ifdef __CUDACC__
__device__ __forceinline__ void let_next_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
#endif
