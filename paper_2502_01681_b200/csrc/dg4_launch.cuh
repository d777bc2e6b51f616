// How many blocks of a kernel the current device holds at once, asked of the runtime once per kernel and device (the
// question costs about 2 us, a quarter of a small call).
#pragma once

#include <atomic>

#include "dg4_internal.h"

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
