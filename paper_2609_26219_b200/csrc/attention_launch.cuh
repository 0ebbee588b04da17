// What the attention's launch functions share.
#pragma once

#include <atomic>

#include "attention.cuh"

namespace patchkv {

// Opts a kernel into `bytes` of dynamic shared memory, once per device (a bit each; the attribute is per device and sticks).
inline cudaError_t allow_smem(const void* kernel, int bytes, std::atomic<uint64_t>* done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (done->load(std::memory_order_acquire) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done->fetch_or(bit, std::memory_order_release);
    return e;
}

}  // namespace patchkv
