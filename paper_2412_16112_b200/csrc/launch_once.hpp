// What a launch asks the runtime about a kernel and a device does not change: asked once a device, as each answer takes about as
// long as the launch itself.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

#include "clear_internal.hpp"

namespace clear {

constexpr int kMaxDevices = 64;  // devices beyond are asked every time

// The current device and its number of SMs.
inline int current_sms(int *device, int *n_sm)
{
    static std::atomic<int> known[kMaxDevices];
    CLEAR_CUDA_TRY(cudaGetDevice(device));
    *n_sm = *device < kMaxDevices ? known[*device].load(std::memory_order_relaxed) : 0;
    if (*n_sm > 0) return CLEAR_OK;
    CLEAR_CUDA_TRY(cudaDeviceGetAttribute(n_sm, cudaDevAttrMultiProcessorCount, *device));
    if (*device < kMaxDevices) known[*device].store(*n_sm, std::memory_order_relaxed);
    return CLEAR_OK;
}

// Lets a kernel have `most_smem` bytes of dynamic shared memory on the device; *per_sm: blocks of `threads` that an SM then holds.
// `known` belongs to that kernel alone.
template <typename K>
int kernel_once(std::atomic<int> (&known)[kMaxDevices], K kernel, int threads, int most_smem, int device, int *per_sm)
{
    *per_sm = device < kMaxDevices ? known[device].load(std::memory_order_acquire) : 0;
    if (*per_sm > 0) return CLEAR_OK;
    if (most_smem > 32 * 1024)
        CLEAR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem));
    CLEAR_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(per_sm, kernel, threads, most_smem));
    if (*per_sm < 1) return CLEAR_ERR_CUDA;
    if (device < kMaxDevices) known[device].store(*per_sm, std::memory_order_release);
    return CLEAR_OK;
}

}  // namespace clear
