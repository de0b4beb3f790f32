// What belongs to a device, kept for each device that the process uses.  Host code.
#pragma once
#include <cuda_runtime.h>

#include <atomic>

namespace xc {

constexpr int MAX_DEVICES = 64;

// The current device; -1 if there is none, or its number is past MAX_DEVICES.
inline int current_device() {
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < MAX_DEVICES ? dev : -1;
}

// Multiprocessors of the current device (1 where the device does not say).
inline int device_sms() {
    static std::atomic<int> sms[MAX_DEVICES];
    const int dev = current_device();
    if (dev < 0) return 1;
    int n = sms[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 1;
        sms[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// A kernel's leave to take more dynamic shared memory than a CTA has without asking holds on the
// device it was asked for.  `asked`: the devices where it was, one set for each kernel.
using DeviceSet = std::atomic<unsigned long long>;
template <typename Kernel> cudaError_t allow_smem(Kernel kernel, int bytes, DeviceSet &asked) {
    const int dev = current_device();
    if (dev < 0) return cudaErrorInvalidDevice;
    if (asked.load(std::memory_order_relaxed) >> dev & 1) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) asked.fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}

}  // namespace xc
