// What belongs to a device, kept for each device that the process uses.  Host code.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <mutex>

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

// The word in the current device's memory in which the operators' kernels set error bits; NULL if
// it cannot be made.  Made by the first call on a device, which must not be in a capture.
inline int *device_error_word() {
    static std::atomic<int *> words[MAX_DEVICES];
    static std::mutex making;
    const int dev = current_device();
    if (dev < 0) return nullptr;
    int *word = words[dev].load(std::memory_order_acquire);
    if (word != nullptr) return word;
    std::lock_guard<std::mutex> one(making);
    word = words[dev].load(std::memory_order_acquire);
    if (word != nullptr) return word;
    void *p = nullptr;
    if (cudaMalloc(&p, sizeof(int)) != cudaSuccess) return nullptr;
    if (cudaMemset(p, 0, sizeof(int)) != cudaSuccess) {
        cudaFree(p);
        return nullptr;
    }
    word = static_cast<int *>(p);
    words[dev].store(word, std::memory_order_release);
    return word;
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
