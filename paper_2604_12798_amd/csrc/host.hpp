// What the C entry points of the translation units (vfa_fwd.hip, serving.hip, masked.hip) use on the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <atomic>

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Workgroups of 256 threads that one launch can have: of 2^32 work-items or more HIP runs a part, without an error
constexpr long long kMaxWorkgroups256 = (1LL << 24) - 1;

// Host-side caches.  Everything the library remembers between calls is a per-device fact that any thread would
// compute to the same value (a CU count, "this kernel's LDS limit has been raised", the address of the device
// array), held in atomics: two threads that race on a first call both do the lookup and store the same thing.
constexpr int kMaxDevices = 64;

int current_device() {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return -1;
    return dev;
}

// number of compute units of the current device (0 if the query fails), looked up once per device
int cu_count() {
    static std::atomic<int> cached[kMaxDevices];
    const int dev = current_device();
    if (dev < 0) return 0;
    int n = cached[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = -1;
        cached[dev].store(n, std::memory_order_relaxed);
    }
    return n > 0 ? n : 0;
}

}  // namespace
