// What the C calls of the paged caches' operators check with (paged_api.hip, latent_api.hip,
// weight_api.hip): limits, alignment, refusals.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstdio>

#include "ptstore.h"

namespace ptsd {

int set_last_error(int code, const char* what);  // csrc/api.hip

constexpr int64_t kMaxEntries = 1ll << 29;  // (request, block) entries of a call
constexpr int64_t kMaxKeys = 1ll << 30;     // keys of a request: block-table columns * page size
constexpr int64_t kMaxItems = 1ll << 32;    // work-items of a launch, fewer than that

inline int refuse(const char* what) { return set_last_error(PTSTORE_ERR_INVALID, what); }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline int refuse_as(const char* call, const char* what) {
    char text[256];
    snprintf(text, sizeof text, "%s: %s", call, what);
    return refuse(text);
}

// Rows of a packed tensor: 16-byte aligned rows, so strides of 8 elements.
inline bool rows_ok(const void* p, int64_t token, int64_t head) {
    return p && aligned16(p) && token % 8 == 0 && head % 8 == 0;
}

// Compute units of the current device, asked for once a device.
inline int compute_units(const char* call, int* cus) {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return set_last_error(PTSTORE_ERR_HIP, call);
    if (dev >= 0 && dev < kDevices && (*cus = known[dev].load(std::memory_order_relaxed)) > 0) return PTSTORE_OK;
    if (hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess)
        return set_last_error(PTSTORE_ERR_HIP, call);
    if (dev >= 0 && dev < kDevices) known[dev].store(*cus, std::memory_order_relaxed);
    return PTSTORE_OK;
}

}  // namespace ptsd
