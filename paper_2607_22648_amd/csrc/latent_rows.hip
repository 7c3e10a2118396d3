// New tokens' rows into the pages of a latent cache, and rows of pages back out: a copy, 16 bytes a
// lane, consecutive lanes along a row of 72 (40) such pieces.
//
// Bound by memory: 2 bytes read and 2 written a value. 16,384 tokens of 576 values (38 MB) take 8.7 us into pages and
// 6.4 out of them, where the 256 MB cache still holds them (a copy from memory takes 6.6); 64 tokens 2.3.
#include <hip/hip_runtime.h>

#include "latent.hpp"

namespace ptsd {
namespace {

typedef unsigned int v4u __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// kRead: pages to rows, else rows to pages.
template <bool kRead>
__global__ __launch_bounds__(kThreads) void k_latent_rows(LatentPlane kv, uint8_t* latent, int64_t latent_stride,
                                                          uint8_t* rope, int64_t rope_stride, const int64_t* slots,
                                                          uint32_t pieces, PageDiv line) {
    const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
    if (at >= pieces) return;
    const uint32_t t = div_page(at, line), c = at - t * line.page, split = (uint32_t)kv.latent / 8;
    const int64_t slot = slots[t];
    const bool there = slot >= 0 && slot < kv.blocks * kv.div.page;
    // a token's values and its part that heads share, strides in elements
    v4u* const outside = (v4u*)(c < split ? latent + ((int64_t)t * latent_stride + c * 8) * 2
                                          : rope + ((int64_t)t * rope_stride + (c - split) * 8) * 2);
    v4u* const page = (v4u*)kv.rows + ((there ? slot : 0) * kv.line + c);
    if constexpr (kRead) {
        const v4u zero = {0u, 0u, 0u, 0u};
        *outside = there ? *page : zero;
    } else if (there) {
        *page = __builtin_nontemporal_load(outside);  // read once, as in append.hip
    }
}

template <bool kRead>
hipError_t launch_rows(const LatentPlane& kv, const void* latent, int64_t latent_stride, const void* rope,
                       int64_t rope_stride, const int64_t* slots, int64_t n, hipStream_t s) {
    const uint32_t pieces = (uint32_t)(n * kv.line);
    hipLaunchKernelGGL((k_latent_rows<kRead>), dim3((pieces + kThreads - 1) / kThreads), dim3(kThreads), 0, s, kv,
                       (uint8_t*)latent, latent_stride, (uint8_t*)rope, rope_stride, slots, pieces,
                       page_div((int)kv.line));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_latent_append(const LatentPlane& kv, const void* latent, int64_t latent_stride, const void* rope,
                                int64_t rope_stride, const int64_t* slots, int64_t n, hipStream_t s) {
    return launch_rows<false>(kv, latent, latent_stride, rope, rope_stride, slots, n, s);
}

hipError_t launch_latent_read(const LatentPlane& kv, void* latent, int64_t latent_stride, void* rope,
                              int64_t rope_stride, const int64_t* slots, int64_t n, hipStream_t s) {
    return launch_rows<true>(kv, latent, latent_stride, rope, rope_stride, slots, n, s);
}

}  // namespace ptsd
