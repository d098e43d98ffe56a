// What the operators between pruning and the answer share (page tables, norms and rotation, the 8-bit cache and the
// attention that reads it): the launch that may begin while the kernel ahead drains, the cache as the kernels see it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/rtprune.h"
#include "common.cuh"
#include "ptx.cuh"

namespace rtp {

// Launch that may begin while the kernel ahead of it in the stream drains (each kernel waits for that one's end itself,
// before it reads or writes anything).
template <typename... KArgs, typename... Args>
inline cudaError_t launch_chained(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// SMs of the current device, asked for once (0: no answer).
inline int device_sms()
{
    static std::atomic<int> known[64];
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev < 64 && (sms = known[dev].load(std::memory_order_relaxed))) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

// Pages [num_pages][kv_heads][page_size][head_dim] of codes, scales [num_pages][kv_heads].
struct CacheView {
    int8_t *k, *v;
    float *k_scale, *v_scale;
    int32_t num_pages, kv_heads, dim;
    int32_t page_size, page_shift;      // page_size = 1 << page_shift
};

// The caller's cache, checked; false = not one the kernels take (`status` says why).
inline bool cache_view(const rtprune_cache_t *c, CacheView &v, rtprune_status_t &status)
{
    status = RTPRUNE_ERR_INVALID_ARG;
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || c->num_pages <= 0 || c->kv_heads <= 0 || c->head_dim <= 0) return false;
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15u || ((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3u) return false;
    status = RTPRUNE_ERR_UNSUPPORTED;
    int shift = 4;
    while (shift < 7 && (1 << shift) != c->page_size) ++shift;
    if ((1 << shift) != c->page_size) return false;                              // 16, 32, 64, 128
    // slots are 32-bit, and so are the rows of codes
    if (c->kv_heads > 1024 || c->num_pages > INT32_MAX / c->page_size / c->kv_heads) return false;
    if (c->head_dim != 64 && c->head_dim != 128) return false;
    v = {c->k, c->v, c->k_scale, c->v_scale, (int32_t)c->num_pages, c->kv_heads, c->head_dim, c->page_size, shift};
    status = RTPRUNE_OK;
    return true;
}

}  // namespace rtp
