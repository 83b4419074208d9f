// What the host sides of the serving operators share: device properties, checks of arguments, launch accounting.
#pragma once

#include <atomic>
#include <cmath>

#include "mcsd_cache.cuh"
#include "mcsd_host.h"

namespace mcsd {
namespace {

constexpr int kDevices = 64;                        // whose properties are kept

// Multiprocessors of the current device, 0 if there is none (asked once per device).
int sm_count()
{
    static std::atomic<int> known[kDevices];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < kDevices && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < kDevices) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Shared memory beyond the default for a kernel, asked for when a device needs more than it has. (Nothing here or elsewhere
// on the way of a call allocates or takes a lock: no exception reaches the C caller.)
template <auto Kernel>
bool allow_smem(int bytes)
{
    static std::atomic<int> known[kDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const bool keep = dev >= 0 && dev < kDevices;
    if (keep && known[dev].load(std::memory_order_relaxed) >= bytes) return true;
    // (always the most that a CTA may have, so that calls at the same time cannot lower each other's)
    int most = 0;
    if (cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess) return false;
    cudaFuncAttributes fa = {};
    if (cudaFuncGetAttributes(&fa, Kernel) != cudaSuccess) return false;
    most -= static_cast<int>(fa.sharedSizeBytes);
    if (most < bytes || cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) return false;
    if (keep) known[dev].store(most, std::memory_order_relaxed);
    return true;
}

bool good_dtype(int dtype) { return dtype == MCSD_DTYPE_F32 || dtype == MCSD_DTYPE_BF16 || dtype == MCSD_DTYPE_F16; }
int elem_size(int dtype) { return dtype == MCSD_DTYPE_F32 ? 4 : 2; }
int shift_of(int page_size) { return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7; }
bool good_page_size(int ps) { return ps == 16 || ps == 32 || ps == 64 || ps == 128; }

// Whether device pointers lie on multiples of `bytes` (a null one does): the kernels would fault on others.
template <typename... Ptr>
bool on_multiples(unsigned bytes, const Ptr *...p)
{
    return ((reinterpret_cast<uintptr_t>(p) | ... | uintptr_t(0)) & (bytes - 1)) == 0;
}

int launched(int n)
{
    if (cudaGetLastError() != cudaSuccess) return MCSD_ERR_CUDA;
    set_last_launches(n);
    return MCSD_OK;
}

// |scale| in log2 units as a part below 1 and a power of two.
float scale_part(float scale, int32_t *power)
{
    int e = 0;
    const float part = std::frexp(std::fabs(scale) * 1.4426950408889634f, &e);
    *power = e;
    return part;
}

int check_cache(const mcsd_kv_cache *c)
{
    if (!c) return MCSD_ERR_NULL;
    if (c->n_pages < 0 || c->n_heads < 1) return MCSD_ERR_SHAPE;
    const size_t block = mcsd_kv_block_bytes(c->head_dim, c->page_size);
    if (block == 0) return MCSD_ERR_UNSUPPORTED;
    if (c->n_heads > 65535) return MCSD_ERR_UNSUPPORTED;
    if (c->page_stride % 16 != 0 || c->page_stride < static_cast<int64_t>(block) * c->n_heads) return MCSD_ERR_STRIDE;
    if (c->n_pages > 0 && !c->pages) return MCSD_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(c->pages) % 16 != 0) return MCSD_ERR_STRIDE;
    return MCSD_OK;
}

CacheParams cache_params(const mcsd_kv_cache *c)
{
    CacheParams p = {};
    p.pages = static_cast<unsigned char *>(c->pages);
    p.page_stride = c->page_stride;
    p.n_pages = c->n_pages;
    p.n_heads = c->n_heads;
    p.page_shift = shift_of(c->page_size);
    return p;
}

}  // namespace
}  // namespace mcsd
