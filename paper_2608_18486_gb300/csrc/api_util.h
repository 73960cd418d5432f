// Helpers shared by the C-ABI entry points (wm_api.cu, longctx_api.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "wm.h"

namespace wm {

constexpr int kMaxDevices = 64;

// SMs of the current device (148 if it cannot be read), cached per device.
int sm_count();

inline bool is_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
inline int ilog2(int x) {
  int r = 0;
  while ((1 << r) < x) ++r;
  return r;
}
inline size_t elem_size(int dtype) { return dtype == WM_DT_F32 ? 4 : 2; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// The cache belongs to the config and its pools are usable.
inline wm_status check_cache(const wm_config& c, const wm_cache* cache) {
  if (!cache || !cache->k_pool || !cache->v_pool || cache->num_pages < 1) return WM_ERR_INVALID_ARG;
  if (cache->k != c.k || cache->Hkv != c.Hkv || cache->page_size != c.page_size ||
      cache->d != c.d || cache->dtype != c.dtype)
    return WM_ERR_INVALID_ARG;
  if (!aligned(cache->k_pool, 16) || !aligned(cache->v_pool, 16)) return WM_ERR_INVALID_ARG;
  return WM_OK;
}

}  // namespace wm
