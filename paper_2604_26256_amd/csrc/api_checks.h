// Argument checks and sizes that the C-ABI front ends share.  Host only.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dora_internal.h"

namespace dora {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline int compute_units() {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      cus <= 0) {
    (void)hipGetLastError();  // no device here: size for a 256-CU part
    cus = 256;
  }
  return cus;
}

// The checks that the attention calls around the cache share, on a valid descriptor.
inline dora_status check_attn(const dora_decode_desc& d, const void* q, const void* k_pages,
                              const void* v_pages, const int32_t* block_table,
                              const int32_t* seq_lens, const int32_t* version_ids, const void* out,
                              const void* workspace) {
  if (!q || !k_pages || !v_pages || !block_table || !seq_lens || !out || !workspace)
    return DORA_ERR_INVALID_ARG;
  if (d.kv_dtype == DORA_KV_FP8_E4M3 && (!d.k_scales || !d.v_scales)) return DORA_ERR_INVALID_ARG;
  if ((d.flags & DORA_FLAG_VALIDATE) && !version_ids && d.page_owner) return DORA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) ||
      !aligned16(workspace))
    return DORA_ERR_INVALID_ARG;
  return DORA_OK;
}

inline float scale_log2_of(const dora_decode_desc& d) {
  const float scale = d.sm_scale > 0.f ? d.sm_scale : 1.0f / sqrtf((float)d.head_dim);
  // (the kernels take it for positive)
  return fmaxf(scale * 1.4426950408889634f, 1e-30f);
}

inline int64_t page_bytes_of(const dora_decode_desc& d) {
  return kv_page_bytes(d.kv_dtype, d.num_kv_heads, d.page_size, d.head_dim);
}

}  // namespace dora
