// What the kernels of the 8-bit paged KV cache share: the cache as kernels see it, host-side argument checks and the
// device helpers around E4M3 codes with power-of-two scales.
#pragma once
#include <cuda_fp16.h>

#include "pd_common.cuh"
#include "pd_ptx.cuh"

namespace pd {

// Device view of a pd_paged_kv_cache.
struct PagedCache {
  uint8_t* k;              // [n_pages, Hkv, page_len, hd] E4M3 codes
  uint8_t* v;
  float* k_scale;          // [n_pages, Hkv]
  float* v_scale;
  const int32_t* table;    // [n_seqs, table_ld]
  int n_pages, log2_page, table_ld;
};

// Checks the description (not the device contents) and fills the device view.
inline pd_status paged_cache_view(const pd_paged_kv_cache* c, PagedCache* out) {
  if (!c || c->struct_size != sizeof(pd_paged_kv_cache)) return PD_ERR_INVALID_ARG;
  if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales || !c->page_table) return PD_ERR_INVALID_ARG;
  if (c->n_pages <= 0 || c->n_seqs <= 0 || c->table_ld <= 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k_codes) | reinterpret_cast<uintptr_t>(c->v_codes)) & 15u) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k_scales) | reinterpret_cast<uintptr_t>(c->v_scales) |
       reinterpret_cast<uintptr_t>(c->page_table)) & 3u)
    return PD_ERR_INVALID_ARG;
  int l2 = 0;
  switch (c->page_len) {
    case 16: l2 = 4; break;
    case 32: l2 = 5; break;
    case 64: l2 = 6; break;
    case 128: l2 = 7; break;
    default: return PD_ERR_UNSUPPORTED_SHAPE;
  }
  // positions are 32-bit: table_ld pages must not reach past them
  if (c->table_ld > (0x7fffffff >> l2)) return PD_ERR_UNSUPPORTED_SHAPE;
  out->k = static_cast<uint8_t*>(c->k_codes); out->v = static_cast<uint8_t*>(c->v_codes);
  out->k_scale = c->k_scales; out->v_scale = c->v_scales; out->table = c->page_table;
  out->n_pages = c->n_pages; out->log2_page = l2; out->table_ld = c->table_ld;
  return PD_OK;
}

// The head shape part of a layer configuration (d_model and d_ff play no role here).
inline pd_status check_paged_heads(const pd_layer_cfg* cfg) {
  if (!cfg || cfg->struct_size != sizeof(pd_layer_cfg)) return PD_ERR_INVALID_ARG;
  if (cfg->n_q_heads <= 0 || cfg->n_kv_heads <= 0) return PD_ERR_INVALID_ARG;
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return PD_ERR_UNSUPPORTED_SHAPE;
  if (cfg->n_q_heads % cfg->n_kv_heads != 0 || cfg->n_q_heads / cfg->n_kv_heads > 16) return PD_ERR_UNSUPPORTED_SHAPE;
  if (cfg->n_kv_heads > 4096) return PD_ERR_UNSUPPORTED_SHAPE;
  return PD_OK;
}

// Page scales are powers of two 2^e with e in [-117, 120].  The lower bound keeps every product code * scale a normal
// number (the smallest code is 2^-9), the upper one is what the largest finite float needs.
constexpr int kPageScaleMinExp = -117;

// The smallest admissible power of two s with amax <= 448 s (amax finite, >= 0).
__device__ __forceinline__ float page_scale(float amax) {
  // 448 = 1.75 * 2^8: the exponent is that of amax minus 8, one more if the mantissa lies above 1.75
  const int e = static_cast<int>((__float_as_uint(amax) + 0x1fffffu) >> 23) - 127 - 8;
  return __uint_as_float(static_cast<uint32_t>(max(e, kPageScaleMinExp) + 127) << 23);
}
// 1 / s of a power of two s = 2^e, |e| <= 126: the exponent field mirrored.
__device__ __forceinline__ float pow2_inverse(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// Two E4M3 codes (bits 0-15) -> two halves, exactly.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t c) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(c));
  return r;
}

}  // namespace pd
