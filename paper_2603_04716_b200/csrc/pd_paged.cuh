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

// Blocks of `block_tokens` consecutive tokens of one request: request r owns the slots from first_slot(cu[r], r) on, as many as
// it has such blocks, or one more (a single request exactly as many), so the host needs only the number of tokens.
__host__ __device__ __forceinline__ int first_slot(int cu, int r, int block_tokens) {
  return static_cast<int>((static_cast<uint32_t>(cu) + static_cast<uint32_t>(r) * (block_tokens - 1)) / block_tokens);
}
struct TokenBlock {
  int req, start, len, pre;  // request, its first row, its rows, tokens cached before them
  int t0;                    // the block's first token within the request; not below len: no block in this slot
};
// The block of a slot.  All lanes of a warp search together, 32 candidates at a time; for up to 32 requests the warp has
// every request's numbers after one load.
__device__ __forceinline__ TokenBlock find_block(const int32_t* cu_seqlens, const int32_t* prefix, int n_req, int n_tokens, int slot,
                                                 int block_tokens) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = n_req;  // the request lies in lo .. lo + n - 1
  while (n > 32) {
    const int stride = (n + 31) / 32, r = lo + lane * stride;
    const bool at_or_before = lane * stride < n && first_slot(cu_seqlens[r], r, block_tokens) <= slot;
    const int k = 31 - __clz(__ballot_sync(0xffffffffu, at_or_before) | 1u);
    lo += k * stride;
    n = min(stride, n - k * stride);
  }
  const int r = lo + min(lane, n - 1);
  const int c0 = cu_seqlens[r], c1 = cu_seqlens[r + 1], pre = prefix ? prefix[r] : 0;
  const int k = 31 - __clz(__ballot_sync(0xffffffffu, lane < n && first_slot(c0, r, block_tokens) <= slot) | 1u);
  TokenBlock b;
  b.req = lo + k;
  b.start = __shfl_sync(0xffffffffu, c0, k);
  b.len = min(__shfl_sync(0xffffffffu, c1, k), n_tokens) - b.start;
  b.pre = __shfl_sync(0xffffffffu, pre, k);
  b.t0 = (slot - first_slot(b.start, b.req, block_tokens)) * block_tokens;
  if (b.t0 < 0 || b.pre < 0) b.t0 = 0x7fffffff;  // (never with consistent inputs)
  return b;
}

// Attention of ragged runs of fresh rows over the cache, as the kernels behind pd_paged_prefill_attention take it.
struct PagedRuns {
  const bf16* q;              // [T, ldq]
  bf16* o;                    // [T, Hq*hd]
  const int32_t* cu_seqlens;  // device [n_req + 1]
  const int32_t* prefix;      // device [n_req] or NULL
  int* err_word;
  PagedCache c;
  int ldq, n_req, n_tokens, n_q_heads, n_kv_heads, head_dim;
  int max_kv;                 // longest prefix + run
  long long tile_blocks;      // blocks of 256 (token, head) rows over all requests and one KV head
};
// Partial results of rows whose key range is cut: outputs [n_splits, rows, hd] (relative to m) and (m, l) [n_splits, rows], row =
// token * Hq + head, m in log2 units.  A part without keys has m = -inf, l = 0 and need not have stored outputs.
struct PagedParts {
  float* o;
  float2* ml;
};
inline size_t paged_parts_ml_offset(size_t part_rows, int head_dim) { return align_up(part_rows * head_dim * sizeof(float), 256); }
inline size_t paged_parts_bytes(size_t part_rows, int head_dim) {
  return paged_parts_ml_offset(part_rows, head_dim) + align_up(part_rows * sizeof(float2), 256);
}
pd_status launch_paged_join(const PagedParts& parts, bf16* o, long long rows, int n_splits, int head_dim, cudaStream_t s);
// The streaming kernel of decode attention over blocks of a few tokens, and how many (token, head) rows a block has.
int paged_rows_block(int group, int longest_run);
pd_status launch_paged_rows(const PagedRuns& r, int longest_run, const PagedParts& parts, cudaStream_t s);
size_t paged_rows_part_rows();  // rows of partial results that the launch may need
// The tensor-memory kernel.  The rows of the first split_slots blocks of tokens (all of them, or as many as are left when the
// SMs have had their last full turn) have their key range cut into n_splits parts.
struct PagedTilesPlan {
  int split_slots, n_splits;
  long long part_rows;  // (token, head) rows of those blocks, the first of the call
};
PagedTilesPlan paged_tiles_plan(const PagedRuns& r, const int32_t* cu_host, const int32_t* prefix_host);
pd_status launch_paged_tiles(const PagedRuns& r, const PagedTilesPlan& plan, const PagedParts& parts, cudaStream_t s);
size_t paged_tiles_part_rows();

// A key that some row of a block does not see meets that row with a weight of 0, and 0 * NaN is NaN: V rows of such keys enter
// the products without their NaN codes, and the rows that do see the key are given their NaN at the end.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t codes) { return ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t drop_nans(uint32_t codes, bool& seen) {
  const uint32_t m = nan_bytes(codes);
  seen |= m != 0;
  return codes & ~((m >> 7) * 0xffu);
}
// V row of a key of the sequence with page table row `table`; NULL: its page number lies outside the pool.
__device__ __forceinline__ const uint8_t* v_row(const PagedCache& c, const int32_t* table, int n_kv_heads, int kvh, int head_dim, int key) {
  const int id = table[key >> c.log2_page];
  if (static_cast<unsigned>(id) >= static_cast<unsigned>(c.n_pages)) return nullptr;
  return c.v + (((static_cast<size_t>(id) * n_kv_heads + kvh) << c.log2_page) + (key & ((1 << c.log2_page) - 1))) * head_dim;
}

// Two E4M3 codes (bits 0-15) -> two halves, exactly.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t c) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(c));
  return r;
}

}  // namespace pd
