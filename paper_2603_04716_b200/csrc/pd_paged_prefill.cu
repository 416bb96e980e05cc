// pd_paged_prefill_attention: which kernel attends the fresh rows of a call over the 8-bit paged KV cache.
#include <cmath>
#include <cstdlib>
#include <initializer_list>

#include "pd_paged.cuh"

namespace pd {
namespace {

// ------------------------------------------------------------------------------------ pages -> contiguous bf16
struct GatherArgs {
  bf16* k;                    // [n_req, Hkv, len_cap, hd]
  bf16* v;
  const int32_t* cu_seqlens;  // [n_req + 1]
  const int32_t* prefix;      // [n_req] or NULL
  int* err_word;
  PagedCache c;
  int n_kv_heads, head_dim, len_cap;
};

__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t pair, float s) {
  const uint32_t h = e4m3x2_to_f16x2(static_cast<uint16_t>(pair));
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return ptx::pack_bf16(f.x * s, f.y * s);  // exact: four significant bits times a power of two
}

// Block (page of the sequence, KV head, request): its K and V rows that hold tokens.
__global__ void __launch_bounds__(256) gather_pages_kernel(const GatherArgs a) {
  const int pi = blockIdx.x, kvh = blockIdx.y, r = blockIdx.z;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int n_new = a.cu_seqlens[r + 1] - a.cu_seqlens[r];
  if (n_new <= 0) return;
  const int total = min((a.prefix ? a.prefix[r] : 0) + n_new, a.len_cap);
  const int first = pi << a.c.log2_page;
  const int rows = min(total - first, 1 << a.c.log2_page);
  if (rows <= 0) return;
  const int id = a.c.table[static_cast<size_t>(r) * a.c.table_ld + pi];
  const bool ok = static_cast<unsigned>(id) < static_cast<unsigned>(a.c.n_pages);
  if (!ok && threadIdx.x == 0 && a.err_word) atomicExch(a.err_word, 2);
  const size_t ph = static_cast<size_t>(ok ? id : 0) * a.n_kv_heads + kvh;
  const uint4* src_k = reinterpret_cast<const uint4*>(a.c.k + (ph << a.c.log2_page) * a.head_dim);
  const uint4* src_v = reinterpret_cast<const uint4*>(a.c.v + (ph << a.c.log2_page) * a.head_dim);
  const float ks = ok ? a.c.k_scale[ph] : 0.f, vs = ok ? a.c.v_scale[ph] : 0.f;
  const size_t dst0 = ((static_cast<size_t>(r) * a.n_kv_heads + kvh) * a.len_cap + first) * a.head_dim;
  uint4* dst_k = reinterpret_cast<uint4*>(a.k + dst0);
  uint4* dst_v = reinterpret_cast<uint4*>(a.v + dst0);
  const int chunks = rows * a.head_dim / 16;
  for (int i = threadIdx.x; i < chunks; i += blockDim.x) {
    uint4 wk = make_uint4(0u, 0u, 0u, 0u), wv = wk;
    if (ok) { wk = src_k[i]; wv = src_v[i]; }
    dst_k[2 * i] = make_uint4(codes_to_bf16(wk.x, ks), codes_to_bf16(wk.x >> 16, ks), codes_to_bf16(wk.y, ks), codes_to_bf16(wk.y >> 16, ks));
    dst_k[2 * i + 1] = make_uint4(codes_to_bf16(wk.z, ks), codes_to_bf16(wk.z >> 16, ks), codes_to_bf16(wk.w, ks), codes_to_bf16(wk.w >> 16, ks));
    dst_v[2 * i] = make_uint4(codes_to_bf16(wv.x, vs), codes_to_bf16(wv.x >> 16, vs), codes_to_bf16(wv.y, vs), codes_to_bf16(wv.y >> 16, vs));
    dst_v[2 * i + 1] = make_uint4(codes_to_bf16(wv.z, vs), codes_to_bf16(wv.z >> 16, vs), codes_to_bf16(wv.w, vs), codes_to_bf16(wv.w >> 16, vs));
  }
}

size_t gather_half(const pd_layer_cfg* cfg, int n_req, int max_kv_len) {
  return align_up(static_cast<size_t>(n_req) * cfg->n_kv_heads * max_kv_len * cfg->head_dim * sizeof(bf16), 256);
}

// Which kernel attends the rows of a call.  All three give the same result (within the rounding of p and of the result).
//   ROWS   the streaming kernel of decode over blocks of 16 (token, head) rows: each block reads its keys again
//   TILES  tensor-memory tiles of 128 (token, head) rows over codes as they are
//   FULL   the pages decoded to a contiguous bf16 copy, then the prefill kernel, whose tiles are 128 tokens of one head
// Estimated times in microseconds, fitted to measurements (32 query and 8 KV heads of 128, one to 37 requests, 1 to 8192 fresh
// tokens, up to 16000 cached): the fixed part, the steps of the busiest SM, the parts of key ranges that are written and
// joined, the decoded copy.  Heads of 64 take about 0.7 of a step.  Examples, measured (ROWS / TILES / FULL): 1 x 8 tokens over
// 2000 keys 11 / 15 / 44, 1 x 128 over 2000 38 / 29 / 49, 8 x 64 over 4096 220 / 87 / 188, 1 x 512 over 16000 751 / 223 / 303,
// a prompt of 4096 tokens 973 / 209 / 167, 4 x 500 over 5000 at a group of 8 2042 / 497 / 420, 32 x 4 over 2000 39 / 92 / 315.
enum class Path { ROWS, TILES, FULL };

Path choose_path(const PagedRuns& r, const int32_t* cu, const int32_t* prefix, int longest) {
  const int group = r.n_q_heads / r.n_kv_heads;
  const int row_tokens = paged_rows_block(group, longest), tile_tokens = 2 * (128 / group), full_tokens = 256;
  // steps (16 keys of a row block; 128 keys of a tile block or of a block of tokens and one head), blocks
  double rows_steps = 0, tile_steps = 0, full_steps = 0, tile_items = 0, full_items = 0, keys = 0;
  auto steps = [](double len, double pre, double block, double step) {  // over the blocks of a run: the mean of first and last
    const double blocks = std::ceil(len / block);
    const double first = std::ceil((pre + (len < block ? len : block)) / step), last = std::ceil((pre + len) / step);
    return blocks * (first + last) / 2;
  };
  for (int i = 0; i < r.n_req; ++i) {
    const double len = cu[i + 1] - cu[i], pre = prefix ? prefix[i] : 0;
    if (len == 0) continue;
    rows_steps += r.n_kv_heads * steps(len, pre, row_tokens, 16);
    tile_steps += r.n_kv_heads * steps(len, pre, tile_tokens, 128);
    full_steps += r.n_q_heads * steps(len, pre, full_tokens, 128);
    tile_items += r.n_kv_heads * std::ceil(len / tile_tokens);
    full_items += r.n_q_heads * std::ceil(len / full_tokens);
    keys += pre + len;
  }
  const double sms = 148, longest_tiles = std::ceil(r.max_kv / 128.0), hd = r.head_dim == 128 ? 1.0 : 0.7;
  const double splits = paged_tiles_splits(static_cast<long long>(tile_items), r.max_kv);
  const double t_rows = 8 + hd * (1.4e-3 * std::fmin(rows_steps, 8000) + 0.9e-3 * std::fmax(rows_steps - 8000, 0));
  const double tile_step = 1.0 * longest * group <= 128 ? 2.2 : 3.2;  // one row tile of a block in use, or both
  const double t_tiles = 13 + hd * tile_step * std::fmax(tile_steps / sms, std::ceil(longest_tiles / splits)) +
                         4 * tile_items * splits / sms + (splits > 1 ? 8 * splits * r.n_tokens * r.n_q_heads / paged_tiles_part_rows() : 0);
  const double t_full = 21 + hd * 2.35 * std::fmax(full_steps / sms, longest_tiles) + 2.3 * full_items / sms +
                        1.1e-6 * keys * r.n_kv_heads * r.head_dim;
  // what a kernel can address: blocks along one grid axis, 32-bit numbers of K rows, 32-bit numbers of rows of the copy
  const bool rows_fit = first_slot(r.n_tokens, r.n_req, row_tokens) <= 65535;
  const bool tiles_fit = (static_cast<long long>(r.c.n_pages) * r.n_kv_heads << r.c.log2_page) <= 0x7fffffffll;
  // PD_PAGED_PREFILL=0, 1, 2 forces a kernel where it fits (for A/B timing and tests)
  static const int forced = [] {
    const char* e = std::getenv("PD_PAGED_PREFILL");
    return e ? std::atoi(e) : -1;
  }();
  if (forced == 0 && rows_fit) return Path::ROWS;
  if (forced == 1 && tiles_fit) return Path::TILES;
  if (forced == 2) return Path::FULL;
  if (rows_fit && t_rows <= t_full && (t_rows <= t_tiles || !tiles_fit)) return Path::ROWS;
  return tiles_fit && t_tiles <= t_full ? Path::TILES : Path::FULL;
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_paged_prefill_attention_workspace_bytes(const pd_layer_cfg* cfg, int32_t n_req, int32_t max_kv_len,
                                                                size_t* out_bytes) {
  using namespace pd;
  PD_TRY(check_paged_heads(cfg));
  if (!out_bytes || n_req < 0 || max_kv_len < 0) return PD_ERR_INVALID_ARG;
  // the largest of what the kernels need
  size_t need = 2 * gather_half(cfg, n_req, max_kv_len);
  for (const size_t part_rows : {paged_rows_part_rows(), paged_tiles_part_rows()}) {
    const size_t bytes = paged_parts_bytes(part_rows, cfg->head_dim);
    if (bytes > need) need = bytes;
  }
  *out_bytes = n_req && max_kv_len ? need : 0;
  return PD_OK;
}

extern "C" pd_status pd_paged_prefill_attention(const pd_layer_cfg* cfg, const void* q, int32_t ldq, void* out,
                                                const int32_t* cu_dev, const int32_t* cu_host, int32_t n_req,
                                                const int32_t* prefix_dev, const int32_t* prefix_host,
                                                const pd_paged_kv_cache* cache, void* workspace, size_t workspace_bytes,
                                                int32_t* err_word, void* stream) {
  using namespace pd;
  PD_TRY(check_paged_heads(cfg));
  PagedRuns r{};
  PD_TRY(paged_cache_view(cache, &r.c));
  if (!cu_host || n_req < 0 || n_req > 4095 || n_req > cache->n_seqs || (prefix_dev == nullptr) != (prefix_host == nullptr))
    return PD_ERR_INVALID_ARG;
  if (cu_host[0] != 0) return PD_ERR_INVALID_ARG;
  const int cap = cache->table_ld << r.c.log2_page;
  const int group = cfg->n_q_heads / cfg->n_kv_heads;
  int longest = 0;
  for (int i = 0; i < n_req; ++i) {
    const long long len = 1ll * cu_host[i + 1] - cu_host[i];
    const int pre = prefix_host ? prefix_host[i] : 0;
    if (len < 0 || pre < 0 || pre + len > cap) return PD_ERR_INVALID_ARG;
    if (len > longest) longest = static_cast<int>(len);
    if (len > 0 && pre + len > r.max_kv) r.max_kv = static_cast<int>(pre + len);
  }
  r.n_tokens = cu_host[n_req];
  if (r.n_tokens == 0) return PD_OK;
  if (!q || !out || !cu_dev || ldq < cfg->n_q_heads * cfg->head_dim || ldq % 8 != 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) & 15u) || (reinterpret_cast<uintptr_t>(out) & 31u)) return PD_ERR_INVALID_ARG;
  if (r.max_kv > 0x7fffffff - 1024) return PD_ERR_UNSUPPORTED_SHAPE;
  size_t need = 0;
  PD_TRY(pd_paged_prefill_attention_workspace_bytes(cfg, n_req, r.max_kv, &need));
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PD_ERR_INVALID_ARG;
  if (workspace_bytes < need) return PD_ERR_WORKSPACE_TOO_SMALL;
  r.q = static_cast<const bf16*>(q); r.o = static_cast<bf16*>(out); r.cu_seqlens = cu_dev; r.prefix = prefix_dev; r.err_word = err_word;
  r.ldq = ldq; r.n_req = n_req; r.n_q_heads = cfg->n_q_heads; r.n_kv_heads = cfg->n_kv_heads; r.head_dim = cfg->head_dim;

  const int tile_tokens = 2 * (128 / group);
  for (int i = 0; i < n_req; ++i) r.tile_blocks += (cu_host[i + 1] - cu_host[i] + tile_tokens - 1) / tile_tokens;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_ATTN_PREFILL, st);
  const Path path = choose_path(r, cu_host, prefix_host, longest);
  if (path != Path::FULL) {
    const size_t part_rows = path == Path::ROWS ? paged_rows_part_rows() : paged_tiles_part_rows();
    PagedParts parts;
    parts.o = static_cast<float*>(workspace);
    parts.ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + paged_parts_ml_offset(part_rows, cfg->head_dim));
    return path == Path::ROWS ? launch_paged_rows(r, longest, parts, st) : launch_paged_tiles(r, parts, st);
  }
  // 32-bit row numbers of the decoded copy
  if (1ll * n_req * cfg->n_kv_heads * r.max_kv > 0x7fffffffll - 256) return PD_ERR_UNSUPPORTED_SHAPE;
  GatherArgs ga{};
  ga.c = r.c;
  ga.k = static_cast<bf16*>(workspace);
  ga.v = reinterpret_cast<bf16*>(static_cast<uint8_t*>(workspace) + gather_half(cfg, n_req, r.max_kv));
  ga.cu_seqlens = cu_dev; ga.prefix = prefix_dev; ga.err_word = err_word;
  ga.n_kv_heads = cfg->n_kv_heads; ga.head_dim = cfg->head_dim; ga.len_cap = r.max_kv;
  const int pages = (r.max_kv + (1 << ga.c.log2_page) - 1) >> ga.c.log2_page;
  PD_CUDA_TRY(launch_pdl(gather_pages_kernel, dim3(pages, cfg->n_kv_heads, n_req), dim3(256), 0, st, ga));
  count_launch();
  PrefillAttnArgs a{};
  a.q = r.q; a.ldq = ldq;
  a.k_cache = ga.k; a.v_cache = ga.v;
  a.o = r.o; a.cu_seqlens = cu_dev; a.prefix = prefix_dev;
  a.n_req = n_req; a.n_tokens = r.n_tokens; a.max_len = longest;
  a.n_q_heads = cfg->n_q_heads; a.n_kv_heads = cfg->n_kv_heads; a.head_dim = cfg->head_dim;
  a.len_cap = r.max_kv; a.batch_cap = n_req;
  return launch_prefill_attention_tc(a, err_word, st);
}
