// pd_paged_prefill_attention: which kernel attends the fresh rows of a call over the 8-bit paged KV cache.
#include <cmath>
#include <cstdlib>
#include <initializer_list>

#include "pd_paged.cuh"

namespace pd {
namespace {

// Which kernel attends the rows of a call.  Both give the same result (within the rounding of p and of the result).
//   ROWS   the streaming kernel of decode over blocks of 16 (token, head) rows: each block reads its keys again
//   TILES  tensor-memory tiles of 128 (token, head) rows
// Estimated times in microseconds, fitted to measurements (32 query and 8 KV heads of 128, one to 37 requests, 1 to 8192 fresh
// tokens, up to 16000 cached): the fixed part, the steps of the busiest SM, the row blocks, the join.  Heads of 64 take
// about 0.7 of a tile step.  Examples, measured (ROWS / TILES): 1 x 8 tokens over 2000 keys 11 / 15, 1 x 32 16 / 19, 1 x 64 21 / 25, 1 x 128 40 / 26,
// 4 x 16 over 5000 41 / 38, 8 x 64 over 4096 231 / 63, 32 x 4 over 2000 41 / 84, a prompt of 4096 tokens 989 / 160.
// Of 24 measured calls around the border the estimates miss the faster kernel in four: 1 x 64 (by 4 us), 8 x 16 over 200 keys (2) and
// prompts without a prefix, whose short key ranges the streaming kernel's fixed cost outweighs: 1 x 200 20 / 14, 4 x 100 36 / 13.
// (A third way, pages decoded to a contiguous bf16 copy for the kernel of pd_prefill_attention, took 303 us for 1 x 512 over
// 16000 keys where TILES take 162, 165 for the prompt, and was ahead only for short prompts without a prefix, 131 against 142
// at 8 x 1000; its copy of n_req * max_kv_len rows was the price.)
enum class Path { ROWS, TILES };

Path choose_path(const PagedRuns& r, const PagedTilesPlan& plan, const int32_t* cu, const int32_t* prefix, int longest) {
  const int group = r.n_q_heads / r.n_kv_heads;
  const int row_tokens = paged_rows_block(group, longest), tile_tokens = 2 * (128 / group);
  double rows_steps = 0, tile_steps = 0;  // 16 keys of a row block; 128 keys of a tile block
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
  }
  const double sms = 148, hd = r.head_dim == 128 ? 1.0 : 0.7, items = static_cast<double>(r.tile_blocks) * r.n_kv_heads;
  const double splits = plan.part_rows == 1ll * r.n_tokens * r.n_q_heads ? plan.n_splits : 1;  // (of all key ranges)
  const double t_rows = 8 + 0.9e-3 * std::fmin(rows_steps, 8000) + 0.85e-3 * std::fmax(rows_steps - 8000, 0);
  const double tile_step = 1.0 * longest * group <= 128 ? 2.0 : 2.35;  // one row tile of a block in use, or both
  const double t_tiles = 11 + hd * tile_step * std::fmax(tile_steps / sms, std::ceil(r.max_kv / 128.0) / splits) + 2.5 * items * splits / sms +
                         (splits > 1 ? 5 : 0);
  // what a kernel can address: blocks along one grid axis
  const bool rows_fit = first_slot(r.n_tokens, r.n_req, row_tokens) <= 65535;
  // PD_PAGED_PREFILL=0, 1 forces a kernel where it fits (for A/B timing and tests)
  static const int forced = [] {
    const char* e = std::getenv("PD_PAGED_PREFILL");
    return e ? std::atoi(e) : -1;
  }();
  if (forced == 1 || !rows_fit) return Path::TILES;
  return forced == 0 || t_rows <= t_tiles ? Path::ROWS : Path::TILES;
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_paged_prefill_attention_workspace_bytes(const pd_layer_cfg* cfg, int32_t n_req, int32_t max_kv_len,
                                                                size_t* out_bytes) {
  using namespace pd;
  PD_TRY(check_paged_heads(cfg));
  if (!out_bytes || n_req < 0 || max_kv_len < 0) return PD_ERR_INVALID_ARG;
  size_t need = 0;  // the larger of what the two kernels need, whatever the lengths
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
    if (len < 0) return PD_ERR_INVALID_ARG;
    if (len == 0) continue;  // (its prefix plays no role)
    if (pre < 0 || pre + len > cap) return PD_ERR_INVALID_ARG;
    if (len > longest) longest = static_cast<int>(len);
    if (pre + len > r.max_kv) r.max_kv = static_cast<int>(pre + len);
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
  const PagedTilesPlan plan = paged_tiles_plan(r, cu_host, prefix_host);
  const Path path = choose_path(r, plan, cu_host, prefix_host, longest);
  const size_t part_rows = path == Path::ROWS ? paged_rows_part_rows() : paged_tiles_part_rows();
  PagedParts parts;
  parts.o = static_cast<float*>(workspace);
  parts.ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + paged_parts_ml_offset(part_rows, cfg->head_dim));
  return path == Path::ROWS ? launch_paged_rows(r, longest, parts, st) : launch_paged_tiles(r, plan, parts, st);
}
