// Writing the 4-bit paged KV cache, from projection rows with norm and rotation on the way (pd_paged_kv4_append) or from a bf16 cache
// (pd_paged_kv4_write), and reading it back (pd_paged_kv4_read).
//
// Per row and KV head, 16 neighbouring features x in units of 2^exp: scale = E4M3(max|x| / 6), code = E2M1(x / scale).  Every row
// has scales of its own, so rows are independent: no page is rescaled, nothing is shared or atomic.  k is transformed in double
// (a few per cent of the arithmetic units' time): a code is a decision, and one that depended on the order of an fp32 sum
// would make a cache filled in one piece differ from one filled in chunks or elsewhere.
// All three are bound by HBM at size and by launch and a chain of loads (length, page number) at decode sizes.
#include "pd_kv4.cuh"

namespace pd {
namespace {

constexpr int KW_THREADS = 256;
constexpr int KW_Q_HEADS = 4;  // query heads per block

struct Kv4AppendArgs {
  const bf16* qkv;            // [T, ldqkv]: q heads, k heads, v heads
  bf16* q_out;                // [T, Hq*hd] or NULL
  const int32_t* cu_seqlens;  // [n_req + 1], NULL: one row per request
  const int32_t* kv_len;      // [n_req] tokens cached before; negative: the request is left out
  int* err_word;
  QkTransform t;
  Kv4Cache c;
  int ldqkv, n_req, n_tokens, n_q_heads, n_kv_heads, q_blocks;
};

// The request of row `row`: how many requests end at or before it.  All lanes of a warp call it; its rows are the warp's
// WARP_ROWS neighbouring ones.  Up to 32 requests take one load and a vote per row.
template <int J>
__device__ __forceinline__ int request_of(const int32_t* cu, int n_req, int row) {
  const int lane = threadIdx.x & 31;
  if (n_req <= 32) {
    const int end = lane < n_req ? cu[lane + 1] : 0x7fffffff;
    int req = 0;
#pragma unroll
    for (int i = 0; i < 32 / J; ++i) {
      const int r = __shfl_sync(0xffffffffu, row, i * J);
      const int n = __popc(__ballot_sync(0xffffffffu, end <= r));
      if (lane / J == i) req = n;
    }
    return req;
  }
  int lo = 0, hi = n_req;  // the first r with cu[r + 1] > row
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid + 1] <= row) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// The row of a position of a sequence in the pool, in rows; -1: no such page.
__device__ __forceinline__ long long pool_row(const Kv4Cache& c, int seq, int pos, int n_kv_heads, int kvh) {
  const int pi = pos >> c.log2_page;
  if (pi >= c.table_ld) return -1;
  const int page = c.table[static_cast<size_t>(seq) * c.table_ld + pi];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(c.n_pages)) return -1;
  return ((1ll * page * n_kv_heads + kvh) << c.log2_page) + (pos & ((1 << c.log2_page) - 1));
}

// Blocks along y are groups of query heads, then K heads, then V heads.
template <int HD, bool PAIRS>
__global__ void __launch_bounds__(KW_THREADS, 3) kv4_append_kernel(const Kv4AppendArgs a) {
  constexpr int J = HD / 16;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int row = blockIdx.x * (KW_THREADS / J) + threadIdx.x / J, j = threadIdx.x % J;
  const HeadShare<PAIRS> at(j, a.t.rot);
  const bf16* const src = a.qkv + static_cast<size_t>(row < a.n_tokens ? row : 0) * a.ldqkv;
  const int kv_block = static_cast<int>(blockIdx.y) - a.q_blocks;  // below 0: query heads
  // the row goes out first, its place is looked up meanwhile
  int req = row, first = row, len = -1;
  auto find_request = [&] {
    if (a.cu_seqlens) {
      req = request_of<J>(a.cu_seqlens, a.n_req, row);
      if (req < a.n_req) first = a.cu_seqlens[req];
    }
    if (row < a.n_tokens && req < a.n_req) len = a.kv_len[req];
  };
  auto position = [&](bool& live, bool& far) {
    const long long p = 1ll * len + (row - first);
    far = len >= 0 && (a.t.rot > 0 ? p >= a.t.n_pos : p > 0x7fffffffll);
    live = len >= 0 && !far;
    return live ? static_cast<int>(p) : 0;
  };
  bool live, far;
  if (kv_block < 0) {
    const int h0 = blockIdx.y * KW_Q_HEADS, n_h = a.n_q_heads - h0;
    HeadsOfRow<HD, PAIRS, KW_Q_HEADS> heads(src + h0 * HD, n_h, row < a.n_tokens, at);
    find_request();
    const int pos = position(live, far);
    bf16* const dst = a.q_out + static_cast<size_t>(live ? row : 0) * (a.n_q_heads * HD) + h0 * HD;
    heads.transform(dst, n_h, live, at, a.t.q_gain, a.t.eps, a.t.table + static_cast<size_t>(pos) * (a.t.rot / 2), j);
    return;
  }
  const bool is_v = kv_block >= a.n_kv_heads;
  const int kvh = is_v ? kv_block - a.n_kv_heads : kv_block;
  uint4 w[2] = {}, g[2] = {};
  if (row < a.n_tokens) load_share(src + (a.n_q_heads + kv_block) * HD, at.a, at.b, w);
  if (!is_v && a.t.k_gain) load_share(a.t.k_gain, at.a, at.b, g);
  const int exp = kv4_exp(is_v ? a.c.v_exp : a.c.k_exp, kvh);
  find_request();
  const int pos = position(live, far);
  float cs[16] = {};
  if (!is_v && live && at.turns) load_angles(a.t.table + static_cast<size_t>(pos) * (a.t.rot / 2), j, cs);
  const long long place = live ? pool_row(a.c, req, pos, a.n_kv_heads, kvh) : -1;
  if ((far || (live && place < 0)) && j == 0) report_place(a.err_word);
  const size_t to = static_cast<size_t>(place < 0 ? 0 : place);
  float t[16];
  if (is_v) {
    unpack8(w[0], t);
    unpack8(w[1], t + 8);
    const float unit = pow2f(-exp);
#pragma unroll
    for (int e = 0; e < 16; ++e) t[e] = __fmul_rz(t[e], unit);  // (a finite value stays one, and an infinite one stays infinite)
  } else {
    double f[16];
    transform_share<HD, PAIRS>(w, a.t.k_gain != nullptr, g, a.t.eps, at.turns, cs, static_cast<double>(pow2f(-exp)), f);
#pragma unroll
    for (int e = 0; e < 16; ++e) t[e] = sticky_float(f[e]);
  }
  store_kv4<HD, PAIRS>(t, at, j, a.t.rot, place >= 0, (is_v ? a.c.v : a.c.k) + to * (HD / 2), (is_v ? a.c.v_scale : a.c.k_scale) + to * (HD / 16));
}

// ------------------------------------------------------------------------------- between pages and a contiguous bf16 cache
struct Kv4CopyArgs {
  Kv4Cache c;
  bf16* k;                 // [batch_cap, Hkv, len_cap, hd]
  bf16* v;
  const int32_t* begin;
  const int32_t* end;
  const int32_t* slots;
  const int32_t* origin;
  int* err_word;
  int n_seqs, max_len, n_kv_heads, batch_cap, len_cap;
};
// What a sequence's range is, and where its rows lie in the bf16 cache.
struct CopyRange {
  int begin, n, slot, origin;
};
__device__ __forceinline__ CopyRange copy_range(const Kv4CopyArgs& a, int seq) {
  CopyRange r;
  r.begin = a.begin ? a.begin[seq] : 0;
  const long long n = 1ll * a.end[seq] - r.begin;
  r.n = static_cast<int>(max(0ll, min(n, static_cast<long long>(a.max_len))));
  r.slot = a.slots ? a.slots[seq] : seq;
  r.origin = a.origin ? a.origin[seq] : 0;
  return r;
}
// The bf16 row of position begin + i (K and V alike), in rows; -1: outside.
__device__ __forceinline__ long long bf16_row(const Kv4CopyArgs& a, const CopyRange& r, int i, int kvh) {
  const long long row = 1ll * r.begin + i - r.origin;
  if (static_cast<unsigned>(r.slot) >= static_cast<unsigned>(a.batch_cap) || row < 0 || row >= a.len_cap) return -1;
  return (1ll * r.slot * a.n_kv_heads + kvh) * a.len_cap + row;
}
__device__ __forceinline__ long long copy_pool_row(const Kv4CopyArgs& a, const CopyRange& r, int seq, int i, int kvh) {
  const long long pos = 1ll * r.begin + i;
  return pos < 0 || pos > 0x7fffffffll ? -1 : pool_row(a.c, seq, static_cast<int>(pos), a.n_kv_heads, kvh);
}

// hd / 16 lanes have a row of K and of V.
template <int HD>
__global__ void __launch_bounds__(KW_THREADS) kv4_write_kernel(const Kv4CopyArgs a) {
  constexpr int J = HD / 16;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int seq = blockIdx.z, kvh = blockIdx.y, j = threadIdx.x % J;
  const CopyRange r = copy_range(a, seq);
  const int i = blockIdx.x * (KW_THREADS / J) + threadIdx.x / J;
  const bool mine = i < r.n;
  const long long to = mine ? copy_pool_row(a, r, seq, i, kvh) : -1, from = mine ? bf16_row(a, r, i, kvh) : -1;
  const bool live = to >= 0 && from >= 0;
  if (mine && !live && j == 0) report_place(a.err_word);
  const HeadShare<true> at(j, 0);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    uint4 w[2] = {};
    if (live) load_share((kv ? a.v : a.k) + static_cast<size_t>(from) * HD, at.a, at.b, w);
    float t[16];
    unpack8(w[0], t);
    unpack8(w[1], t + 8);
    const float unit = pow2f(-kv4_exp(kv ? a.c.v_exp : a.c.k_exp, kvh));
#pragma unroll
    for (int e = 0; e < 16; ++e) t[e] = __fmul_rz(t[e], unit);
    const size_t row = static_cast<size_t>(live ? to : 0);
    store_kv4<HD, true>(t, at, j, 0, live, (kv ? a.c.v : a.c.k) + row * (HD / 2), (kv ? a.c.v_scale : a.c.k_scale) + row * (HD / 16));
  }
}

__device__ __forceinline__ uint4 kv4_to_bf16(uint32_t codes, float unit) {
  uint32_t h[4];
  asm("{ .reg .b8 b0, b1, b2, b3; mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0; cvt.rn.f16x2.e2m1x2 %1, b1; cvt.rn.f16x2.e2m1x2 %2, b2; cvt.rn.f16x2.e2m1x2 %3, b3; }"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    asm("{ .reg .b16 l, u; mov.b32 {l, u}, %2; cvt.f32.f16 %0, l; cvt.f32.f16 %1, u; }" : "=f"(lo), "=f"(hi) : "r"(h[i]));
    o[i] = ptx::pack_bf16(lo * unit, hi * unit);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// A lane turns 8 features, 4 bytes of codes, into 16 bytes: hd / 8 lanes have a row, so that stores are contiguous.  KR_ROWS rows
// of K and of V per lane are in flight together.
constexpr int KR_ROWS = 4;
template <int HD>
__global__ void __launch_bounds__(KW_THREADS) kv4_read_kernel(const Kv4CopyArgs a) {
  constexpr int J = HD / 8, ROWS = KW_THREADS / J;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int seq = blockIdx.z, kvh = blockIdx.y, j = threadIdx.x % J;
  const CopyRange r = copy_range(a, seq);
  const int i0 = blockIdx.x * (ROWS * KR_ROWS) + threadIdx.x / J;
  if (static_cast<int>(blockIdx.x) * (ROWS * KR_ROWS) >= r.n) return;
  long long from[KR_ROWS];
#pragma unroll
  for (int n = 0; n < KR_ROWS; ++n) from[n] = i0 + n * ROWS < r.n ? copy_pool_row(a, r, seq, i0 + n * ROWS, kvh) : -1;
  uint32_t w[2][KR_ROWS], s[2][KR_ROWS];
#pragma unroll
  for (int n = 0; n < KR_ROWS; ++n) {
    if (from[n] < 0) continue;
    const size_t row = static_cast<size_t>(from[n]);
    w[0][n] = *reinterpret_cast<const uint32_t*>(a.c.k + row * (HD / 2) + j * 4);
    w[1][n] = *reinterpret_cast<const uint32_t*>(a.c.v + row * (HD / 2) + j * 4);
    s[0][n] = a.c.k_scale[row * (HD / 16) + j / 2];
    s[1][n] = a.c.v_scale[row * (HD / 16) + j / 2];
  }
  const float k_unit = pow2f(kv4_exp(a.c.k_exp, kvh)), v_unit = pow2f(kv4_exp(a.c.v_exp, kvh));
#pragma unroll
  for (int n = 0; n < KR_ROWS; ++n) {
    const int i = i0 + n * ROWS;
    if (i >= r.n) continue;
    const long long to = bf16_row(a, r, i, kvh);
    if (from[n] < 0 || to < 0) {
      if (j == 0) report_place(a.err_word);
      continue;
    }
    const size_t at = static_cast<size_t>(to) * HD + j * 8;
    *reinterpret_cast<uint4*>(a.k + at) = kv4_to_bf16(w[0][n], e4m3_value(s[0][n]) * k_unit);
    *reinterpret_cast<uint4*>(a.v + at) = kv4_to_bf16(w[1][n], e4m3_value(s[1][n]) * v_unit);
  }
}

pd_status copy_args(const pd_layer_cfg* cfg, const pd_paged_kv4_cache* cache, const int32_t* begin, const int32_t* end, int32_t n_seqs,
                    int32_t max_len, const pd_kv_cache* flat, const int32_t* slots, const int32_t* origin, int32_t* err_word,
                    Kv4CopyArgs* a) {
  PD_TRY(check_kv4_heads(cfg));
  PD_TRY(kv4_cache_view(cache, &a->c));
  if (!flat || flat->struct_size != sizeof(pd_kv_cache) || n_seqs < 0 || n_seqs > cache->n_seqs || max_len < 0) return PD_ERR_INVALID_ARG;
  if (n_seqs > 65535) return PD_ERR_UNSUPPORTED_SHAPE;
  if (n_seqs == 0 || max_len == 0) return PD_OK;
  if (!end || !flat->k || !flat->v || flat->batch_cap <= 0 || flat->len_cap <= 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(flat->k) | reinterpret_cast<uintptr_t>(flat->v)) & 15u) return PD_ERR_INVALID_ARG;
  a->k = static_cast<bf16*>(flat->k); a->v = static_cast<bf16*>(flat->v);
  a->begin = begin; a->end = end; a->slots = slots; a->origin = origin; a->err_word = err_word;
  a->n_seqs = n_seqs; a->max_len = max_len; a->n_kv_heads = cfg->n_kv_heads;
  a->batch_cap = flat->batch_cap; a->len_cap = flat->len_cap;
  return PD_OK;
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_paged_kv4_append(const pd_layer_cfg* cfg, const pd_qk_transform* transform, const void* qkv, int32_t ldqkv,
                                         void* q_out, const int32_t* cu_dev, const int32_t* cu_host, int32_t n_req,
                                         const int32_t* kv_len_dev, const pd_paged_kv4_cache* cache, int32_t* err_word, void* stream) {
  using namespace pd;
  PD_TRY(check_kv4_heads(cfg));
  Kv4AppendArgs a{};
  PD_TRY(kv4_cache_view(cache, &a.c));
  PD_TRY(qk_transform_view(transform, cfg, &a.t));
  if (n_req < 0 || n_req > cache->n_seqs || (cu_dev == nullptr) != (cu_host == nullptr)) return PD_ERR_INVALID_ARG;
  int tokens = n_req;
  if (cu_host) {
    if (cu_host[0] != 0) return PD_ERR_INVALID_ARG;
    for (int r = 0; r < n_req; ++r)
      if (cu_host[r + 1] < cu_host[r]) return PD_ERR_INVALID_ARG;
    tokens = cu_host[n_req];
  }
  if (tokens == 0) return PD_OK;
  const int hd = cfg->head_dim;
  const long long width = (cfg->n_q_heads + 2ll * cfg->n_kv_heads) * hd;
  if (!qkv || !kv_len_dev || ldqkv < width || ldqkv % 8 != 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(qkv) | reinterpret_cast<uintptr_t>(q_out)) & 15u) return PD_ERR_INVALID_ARG;
  a.qkv = static_cast<const bf16*>(qkv); a.q_out = static_cast<bf16*>(q_out);
  a.cu_seqlens = cu_dev; a.kv_len = kv_len_dev; a.err_word = err_word;
  a.ldqkv = ldqkv; a.n_req = n_req; a.n_tokens = tokens; a.n_q_heads = cfg->n_q_heads; a.n_kv_heads = cfg->n_kv_heads;
  a.q_blocks = q_out ? (cfg->n_q_heads + KW_Q_HEADS - 1) / KW_Q_HEADS : 0;
  const int rows = KW_THREADS / (hd / 16);
  const dim3 grid((tokens + (rows - 1ll)) / rows, a.q_blocks + 2 * cfg->n_kv_heads), block(KW_THREADS);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_KV_APPEND, st);
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, block, 0, st, a); };
  const bool pairs = transform->layout == PD_ROPE_PAIRS;
  PD_CUDA_TRY(hd == 128 ? (pairs ? go(kv4_append_kernel<128, true>) : go(kv4_append_kernel<128, false>))
                        : (pairs ? go(kv4_append_kernel<64, true>) : go(kv4_append_kernel<64, false>)));
  count_launch();
  return PD_OK;
}

extern "C" pd_status pd_paged_kv4_write(const pd_layer_cfg* cfg, const pd_paged_kv4_cache* cache, const int32_t* begin, const int32_t* end,
                                        int32_t n_seqs, int32_t max_len, const pd_kv_cache* in, const int32_t* slots,
                                        const int32_t* origin, int32_t* err_word, void* stream) {
  using namespace pd;
  Kv4CopyArgs a{};
  PD_TRY(copy_args(cfg, cache, begin, end, n_seqs, max_len, in, slots, origin, err_word, &a));
  if (a.n_seqs == 0) return PD_OK;
  const int rows = KW_THREADS / (cfg->head_dim / 16);
  const dim3 grid((max_len + (rows - 1ll)) / rows, cfg->n_kv_heads, n_seqs), block(KW_THREADS);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_KV_APPEND, st);
  PD_CUDA_TRY(cfg->head_dim == 128 ? launch_pdl(kv4_write_kernel<128>, grid, block, 0, st, a) : launch_pdl(kv4_write_kernel<64>, grid, block, 0, st, a));
  count_launch();
  return PD_OK;
}

extern "C" pd_status pd_paged_kv4_read(const pd_layer_cfg* cfg, const pd_paged_kv4_cache* cache, const int32_t* begin, const int32_t* end,
                                       int32_t n_seqs, int32_t max_len, const pd_kv_cache* out, const int32_t* slots,
                                       const int32_t* origin, int32_t* err_word, void* stream) {
  using namespace pd;
  Kv4CopyArgs a{};
  PD_TRY(copy_args(cfg, cache, begin, end, n_seqs, max_len, out, slots, origin, err_word, &a));
  if (a.n_seqs == 0) return PD_OK;
  const int rows = KR_ROWS * (KW_THREADS / (cfg->head_dim / 8));
  const dim3 grid((max_len + (rows - 1ll)) / rows, cfg->n_kv_heads, n_seqs), block(KW_THREADS);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  PD_CUDA_TRY(cfg->head_dim == 128 ? launch_pdl(kv4_read_kernel<128>, grid, block, 0, st, a) : launch_pdl(kv4_read_kernel<64>, grid, block, 0, st, a));
  count_launch();
  return PD_OK;
}
