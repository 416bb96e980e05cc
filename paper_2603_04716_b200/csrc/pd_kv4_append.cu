// Writing the 4-bit paged KV cache, from projection rows with norm and rotation on the way (pd_paged_kv4_append) or from a bf16 cache
// (pd_paged_kv4_write), and reading it back (pd_paged_kv4_read).
//
// Per row and KV head, 16 neighbouring features x in units of 2^exp: scale = E4M3(max|x| / 6), code = E2M1(x / scale).  Every row
// has scales of its own, so rows are independent: no page is rescaled, nothing is shared or atomic.  k is transformed in double:
// a code is a decision, and one that depended on the order of an fp32 sum would make a cache filled in one piece differ from one
// filled in chunks or elsewhere.  (fp32 wherever a bound on its error shows that the decision is the same, double elsewhere: 68 us for
// the prompts below when double throughout took 64.)
// Bound by a chain of loads (length, page number) at decode sizes; at size reading back is bound by HBM, appending by HBM and
// by instructions together (two thirds of the issue slots).
// Measured, 32 + 8 + 8 heads of 128: append of 13,123 rows (284 MB) 60 us, 4.7 TB/s; of 256 rows 3.4; of one 2.5; read-back of 24
// prefixes (625 MB) 99.7 us, 6.3 TB/s; the same prefixes written from a bf16 cache 229 us, 2.7 TB/s (bound by instructions:
// 77 % of the issue slots, 80 % of the ALU pipe).
#include "pd_kv4.cuh"

namespace pd {
namespace {

constexpr int KW_THREADS = 128;
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

// The request of row `row`: how many requests end at or before it.  All lanes of a warp call it with the same row.
__device__ __forceinline__ int request_of(const int32_t* cu, int n_req, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = n_req;  // candidates lo .. lo + n - 1, and lo + n
  while (n > 32) {        // 32 equal parts at a time: those whose last request ends at or before the row are passed over
    const int part = (n + 31) / 32, last = min((lane + 1) * part, n) - 1;
    const int passed = __popc(__ballot_sync(0xffffffffu, lane * part < n && cu[lo + last + 1] <= row));
    lo += min(passed * part, n);
    n = min(part, n - min(passed * part, n));
  }
  return lo + __popc(__ballot_sync(0xffffffffu, lane < n && cu[lo + lane + 1] <= row));
}

// A warp has a row; blocks along y are groups of query heads, then of K heads, then of V heads, 256 features STEPS times each.  With
// many rows a warp goes on to further query heads, for what concerns the row (its request, position, angles, gains) is a third of the
// instructions: 63.3 -> 59.2 us for 13,123 rows of 32 + 8 + 8 heads of 128 (60 now); with 256 rows it would cost 0.6 of 3.4 us.
constexpr int query_rounds(int steps) { return steps == 4 ? 4 : 1; }
template <int HD, bool PAIRS, int STEPS>
__global__ void __launch_bounds__(KW_THREADS, STEPS == 4 ? 8 : 5) kv4_append_kernel(const Kv4AppendArgs a) {
  constexpr int J = HD / 8, STEP = heads_per_step<HD>(), HEADS = STEPS * STEP, Q_HEADS = query_rounds(STEPS) * HEADS;
  __shared__ __align__(16) float maxima[KW_THREADS * 2];
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, j = lane % J, mine = lane / J;
  const int row = blockIdx.x * (KW_THREADS / 32) + warp;
  if (row >= a.n_tokens) return;
  const int kv_blocks = (a.n_kv_heads + HEADS - 1) / HEADS, kv_block = static_cast<int>(blockIdx.y) - a.q_blocks;
  const bool is_q = kv_block < 0, is_v = kv_block >= kv_blocks;
  const int h0 = is_q ? blockIdx.y * Q_HEADS : (is_v ? kv_block - kv_blocks : kv_block) * HEADS;
  const int n_heads = min((is_q ? a.n_q_heads : a.n_kv_heads) - h0, is_q ? Q_HEADS : HEADS);
  const HeadShare<PAIRS> at(j, a.t.rot);
  const HeadShare<true> plain(j, 0);  // of V: neighbours
  // the row goes out first, its place is looked up meanwhile
  uint4 w[STEPS];
  const bf16* const src = a.qkv + static_cast<size_t>(row) * a.ldqkv + ((is_q ? 0 : a.n_q_heads + (is_v ? a.n_kv_heads : 0)) + h0) * HD;
  if (is_v) load_heads<HD, true>(w, src, n_heads, plain); else load_heads<HD, PAIRS>(w, src, n_heads, at);
  int req = row, first = row;
  if (a.cu_seqlens) {
    req = request_of(a.cu_seqlens, a.n_req, row);
    if (req >= a.n_req) return;
    first = a.cu_seqlens[req];
  }
  const int len = a.kv_len[req];
  if (len < 0 || row < first) return;  // a request that is left out (and never with consistent inputs)
  const uint32_t pos = static_cast<uint32_t>(len) + static_cast<uint32_t>(row - first);
  if (a.t.rot > 0 && pos >= static_cast<uint32_t>(a.t.n_pos)) {
    report_place(a.err_word);
    return;
  }
  const float2* const angles = a.t.table + static_cast<size_t>(pos) * (a.t.rot / 2);
  if (is_q) {
    with_flags(a.t.q_gain != nullptr, a.t.rot == HD, [&](auto norm, auto whole) {
      const FastTransform<HD, PAIRS, decltype(norm)::value, decltype(whole)::value> transform(at, a.t.q_gain, angles, j);
      bf16* const dst = a.q_out + (static_cast<size_t>(row) * a.n_q_heads + h0) * HD;
#pragma unroll 1
      for (int h = 0;;) {
        transform(w, dst + h * HD, n_heads - h, at, a.t.eps_fast);
        if ((h += HEADS) >= n_heads) break;
        load_heads<HD, PAIRS>(w, src + h * HD, n_heads - h, at);
      }
    });
    return;
  }
  const uint32_t pi = pos >> a.c.log2_page;
  const int page = pi < static_cast<uint32_t>(a.c.table_ld) ? a.c.table[static_cast<size_t>(req) * a.c.table_ld + pi] : -1;
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.c.n_pages)) {
    report_place(a.err_word);
    return;
  }
  // the row of the pool of this lane's first head
  const uint32_t to = ((static_cast<uint32_t>(page) * a.n_kv_heads + h0 + mine) << a.c.log2_page) + (pos & ((1u << a.c.log2_page) - 1));
  uint8_t* const codes = is_v ? a.c.v : a.c.k;
  uint8_t* const scales = is_v ? a.c.v_scale : a.c.k_scale;
  const int32_t* const exps = is_v ? a.c.v_exp : a.c.k_exp;
  // group s of the heads
  auto store = [&](int s, const float (&t)[8], const auto& share) {
    const bool live = s * STEP + mine < n_heads;
    const size_t at_row = to + (static_cast<uint32_t>(s * STEP) << a.c.log2_page);
    store_kv4<HD>(t, live ? kv4_exp(exps, h0 + s * STEP + mine) : 0, share, j, live, maxima + warp * 64, codes + at_row * (HD / 2),
                  scales + at_row * (HD / 16));
  };
  if (is_v) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (s * STEP >= n_heads) break;
      float t[8];
      unpack8(w[s], t);
      store(s, t, plain);
    }
    return;
  }
  with_flags(a.t.k_gain != nullptr, a.t.rot == HD, [&](auto norm, auto whole) {
    const ExactTransform<HD, PAIRS, decltype(norm)::value, decltype(whole)::value> transform(at, a.t.k_gain, angles, j);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (s * STEP >= n_heads) break;
      double f[8];
      float t[8];
      transform(w[s], a.t.eps, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = sticky_float(f[e]);
      store(s, t, at);
    }
  });
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
// What a sequence's range is, and where its rows lie in the bf16 cache: of positions begin + i, i below n, those with lo <= i < hi have
// a row there and an entry of the page table.
struct CopyRange {
  int begin, n, lo, hi;
  long long row0;  // bf16 row of position begin (K and V alike); may lie outside
};
__device__ __forceinline__ CopyRange copy_range(const Kv4CopyArgs& a, int seq, int kvh) {
  CopyRange r;
  r.begin = a.begin ? a.begin[seq] : 0;
  const int slot = a.slots ? a.slots[seq] : seq;
  const long long n = min(1ll * a.end[seq] - r.begin, static_cast<long long>(a.max_len));
  const long long shift = 1ll * r.begin - (a.origin ? a.origin[seq] : 0);
  const long long lo = max(max(0ll, -shift), -static_cast<long long>(r.begin));
  const long long hi = min(min(n, a.len_cap - shift), (1ll * a.c.table_ld << a.c.log2_page) - r.begin);
  const bool there = static_cast<unsigned>(slot) < static_cast<unsigned>(a.batch_cap) && hi > lo;
  r.n = static_cast<int>(max(0ll, n));
  r.lo = there ? static_cast<int>(lo) : 0;
  r.hi = there ? static_cast<int>(hi) : 0;
  r.row0 = (1ll * slot * a.n_kv_heads + kvh) * a.len_cap + shift;
  return r;
}
// The row in the pool of position begin + i, lo <= i < hi; false: no such page.
__device__ __forceinline__ bool copy_pool_row(const Kv4CopyArgs& a, const CopyRange& r, int seq, int i, int kvh, uint32_t& row) {
  const int pos = r.begin + i, page = a.c.table[static_cast<size_t>(seq) * a.c.table_ld + (pos >> a.c.log2_page)];
  row = ((static_cast<uint32_t>(page) * a.n_kv_heads + kvh) << a.c.log2_page) + (pos & ((1 << a.c.log2_page) - 1));
  return static_cast<unsigned>(page) < static_cast<unsigned>(a.c.n_pages);
}

// hd / 8 lanes have a row of K and of V.
template <int HD>
__global__ void __launch_bounds__(KW_THREADS) kv4_write_kernel(const Kv4CopyArgs a) {
  constexpr int J = HD / 8;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int seq = blockIdx.z, kvh = blockIdx.y, j = threadIdx.x % J;
  const CopyRange r = copy_range(a, seq, kvh);
  const int i = blockIdx.x * (KW_THREADS / J) + threadIdx.x / J;
  uint32_t to = 0;
  const bool live = i >= r.lo && i < r.hi && copy_pool_row(a, r, seq, i, kvh, to);
  if (i < r.n && !live && j == 0) report_place(a.err_word);
  const size_t from = static_cast<size_t>(live ? r.row0 + i : 0);
  const HeadShare<true> at(j, 0);
  uint4 w[2] = {};
  if (live) {
    w[0] = at.load(a.k + from * HD);
    w[1] = at.load(a.v + from * HD);
  }
  const size_t row = to;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    float t[8];
    unpack8(w[kv], t);
    store_kv4<HD>(t, kv4_exp(kv ? a.c.v_exp : a.c.k_exp, kvh), at, j, live, nullptr, (kv ? a.c.v : a.c.k) + row * (HD / 2),
                  (kv ? a.c.v_scale : a.c.k_scale) + row * (HD / 16));
  }
}

// Eight codes times `unit`: eight bf16 values, exactly.
__device__ __forceinline__ uint4 kv4_to_bf16(uint32_t codes, uint64_t unit) {
  uint32_t h[4], o[4];
  asm("{ .reg .b8 b0, b1, b2, b3; mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0; cvt.rn.f16x2.e2m1x2 %1, b1; cvt.rn.f16x2.e2m1x2 %2, b2; cvt.rn.f16x2.e2m1x2 %3, b3; }"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    asm("{ .reg .b16 l, u; mov.b32 {l, u}, %2; cvt.f32.f16 %0, l; cvt.f32.f16 %1, u; }" : "=f"(lo), "=f"(hi) : "r"(h[i]));
    ptx::unpack_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(lo, hi), unit), lo, hi);
    o[i] = ptx::pack_bf16(lo, hi);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// A lane turns 16 features, 8 bytes of codes and their scale, into 32 bytes, one store where the cache starts on 32 bytes (WIDE): hd / 16
// lanes have a row, KR_ROWS rows of K and of V per lane are in flight together.  (With 8 features a lane the instructions were the
// bound: 104 us instead of 99.5 for 24 prefixes, 625 MB; 4 rows in flight: 100.4, and 2.5 us instead of 1.8 for one prefix
// of 1,500 tokens.)
constexpr int KR_ROWS = 2;
template <int HD, bool WIDE>
__global__ void __launch_bounds__(KW_THREADS) kv4_read_kernel(const Kv4CopyArgs a) {
  constexpr int J = HD / 16, ROWS = KW_THREADS / J;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int seq = blockIdx.z, kvh = blockIdx.y, j = threadIdx.x % J;
  const CopyRange r = copy_range(a, seq, kvh);
  const int i0 = blockIdx.x * (ROWS * KR_ROWS) + threadIdx.x / J;
  if (static_cast<int>(blockIdx.x) * (ROWS * KR_ROWS) >= r.n) return;
  uint2 w[2][KR_ROWS];
  uint32_t s[2][KR_ROWS];
  bool live[KR_ROWS];
#pragma unroll
  for (int n = 0; n < KR_ROWS; ++n) {
    const int i = i0 + n * ROWS;
    uint32_t row;
    live[n] = i >= r.lo && i < r.hi && copy_pool_row(a, r, seq, i, kvh, row);
    if (live[n]) {
      const size_t at = static_cast<size_t>(row) * J + j;
      w[0][n] = reinterpret_cast<const uint2*>(a.c.k)[at];
      w[1][n] = reinterpret_cast<const uint2*>(a.c.v)[at];
      s[0][n] = a.c.k_scale[at];
      s[1][n] = a.c.v_scale[at];
    } else if (i < r.n && j == 0) {
      report_place(a.err_word);
    }
  }
  const float unit[2] = {pow2f(kv4_exp(a.c.k_exp, kvh)), pow2f(kv4_exp(a.c.v_exp, kvh))};
  const long long out = (r.row0 + i0) * HD + j * 16;
  bf16* const base[2] = {a.k + out, a.v + out};
#pragma unroll
  for (int n = 0; n < KR_ROWS; ++n) {
    if (!live[n]) continue;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const uint64_t u = dup_f32x2(e4m3_value(s[kv][n]) * unit[kv]);
      const uint4 x = kv4_to_bf16(w[kv][n].x, u), y = kv4_to_bf16(w[kv][n].y, u);
      bf16* const to = base[kv] + n * ROWS * HD;
      if (WIDE) {
        const uint32_t o[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        ptx::st_global_v8(to, o);
      } else {
        reinterpret_cast<uint4*>(to)[0] = x;
        reinterpret_cast<uint4*>(to)[1] = y;
      }
    }
  }
}

pd_status copy_args(const pd_layer_cfg* cfg, const pd_paged_kv4_cache* cache, const int32_t* begin, const int32_t* end, int32_t n_seqs,
                    int32_t max_len, const pd_kv_cache* flat, const int32_t* slots, const int32_t* origin, int32_t* err_word,
                    Kv4CopyArgs* a) {
  PD_TRY(check_kv4_heads(cfg));
  PD_TRY(kv4_cache_view(cache, cfg->n_kv_heads, &a->c));
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
  PD_TRY(kv4_cache_view(cache, cfg->n_kv_heads, &a.c));
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
  // few rows: short chains count, so a warp has few heads; many: what concerns a row is done once for many heads.  Two and four steps, 32 + 8
  // + 8 heads of 128, in us: 256 rows 3.9 and 6.6, 512 4.9 and 8.3, 1024 8.2 and 9.3, 1280 10.6 and 10.3, 1536 13.7 and 11.2, 4096 33 and 21
  const int steps = tokens <= 1024 ? 2 : 4;
  const int heads = steps * (256 / hd), q_heads = heads * query_rounds(steps), rows = KW_THREADS / 32;
  a.q_blocks = q_out ? (cfg->n_q_heads + q_heads - 1) / q_heads : 0;
  const dim3 grid((tokens + (rows - 1ll)) / rows, a.q_blocks + 2 * ((cfg->n_kv_heads + heads - 1) / heads));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_KV_APPEND, st);
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(KW_THREADS), 0, st, a); };
  const bool pairs = transform->layout == PD_ROPE_PAIRS;
  auto of_steps = [&](auto n) {
    constexpr int S = decltype(n)::value;
    return hd == 128 ? (pairs ? go(kv4_append_kernel<128, true, S>) : go(kv4_append_kernel<128, false, S>))
                     : (pairs ? go(kv4_append_kernel<64, true, S>) : go(kv4_append_kernel<64, false, S>));
  };
  PD_CUDA_TRY(steps == 4 ? of_steps(std::integral_constant<int, 4>()) : of_steps(std::integral_constant<int, 2>()));
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
  const int rows = KW_THREADS / (cfg->head_dim / 8);
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
  const int rows = KR_ROWS * (KW_THREADS / (cfg->head_dim / 16));
  const dim3 grid((max_len + (rows - 1ll)) / rows, cfg->n_kv_heads, n_seqs), block(KW_THREADS);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 31u) == 0;
  TraceScope ts(PD_K_KV_APPEND, st);
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, block, 0, st, a); };
  PD_CUDA_TRY(cfg->head_dim == 128 ? (wide ? go(kv4_read_kernel<128, true>) : go(kv4_read_kernel<128, false>))
                                   : (wide ? go(kv4_read_kernel<64, true>) : go(kv4_read_kernel<64, false>)));
  count_launch();
  return PD_OK;
}
