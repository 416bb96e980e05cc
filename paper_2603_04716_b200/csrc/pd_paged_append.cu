// Appending to the 8-bit paged KV cache, with the rotary position rotation on the way (pd_paged_kv_append).
//
// Per fresh row at position p: q and k heads are rotated (x_i, x_{i + hd/2}) -> (x_i c - x_{i+hd/2} s, x_{i+hd/2} c + x_i s)
// in fp32, q is stored in bf16, k and v go to their page as E4M3 codes.  One scale per (page, KV head) and K or V: the
// smallest power of two with max|x| <= 448 * scale over the tokens the page has received since its first slot was written.
// When a later token needs a larger scale, the codes already in the page are multiplied by the (power of two) quotient of
// the scales, which is exact except where a value falls into the subnormal codes.
//
// Whoever writes tokens to a (page, head) also owns its scale, so nothing is atomic: a warp per (sequence, KV head) when
// every sequence gets one token (decode), a block per (page, head) of a ragged batch of longer runs (prefill).  Both are
// bound by HBM at size (rows in, q and codes out) and by launch latency at decode sizes.  Measured: prompts of 298 MB in 53 us =
// 5.6 TB/s, 87 % of a copy; one token of 256 sequences 4.5 us, of one sequence 2.8 us (a chain of three loads: length, page
// number, scale).
#include "pd_paged.cuh"

namespace pd {
namespace {

struct AppendArgs {
  const bf16* qkv;            // [T, ldqkv]: q heads, k heads, v heads
  bf16* q_out;                // [T, Hq*hd] or NULL
  const float2* rope;         // [max_pos, hd/2] (cos, sin)
  const int32_t* cu_seqlens;  // [n_req + 1], NULL: one row per request
  const int32_t* kv_len;      // [n_req] tokens cached before; negative: the request is left out
  int* err_word;
  PagedCache c;
  int ldqkv, n_req, n_tokens, n_q_heads, n_kv_heads, max_pos;
};

__device__ __forceinline__ void unpack8(const uint4& v, float* f) {
  f[0] = ptx::bf16_lo(v.x); f[1] = ptx::bf16_hi(v.x);
  f[2] = ptx::bf16_lo(v.y); f[3] = ptx::bf16_hi(v.y);
  f[4] = ptx::bf16_lo(v.z); f[5] = ptx::bf16_hi(v.z);
  f[6] = ptx::bf16_lo(v.w); f[7] = ptx::bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(ptx::pack_bf16(f[0], f[1]), ptx::pack_bf16(f[2], f[3]), ptx::pack_bf16(f[4], f[5]),
                    ptx::pack_bf16(f[6], f[7]));
}

// A task is 16 features of one head of one row: 8 in the lower half of the head and their rotation partners.
template <int HD>
__device__ __forceinline__ void load_task(const bf16* head, int j, float (&f)[16]) {
  unpack8(*reinterpret_cast<const uint4*>(head + j * 8), f);
  unpack8(*reinterpret_cast<const uint4*>(head + HD / 2 + j * 8), f + 8);
}
__device__ __forceinline__ void load_angles(const float2* row, int j, float (&cs)[16]) {
  const float4* p = reinterpret_cast<const float4*>(row + j * 8);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = p[i];
    cs[4 * i] = v.x; cs[4 * i + 1] = v.y; cs[4 * i + 2] = v.z; cs[4 * i + 3] = v.w;
  }
}
// Every product and sum rounded on its own (no contraction), so that the result is that of the written formula.
__device__ __forceinline__ void rotate(float (&f)[16], const float (&cs)[16]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float c = cs[2 * e], s = cs[2 * e + 1], lo = f[e], hi = f[8 + e];
    f[e] = __fsub_rn(__fmul_rn(lo, c), __fmul_rn(hi, s));
    f[8 + e] = __fadd_rn(__fmul_rn(hi, c), __fmul_rn(lo, s));
  }
}
// An infinite value has no code and no finite scale: it is stored as NaN, like a NaN, and takes no part in the scale.
__device__ __forceinline__ float finite_max(float (&f)[16], float amax) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    if (!(fabsf(f[e]) <= 3.402823466e38f)) f[e] = __int_as_float(0x7fc00000);
    amax = fmaxf(amax, fabsf(f[e]));  // (fmaxf drops a NaN)
  }
  return amax;
}
template <int HD>
__device__ __forceinline__ void store_codes(uint8_t* row, int j, const float (&f)[16], float inv) {
  uint2 w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float* g = f + 8 * h;
    w[h].x = ptx::cvt_e4m3x2(g[0] * inv, g[1] * inv) | (ptx::cvt_e4m3x2(g[2] * inv, g[3] * inv) << 16);
    w[h].y = ptx::cvt_e4m3x2(g[4] * inv, g[5] * inv) | (ptx::cvt_e4m3x2(g[6] * inv, g[7] * inv) << 16);
  }
  *reinterpret_cast<uint2*>(row + j * 8) = w[0];
  *reinterpret_cast<uint2*>(row + HD / 2 + j * 8) = w[1];
}
// Sixteen codes times a power of two <= 1, rounded to codes again.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float r) {
  const uint32_t a = e4m3x2_to_f16x2(static_cast<uint16_t>(w)), b = e4m3x2_to_f16x2(static_cast<uint16_t>(w >> 16));
  const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&a));
  const float2 fb = __half22float2(*reinterpret_cast<const __half2*>(&b));
  return ptx::cvt_e4m3x2(fa.x * r, fa.y * r) | (ptx::cvt_e4m3x2(fb.x * r, fb.y * r) << 16);
}
__device__ __forceinline__ void rescale_rows(uint8_t* base, int bytes, float r, int tid, int n_threads) {
  uint4* p = reinterpret_cast<uint4*>(base);
  for (int i = tid; i < bytes / 16; i += n_threads) {
    uint4 v = p[i];
    v.x = rescale4(v.x, r); v.y = rescale4(v.y, r); v.z = rescale4(v.z, r); v.w = rescale4(v.w, r);
    p[i] = v;
  }
}
__device__ __forceinline__ void report(int* err_word) {
  if (err_word) atomicExch(err_word, 2);
}

// --------------------------------------------------------------- one token per sequence
constexpr int AD_WARPS = 4;

// One warp per (sequence, KV head): its K row, its V row and the G query heads of the group.  Lanes 0 .. J-1 hold K,
// J .. 2J-1 hold V (J = hd / 16 tasks a row), the others begin with q.
template <int HD>
__global__ void __launch_bounds__(AD_WARPS * 32) append_decode_kernel(const AppendArgs a) {
  constexpr int J = HD / 16;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int item = blockIdx.x * AD_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (item >= a.n_req * a.n_kv_heads) return;
  const int req = item / a.n_kv_heads, kvh = item - req * a.n_kv_heads;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int pos = a.kv_len[req];
  if (pos < 0) return;  // a padding row of the batch
  const int pi = pos >> a.c.log2_page;
  if (pos >= a.max_pos) {
    if (lane == 0) report(a.err_word);
    return;
  }
  const int page = pi < a.c.table_ld ? a.c.table[static_cast<size_t>(req) * a.c.table_ld + pi] : -1;
  const bf16* row = a.qkv + static_cast<size_t>(req) * a.ldqkv;
  const float2* rope = a.rope + static_cast<size_t>(pos) * (HD / 2);
  const int j = lane % J;
  float cs[16];
  load_angles(rope, j, cs);

  const int part = lane / J;  // 0: K, 1: V, above: query heads
  float f[16];
  bool have = false;
  if (part < 2) {
    load_task<HD>(row + (a.n_q_heads + (part ? a.n_kv_heads : 0) + kvh) * HD, j, f);
    have = true;
  }
  // the query heads of the group, as many at a time as the lanes hold
  if (a.q_out) {
    for (int h = part - 2; h < group; h += 32 / J) {
      if (h < 0) continue;
      float q[16];
      load_task<HD>(row + (kvh * group + h) * HD, j, q);
      rotate(q, cs);
      bf16* dst = a.q_out + static_cast<size_t>(req) * (a.n_q_heads * HD) + (kvh * group + h) * HD;
      *reinterpret_cast<uint4*>(dst + j * 8) = pack8(q);
      *reinterpret_cast<uint4*>(dst + HD / 2 + j * 8) = pack8(q + 8);
    }
  }
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.c.n_pages)) {
    if (lane == 0) report(a.err_word);
    return;
  }
  const size_t ph = static_cast<size_t>(page) * a.n_kv_heads + kvh;
  const int off = pos & ((1 << a.c.log2_page) - 1);
  float amax = 0.f;
  if (have) {
    if (part == 0) rotate(f, cs);
    amax = finite_max(f, 0.f);
  }
#pragma unroll
  for (int o = J / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  float* sp = (part == 1 ? a.c.v_scale : a.c.k_scale) + ph;
  const float old = (have && off > 0) ? *sp : 0.f;
  const float s = fmaxf(old, page_scale(amax));
  uint8_t* kp = a.c.k + (ph << a.c.log2_page) * HD;
  uint8_t* vp = a.c.v + (ph << a.c.log2_page) * HD;
  // the page's earlier tokens, when this one needs a larger scale (rare: the scale moves in octaves)
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const float o = __shfl_sync(0xffffffffu, old, kv * J), n = __shfl_sync(0xffffffffu, s, kv * J);
    if (off > 0 && n > o) rescale_rows(kv ? vp : kp, off * HD, o * pow2_inverse(n), lane, 32);
  }
  if (have) {
    store_codes<HD>((part ? vp : kp) + off * HD, j, f, pow2_inverse(s));
    if (j == 0) *sp = s;
  }
}

// ----------------------------------------------------------------------- runs of tokens
constexpr int AP_THREADS = 256;
constexpr int AP_Q_HEADS = 4;  // query heads per block

// The request that owns block `item`: request r owns the blocks floor(cu[r] / P) + 2 r .. floor(cu[r+1] / P) + 2 r + 1, at
// least one more than the pages that its rows can touch, so the host needs no lengths.  All lanes of a warp search
// together, 32 candidates at a time; for up to 32 requests the warp has every request's numbers after one load.
template <int LOG2P>
__device__ __forceinline__ void find_request(const AppendArgs& a, int item, int& req, int& start, int& end, int& pre) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = a.n_req;  // the request lies in lo .. lo + n - 1
  while (n > 32) {
    const int stride = (n + 31) / 32, r = lo + lane * stride;
    const bool at_or_before = lane * stride < n && (a.cu_seqlens[r] >> LOG2P) + 2 * r <= item;
    const int k = 31 - __clz(__ballot_sync(0xffffffffu, at_or_before) | 1u);
    lo += k * stride;
    n = min(stride, n - k * stride);
  }
  const int r = lo + min(lane, n - 1);
  const int c0 = a.cu_seqlens[r], c1 = a.cu_seqlens[r + 1], kv = a.kv_len[r];
  const int k = 31 - __clz(__ballot_sync(0xffffffffu, lane < n && (c0 >> LOG2P) + 2 * r <= item) | 1u);
  req = lo + k;
  start = __shfl_sync(0xffffffffu, c0, k);
  end = __shfl_sync(0xffffffffu, c1, k);
  pre = __shfl_sync(0xffffffffu, kv, k);
}

// Block x is a page of a request, block y a group of query heads or, behind those, the K and V rows of a KV head.  Short
// blocks with a chain of dependent loads in front: all rows of a block are in flight at once, K and V share the chain.
template <int HD, int LOG2P>
__global__ void __launch_bounds__(AP_THREADS) append_pages_kernel(const AppendArgs a) {
  constexpr int P = 1 << LOG2P, J = HD / 16;
  constexpr int NT = (P * J + AP_THREADS - 1) / AP_THREADS;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int item = blockIdx.x;
  int req, start, stop, pre;
  find_request<LOG2P>(a, item, req, start, stop, pre);
  const int len = min(stop, a.n_tokens) - start;
  if (len <= 0 || pre < 0) return;
  const int pi = (pre >> LOG2P) + item - ((start >> LOG2P) + 2 * req);
  // positions of this page that the call fills, as far as the rotation table goes
  const int total = static_cast<int>(min(static_cast<long long>(pre) + len, 0x7fffffffll));
  const long long page_pos = static_cast<long long>(pi) << LOG2P;
  const int p0 = static_cast<int>(max(static_cast<long long>(pre), page_pos));
  const int p1 = static_cast<int>(min(static_cast<long long>(min(total, a.max_pos)), page_pos + P));
  if (total > a.max_pos && threadIdx.x == 0) report(a.err_word);
  const int n_rows = p1 - p0;
  if (n_rows <= 0) return;
  const int tasks = n_rows * J;
  const int row0 = start + (p0 - pre);
  const int q_blocks = gridDim.y - a.n_kv_heads;

  if (static_cast<int>(blockIdx.y) < q_blocks) {
    // ------------------------------------------------------------------ query heads
    const int h0 = blockIdx.y * AP_Q_HEADS, n_h = min(AP_Q_HEADS, a.n_q_heads - h0);
    for (int t = threadIdx.x; t < tasks; t += AP_THREADS) {
      const int r = t / J, j = t % J;
      const bf16* src = a.qkv + static_cast<size_t>(row0 + r) * a.ldqkv + h0 * HD;
      bf16* dst = a.q_out + static_cast<size_t>(row0 + r) * (a.n_q_heads * HD) + h0 * HD;
      uint4 w[AP_Q_HEADS][2];
#pragma unroll
      for (int h = 0; h < AP_Q_HEADS; ++h) {
        if (h < n_h) {
          w[h][0] = *reinterpret_cast<const uint4*>(src + h * HD + j * 8);
          w[h][1] = *reinterpret_cast<const uint4*>(src + h * HD + HD / 2 + j * 8);
        }
      }
      float cs[16];
      load_angles(a.rope + static_cast<size_t>(p0 + r) * (HD / 2), j, cs);
#pragma unroll
      for (int h = 0; h < AP_Q_HEADS; ++h) {
        if (h < n_h) {
          float q[16];
          unpack8(w[h][0], q);
          unpack8(w[h][1], q + 8);
          rotate(q, cs);
          *reinterpret_cast<uint4*>(dst + h * HD + j * 8) = pack8(q);
          *reinterpret_cast<uint4*>(dst + h * HD + HD / 2 + j * 8) = pack8(q + 8);
        }
      }
    }
    return;
  }
  const int kvh = blockIdx.y - q_blocks;
  const int page = pi < a.c.table_ld ? a.c.table[static_cast<size_t>(req) * a.c.table_ld + pi] : -1;
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.c.n_pages)) {
    if (threadIdx.x == 0) report(a.err_word);
    return;
  }
  const size_t ph = static_cast<size_t>(page) * a.n_kv_heads + kvh;
  const int off = p0 & (P - 1);
  const float old_k = off > 0 ? a.c.k_scale[ph] : 0.f, old_v = off > 0 ? a.c.v_scale[ph] : 0.f;
  float k[NT][16];
  uint4 v[NT][2];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = threadIdx.x + i * AP_THREADS;
    if (t < tasks) {
      const bf16* src = a.qkv + static_cast<size_t>(row0 + t / J) * a.ldqkv + (a.n_q_heads + kvh) * HD + (t % J) * 8;
      unpack8(*reinterpret_cast<const uint4*>(src), k[i]);
      unpack8(*reinterpret_cast<const uint4*>(src + HD / 2), k[i] + 8);
      v[i][0] = *reinterpret_cast<const uint4*>(src + a.n_kv_heads * HD);
      v[i][1] = *reinterpret_cast<const uint4*>(src + a.n_kv_heads * HD + HD / 2);
    }
  }
  float amax_k = 0.f, amax_v = 0.f;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = threadIdx.x + i * AP_THREADS;
    if (t < tasks) {
      float cs[16], f[16];
      load_angles(a.rope + static_cast<size_t>(p0 + t / J) * (HD / 2), t % J, cs);
      rotate(k[i], cs);
      amax_k = finite_max(k[i], amax_k);
      unpack8(v[i][0], f);
      unpack8(v[i][1], f + 8);
      amax_v = finite_max(f, amax_v);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    amax_k = fmaxf(amax_k, __shfl_xor_sync(0xffffffffu, amax_k, o));
    amax_v = fmaxf(amax_v, __shfl_xor_sync(0xffffffffu, amax_v, o));
  }
  __shared__ float2 red[AP_THREADS / 32];
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(amax_k, amax_v);
  __syncthreads();  // (also: every thread has read the old scales)
#pragma unroll
  for (int w = 0; w < AP_THREADS / 32; ++w) {
    amax_k = fmaxf(amax_k, red[w].x);
    amax_v = fmaxf(amax_v, red[w].y);
  }
  const float s_k = fmaxf(old_k, page_scale(amax_k)), s_v = fmaxf(old_v, page_scale(amax_v));
  uint8_t* base_k = a.c.k + (ph << LOG2P) * HD;
  uint8_t* base_v = a.c.v + (ph << LOG2P) * HD;
  if (off > 0 && s_k > old_k) rescale_rows(base_k, off * HD, old_k * pow2_inverse(s_k), threadIdx.x, AP_THREADS);
  if (off > 0 && s_v > old_v) rescale_rows(base_v, off * HD, old_v * pow2_inverse(s_v), threadIdx.x, AP_THREADS);
  const float inv_k = pow2_inverse(s_k), inv_v = pow2_inverse(s_v);
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = threadIdx.x + i * AP_THREADS;
    if (t < tasks) {
      float f[16];
      unpack8(v[i][0], f);
      unpack8(v[i][1], f + 8);
      finite_max(f, 0.f);
      store_codes<HD>(base_k + (off + t / J) * HD, t % J, k[i], inv_k);
      store_codes<HD>(base_v + (off + t / J) * HD, t % J, f, inv_v);
    }
  }
  if (threadIdx.x == 0) { a.c.k_scale[ph] = s_k; a.c.v_scale[ph] = s_v; }
}

template <int HD, int LOG2P>
cudaError_t launch_pages(const AppendArgs& a, cudaStream_t s) {
  const dim3 grid((a.n_tokens >> LOG2P) + 2 * a.n_req,
                  a.n_kv_heads + (a.q_out ? (a.n_q_heads + AP_Q_HEADS - 1) / AP_Q_HEADS : 0));
  return launch_pdl(append_pages_kernel<HD, LOG2P>, grid, dim3(AP_THREADS), 0, s, a);
}

template <int HD>
cudaError_t launch(const AppendArgs& a, cudaStream_t s) {
  if (!a.cu_seqlens) {
    const int items = a.n_req * a.n_kv_heads;
    return launch_pdl(append_decode_kernel<HD>, dim3((items + AD_WARPS - 1) / AD_WARPS), dim3(AD_WARPS * 32), 0, s, a);
  }
  switch (a.c.log2_page) {
    case 4: return launch_pages<HD, 4>(a, s);
    case 5: return launch_pages<HD, 5>(a, s);
    case 6: return launch_pages<HD, 6>(a, s);
    default: return launch_pages<HD, 7>(a, s);
  }
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_paged_kv_append(const pd_layer_cfg* cfg, const void* qkv, int32_t ldqkv, void* q_out,
                                        const float* rope_tab, const int32_t* cu_dev, const int32_t* cu_host, int32_t n_req,
                                        const int32_t* kv_len_dev, const pd_paged_kv_cache* cache, int32_t* err_word,
                                        void* stream) {
  using namespace pd;
  PD_TRY(check_paged_heads(cfg));
  AppendArgs a{};
  PD_TRY(paged_cache_view(cache, &a.c));
  if (n_req < 0 || n_req > cache->n_seqs || (cu_dev == nullptr) != (cu_host == nullptr) || cfg->max_pos <= 0)
    return PD_ERR_INVALID_ARG;
  int tokens = n_req;
  if (cu_host) {
    if (n_req > (1 << 20)) return PD_ERR_UNSUPPORTED_SHAPE;
    if (cu_host[0] != 0) return PD_ERR_INVALID_ARG;
    for (int r = 0; r < n_req; ++r)
      if (cu_host[r + 1] < cu_host[r]) return PD_ERR_INVALID_ARG;
    tokens = cu_host[n_req];
  }
  if (tokens == 0) return PD_OK;
  const int width = (cfg->n_q_heads + 2 * cfg->n_kv_heads) * cfg->head_dim;
  if (!qkv || !rope_tab || !kv_len_dev || ldqkv < width || ldqkv % 8 != 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(qkv) | reinterpret_cast<uintptr_t>(q_out) | reinterpret_cast<uintptr_t>(rope_tab)) & 15u)
    return PD_ERR_INVALID_ARG;
  if (1ll * tokens * cfg->n_kv_heads > 0x7fffffffll) return PD_ERR_UNSUPPORTED_SHAPE;
  a.qkv = static_cast<const bf16*>(qkv); a.q_out = static_cast<bf16*>(q_out);
  a.rope = reinterpret_cast<const float2*>(rope_tab);
  a.cu_seqlens = cu_dev; a.kv_len = kv_len_dev; a.err_word = err_word;
  a.ldqkv = ldqkv; a.n_req = n_req; a.n_tokens = tokens;
  a.n_q_heads = cfg->n_q_heads; a.n_kv_heads = cfg->n_kv_heads; a.max_pos = cfg->max_pos;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_KV_APPEND, st);
  PD_CUDA_TRY(cfg->head_dim == 128 ? launch<128>(a, st) : launch<64>(a, st));
  count_launch();
  return PD_OK;
}
