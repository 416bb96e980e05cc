// Attention over the 8-bit paged KV cache: one query token per sequence (pd_paged_decode_attention) and the fresh rows of
// ragged requests (pd_paged_prefill_attention).
//
// Decode.  o = softmax(q K^T / sqrt(hd)) V per query head over the sequence's pages; K and V of a page are E4M3 codes times
// one power of two.  HBM-bound: every code byte is read once.  One block per (split of the key range, KV head, sequence);
// every warp streams its own 16-key tiles through a private cp.async ring (a tile never crosses a page, so it has one page
// number and one pair of scales).
//   S = Q K^T   m16n8k16 in f16: rows are the query heads of the group, columns 8 keys.
//   O^T = V^T P^T   m16n8k16: rows are features, columns 8 heads, so a group of at most 8 heads wastes no product, and the
//               accumulator fragment of S is already the operand fragment of P^T.
// E4M3 -> f16 is exact and one instruction for two codes.  The contraction order of a product is free, so a lane takes 16
// neighbouring features of a K row as its share of four k-steps, and 16 neighbouring features of four V rows (byte-permuted
// into pairs of keys): all shared-memory reads are 16 bytes wide, and the row order within a group of 8 keys is chosen so
// that they are free of bank conflicts.  q is scaled by a power of two per head into f16 range, p = 2^(s - m + 14) keeps
// 11 significant bits down to 2^-28 of the largest; the softmax statistics and O are fp32, the page scales are applied in
// fp32 (K: to the scores; V: to the tile's product).
#include <math_constants.h>

#include "pd_paged.cuh"

namespace pd {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

struct PagedDecodeArgs {
  const bf16* q;          // [B, ldq]
  bf16* o;                // [B, Hq*hd]
  const int32_t* kv_len;  // [B]
  float* partial;         // [B, Hkv, n_splits, G, hd + 2] when n_splits > 1
  int* err_word;
  PagedCache c;
  int ldq, batch, n_splits, n_q_heads, n_kv_heads;
};

constexpr int PA_WARPS = 4;
constexpr int PA_THREADS = PA_WARPS * 32;
constexpr int PA_KEYS = 16;
constexpr int PA_STAGES = 4;
constexpr float P_SHIFT = 14.f;                 // p is kept as 2^14 p
constexpr float P_UNIT = 1.f / 16384.f;

template <int HD>
struct PagedSmem {
  static constexpr int TILE = PA_KEYS * HD;                  // one K (or V) tile
  static constexpr int RING = PA_WARPS * PA_STAGES * 2 * TILE;
  static constexpr int SCALES = RING;                        // float2 per warp and stage
  static constexpr int MERGE = PA_WARPS * 16 * (HD + 2) * 4;
  static constexpr int BYTES = (RING + PA_WARPS * PA_STAGES * 8) > MERGE ? (RING + PA_WARPS * PA_STAGES * 8) : MERGE;
};

// Key that column n of an 8-key group holds, and the 16-byte chunk swizzle of row r.  hd 128: a row fills all banks; eight
// lanes read two K rows (chunks t, t + 4 of lanes t = 0..3) or two V chunks of four rows at a time.  hd 64: two rows share
// the banks.
template <int HD>
__device__ __forceinline__ int key_of(int n) {
  if (HD == 128) return (n & 1) ? (((n & 6) ^ 4) | 1) : n;  // 0 5 2 7 4 1 6 3
  return n ^ ((n >> 1) & 1);                                // 0 1 3 2 4 5 7 6
}
template <int HD>
__device__ __forceinline__ uint32_t chunk_off(int r, int c) {
  const int x = HD == 128 ? (r & 7) : ((r >> 2) & 1) * 2;
  return static_cast<uint32_t>(r * HD + ((c ^ x) << 4));
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}

// WIDE: groups of 9 to 16 query heads (two column groups in the second product).
template <int HD, bool WIDE>
__global__ void __launch_bounds__(PA_THREADS, WIDE ? 2 : 3) paged_decode_kernel(const PagedDecodeArgs a) {
  using SM = PagedSmem<HD>;
  constexpr int CPR = HD / 16;         // 16-byte chunks per row
  constexpr int KS = HD / 16;          // k-steps of Q K^T
  constexpr int MT = HD / 16;          // 16-feature tiles of O^T
  constexpr int NR = WIDE ? 2 : 1;     // rows (heads) per lane of S, column groups of O^T
  extern __shared__ __align__(128) uint8_t smem[];
  const int split = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, t4 = lane & 3;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();

  const int l2p = a.c.log2_page;
  const int cap = a.c.table_ld << l2p;
  const int len = a.kv_len[b];
  if (len >= cap && split == 0 && kvh == 0 && tid == 0 && a.err_word) atomicExch(a.err_word, 2);
  const int total = len >= cap ? cap : len + 1;  // <= 0: no entry
  constexpr int STEP = PA_WARPS * PA_KEYS;
  const int steps = total > 0 ? (total + STEP - 1) / STEP : 0;
  const int per_split = (steps + a.n_splits - 1) / a.n_splits * STEP;
  const int k_begin = static_cast<int>(min(static_cast<long long>(max(total, 0)), 1ll * split * per_split));
  const int k_end = static_cast<int>(min(static_cast<long long>(max(total, 0)), 1ll * k_begin + per_split));

  const int n_tiles_blk = (k_end - k_begin + PA_KEYS - 1) / PA_KEYS;
  const int my_tiles = (n_tiles_blk > warp) ? (n_tiles_blk - warp + PA_WARPS - 1) / PA_WARPS : 0;
  const int32_t* table = a.c.table + static_cast<size_t>(b) * a.c.table_ld;
  const uint32_t ring = ptx::smem_u32(smem) + warp * (PA_STAGES * 2 * SM::TILE);
  float2* scales = reinterpret_cast<float2*>(smem + SM::SCALES) + warp * PA_STAGES;

  // Page numbers and scales of 32 tiles at a time, one tile per lane; the next 32 are fetched ahead.
  auto fetch_pages = [&](int first, int& id, float& ks, float& vs) {
    const int i = first + lane;
    id = -1; ks = -1.f; vs = 0.f;
    if (i < my_tiles) {
      id = table[(k_begin + (i * PA_WARPS + warp) * PA_KEYS) >> l2p];
      if (static_cast<unsigned>(id) < static_cast<unsigned>(a.c.n_pages)) {
        ks = a.c.k_scale[static_cast<size_t>(id) * a.n_kv_heads + kvh];
        vs = a.c.v_scale[static_cast<size_t>(id) * a.n_kv_heads + kvh];
      } else {
        id = -1;  // no such page: its keys are left out
        if (a.err_word) atomicExch(a.err_word, 2);
      }
    }
  };
  int id_cur, id_nxt = -1;
  float ks_cur, vs_cur, ks_nxt = -1.f, vs_nxt = 0.f;
  fetch_pages(0, id_cur, ks_cur, vs_cur);
  if (my_tiles > 32) fetch_pages(32, id_nxt, ks_nxt, vs_nxt);

  auto load_tile = [&](int i, int stage) {
    if (i > 0 && (i & 31) == 0) {
      id_cur = id_nxt; ks_cur = ks_nxt; vs_cur = vs_nxt;
      if (i + 32 < my_tiles) fetch_pages(i + 32, id_nxt, ks_nxt, vs_nxt);
    }
    const int id = __shfl_sync(0xffffffffu, id_cur, i & 31);
    const float ks = __shfl_sync(0xffffffffu, ks_cur, i & 31), vs = __shfl_sync(0xffffffffu, vs_cur, i & 31);
    if (lane == 0) scales[stage] = make_float2(ks, vs * P_UNIT);
    const int key0 = k_begin + (i * PA_WARPS + warp) * PA_KEYS;
    const int row0 = key0 & ((1 << l2p) - 1);
    const size_t base = (((static_cast<size_t>(max(id, 0)) * a.n_kv_heads + kvh) << l2p) + row0) * HD;
    const uint32_t sk = ring + stage * 2 * SM::TILE, sv = sk + SM::TILE;
#pragma unroll
    for (int j = lane; j < PA_KEYS * CPR; j += 32) {
      const int r = j / CPR, c = j % CPR;
      const bool ok = id >= 0 && key0 + r < k_end;  // rows past the end become zeros: whatever they hold is not read
      const size_t off = ok ? base + r * HD + c * 16 : base;
      ptx::cp_async_16(sk + chunk_off<HD>(r, c), a.c.k + off, ok);
      ptx::cp_async_16(sv + chunk_off<HD>(r, c), a.c.v + off, ok);
    }
  };
#pragma unroll
  for (int s = 0; s < PA_STAGES - 1; ++s) {
    if (s < my_tiles) load_tile(s, s);
    ptx::cp_async_commit();
  }

  // Q as f16 operand fragments, every head scaled by a power of two so that its largest entry lies in [1, 2)
  uint32_t qa[KS][2 * NR];
  float row_scale[NR];  // of the scores of this lane's heads, in log2 units
#pragma unroll
  for (int rr = 0; rr < NR; ++rr) {
    const int r = g + rr * 8;
    float f[KS * 4];
    float amax = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      uint2 w = make_uint2(0u, 0u);
      if (r < group)
        w = *reinterpret_cast<const uint2*>(a.q + static_cast<size_t>(b) * a.ldq + (kvh * group + r) * HD + (s >> 2) * 64 +
                                            t4 * 16 + (s & 3) * 4);
      f[4 * s] = ptx::bf16_lo(w.x); f[4 * s + 1] = ptx::bf16_hi(w.x);
      f[4 * s + 2] = ptx::bf16_lo(w.y); f[4 * s + 3] = ptx::bf16_hi(w.y);
#pragma unroll
      for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fabsf(f[4 * s + e]));
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    // 2^e <= amax < 2^(e+1), e kept where 2^e and 2^-e are normal (an infinite q stays infinite)
    const int e = min(max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -126), 126);
    const float up = __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
    const float inv = pow2_inverse(up);
    row_scale[rr] = rsqrtf(static_cast<float>(HD)) * LOG2E * up;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qa[s][2 * rr] = pack_f16(f[4 * s] * inv, f[4 * s + 1] * inv);
      qa[s][2 * rr + 1] = pack_f16(f[4 * s + 2] * inv, f[4 * s + 3] * inv);
    }
  }

  float o_acc[NR][MT][4];
#pragma unroll
  for (int rr = 0; rr < NR; ++rr)
#pragma unroll
    for (int i = 0; i < MT; ++i) o_acc[rr][i][0] = o_acc[rr][i][1] = o_acc[rr][i][2] = o_acc[rr][i][3] = 0.f;
  float m_row[NR], l_row[NR];
#pragma unroll
  for (int rr = 0; rr < NR; ++rr) { m_row[rr] = -CUDART_INF_F; l_row[rr] = 0.f; }

  for (int i = 0; i < my_tiles; ++i) {
    const int stage = i % PA_STAGES;
    {
      const int nxt = i + PA_STAGES - 1;
      if (nxt < my_tiles) load_tile(nxt, nxt % PA_STAGES);
      ptx::cp_async_commit();
    }
    ptx::cp_async_wait<PA_STAGES - 1>();
    __syncwarp();
    const uint32_t sk = ring + stage * 2 * SM::TILE, sv = sk + SM::TILE;
    const float2 sc = scales[stage];
    const int key0 = k_begin + (i * PA_WARPS + warp) * PA_KEYS;

    // ---- S: two column groups of 8 keys
    float s_acc[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      s_acc[nt][0] = s_acc[nt][1] = s_acc[nt][2] = s_acc[nt][3] = 0.f;
#pragma unroll
      for (int h = 0; h < HD / 64; ++h) {
        const uint4 w = lds128(sk + chunk_off<HD>(nt * 8 + key_of<HD>(g), h * 4 + t4));
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t b0 = e4m3x2_to_f16x2(static_cast<uint16_t>(ww[q]));
          const uint32_t b1 = e4m3x2_to_f16x2(static_cast<uint16_t>(ww[q] >> 16));
          const int s = h * 4 + q;
          mma_f16(s_acc[nt], qa[s][0], WIDE ? qa[s][2 * NR - 2] : 0u, qa[s][1], WIDE ? qa[s][2 * NR - 1] : 0u, b0, b1);
        }
      }
    }
    // ---- online softmax; rows of S are heads
    const bool masked = key0 + PA_KEYS > k_end || sc.x < 0.f;
    uint32_t pb[NR][2];
    float corr[NR];
    bool moved = false;
#pragma unroll
    for (int rr = 0; rr < NR; ++rr) {
      const float f = row_scale[rr] * sc.x;
      float v[4] = {s_acc[0][2 * rr] * f, s_acc[0][2 * rr + 1] * f, s_acc[1][2 * rr] * f, s_acc[1][2 * rr + 1] * f};
      if (masked) {
        const int lim = sc.x < 0.f ? -1 : k_end - 1 - key0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((e >> 1) * 8 + key_of<HD>(t4 * 2 + (e & 1)) > lim) v[e] = -CUDART_INF_F;
      }
      float mx = ptx::fmax3(fmaxf(v[0], v[1]), v[2], v[3]);
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const float m_new = fmaxf(m_row[rr], mx);
      const float m_use = m_new == -CUDART_INF_F ? 0.f : m_new;  // nothing seen yet: every p below is 0
      corr[rr] = ptx::ex2_approx(m_row[rr] - m_use);
      moved |= m_new != m_row[rr];
      m_row[rr] = m_new;
      const float ref = m_use - P_SHIFT;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = ptx::ex2_approx(v[e] - ref);
      l_row[rr] = l_row[rr] * corr[rr] + ((v[0] + v[1]) + (v[2] + v[3]));
      pb[rr][0] = pack_f16(v[0], v[1]);
      pb[rr][1] = pack_f16(v[2], v[3]);
    }
    if (__any_sync(0xffffffffu, moved)) {
      // columns of O^T are heads: fetch their corrections from the lanes that hold the rows
#pragma unroll
      for (int rr = 0; rr < NR; ++rr) {
        const float c0 = __shfl_sync(0xffffffffu, corr[rr], t4 * 8), c1 = __shfl_sync(0xffffffffu, corr[rr], t4 * 8 + 4);
#pragma unroll
        for (int n = 0; n < MT; ++n) {
          o_acc[rr][n][0] *= c0; o_acc[rr][n][1] *= c1;
          o_acc[rr][n][2] *= c0; o_acc[rr][n][3] *= c1;
        }
      }
    }
    // ---- O^T += V^T P^T: this lane's keys are columns 2 t4, 2 t4 + 1 of both groups, its features g * hd/8 ...
    uint32_t vw[4][HD / 32];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = (r >> 1) * 8 + key_of<HD>(t4 * 2 + (r & 1));
      if (HD == 128) {
        const uint4 w = lds128(sv + chunk_off<HD>(row, g));
        vw[r][0] = w.x; vw[r][1] = w.y; vw[r][HD / 32 - 2] = w.z; vw[r][HD / 32 - 1] = w.w;
      } else {
        const uint2 w = lds64(sv + chunk_off<HD>(row, g >> 1) + (g & 1) * 8);
        vw[r][0] = w.x; vw[r][1] = w.y;
      }
    }
#pragma unroll
    for (int w = 0; w < HD / 32; ++w) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // features 4 w + 2 h, 4 w + 2 h + 1
        const uint32_t sel = h ? 0x7362u : 0x5140u;
        const uint32_t x = __byte_perm(vw[0][w], vw[1][w], sel), y = __byte_perm(vw[2][w], vw[3][w], sel);
        const uint32_t a0 = e4m3x2_to_f16x2(static_cast<uint16_t>(x)), a1 = e4m3x2_to_f16x2(static_cast<uint16_t>(x >> 16));
        const uint32_t a2 = e4m3x2_to_f16x2(static_cast<uint16_t>(y)), a3 = e4m3x2_to_f16x2(static_cast<uint16_t>(y >> 16));
#pragma unroll
        for (int rr = 0; rr < NR; ++rr) {
          float f[4] = {0.f, 0.f, 0.f, 0.f};
          mma_f16(f, a0, a1, a2, a3, pb[rr][0], pb[rr][1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) o_acc[rr][2 * w + h][e] = fmaf(f[e], sc.y, o_acc[rr][2 * w + h][e]);
        }
      }
    }
    __syncwarp();  // every lane has read this stage before it is refilled
  }
  ptx::cp_async_wait<0>();
#pragma unroll
  for (int rr = 0; rr < NR; ++rr) {
    l_row[rr] += __shfl_xor_sync(0xffffffffu, l_row[rr], 1);
    l_row[rr] += __shfl_xor_sync(0xffffffffu, l_row[rr], 2);
  }
  __syncthreads();  // every warp has left its ring: the memory is reused for the merge

  float* mrg = reinterpret_cast<float*>(smem);
  constexpr int RS = HD + 2;
#pragma unroll
  for (int rr = 0; rr < NR; ++rr) {
#pragma unroll
    for (int n = 0; n < MT; ++n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int head = rr * 8 + t4 * 2 + (e & 1), d = g * (HD / 8) + 2 * n + (e >> 1);
        if (head < group) mrg[(warp * 16 + head) * RS + d] = o_acc[rr][n][e];
      }
    }
    if (t4 == 0 && g + rr * 8 < group) {
      mrg[(warp * 16 + g + rr * 8) * RS + HD] = m_row[rr];
      mrg[(warp * 16 + g + rr * 8) * RS + HD + 1] = l_row[rr] * P_UNIT;
    }
  }
  __syncthreads();
  for (int idx = tid; idx < group * HD; idx += PA_THREADS) {
    const int r = idx / HD, d = idx - r * HD;
    float m = -CUDART_INF_F;
#pragma unroll
    for (int w = 0; w < PA_WARPS; ++w) m = fmaxf(m, mrg[(w * 16 + r) * RS + HD]);
    const float m_use = m == -CUDART_INF_F ? 0.f : m;
    float l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < PA_WARPS; ++w) {
      const float* src = mrg + (w * 16 + r) * RS;
      const float f = exp2f(src[HD] - m_use);  // 0 for a warp that saw no key
      l += src[HD + 1] * f;
      o += src[d] * f;
    }
    if (a.n_splits == 1) {
      // no visible entry: zeros
      a.o[static_cast<size_t>(b) * (a.n_q_heads * HD) + (kvh * group + r) * HD + d] = __float2bfloat16(l == 0.f ? 0.f : o / l);
    } else {
      float* dst = a.partial + (((static_cast<size_t>(b) * a.n_kv_heads + kvh) * a.n_splits + split) * group + r) * RS;
      dst[d] = o;
      if (d == 0) { dst[HD] = m; dst[HD + 1] = l; }
    }
  }
}

// Merge of the splits: one block per (query head, sequence), one thread per feature.
template <int HD>
__global__ void __launch_bounds__(HD) paged_combine_kernel(const PagedDecodeArgs a) {
  constexpr int RS = HD + 2;
  const int b = blockIdx.y, hq = blockIdx.x, d = threadIdx.x;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int kvh = hq / group, r = hq - kvh * group;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const float* base = a.partial + ((static_cast<size_t>(b) * a.n_kv_heads + kvh) * a.n_splits * group + r) * RS;
  const size_t pitch = static_cast<size_t>(group) * RS;
  float m = -CUDART_INF_F;
  for (int s = 0; s < a.n_splits; ++s) m = fmaxf(m, base[s * pitch + HD]);
  const float m_use = m == -CUDART_INF_F ? 0.f : m;
  float l = 0.f, o = 0.f;
#pragma unroll 4
  for (int s = 0; s < a.n_splits; ++s) {
    const float f = exp2f(base[s * pitch + HD] - m_use);  // 0 for an empty split
    l += base[s * pitch + HD + 1] * f;
    o += base[s * pitch + d] * f;
  }
  a.o[static_cast<size_t>(b) * (a.n_q_heads * HD) + hq * HD + d] = __float2bfloat16(l == 0.f ? 0.f : o / l);
}

template <int HD, bool WIDE>
pd_status launch_decode(const PagedDecodeArgs& a, cudaStream_t s) {
  using SM = PagedSmem<HD>;
  static PerDeviceInt smem_opt_in;
  PD_TRY(opt_in_smem(smem_opt_in, paged_decode_kernel<HD, WIDE>, SM::BYTES));
  PD_CUDA_TRY(launch_pdl(paged_decode_kernel<HD, WIDE>, dim3(a.n_splits, a.n_kv_heads, a.batch), dim3(PA_THREADS), SM::BYTES, s, a));
  count_launch();
  if (a.n_splits > 1) {
    PD_CUDA_TRY(launch_pdl(paged_combine_kernel<HD>, dim3(a.n_q_heads, a.batch), dim3(HD), 0, s, a));
    count_launch();
  }
  return PD_OK;
}

// About three blocks per SM are resident; the key range is split until that many exist, into runs of at least 256 keys,
// and a run is at most about 4096 keys, so that one long sequence of a ragged batch does not run on alone.
int paged_decode_splits(int batch, int n_kv_heads, int max_kv_len) {
  const long long blocks = 1ll * batch * n_kv_heads;
  if (blocks <= 0) return 1;
  long long want = (444 + blocks - 1) / blocks;
  const long long by_len = (max_kv_len + 2047ll) / 4096;
  if (by_len > want) want = by_len;
  long long most = max_kv_len / 256;
  if (most < 1) most = 1;
  if (want > most) want = most;
  return static_cast<int>(want > 64 ? 64 : want);
}

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

size_t prefill_scratch_half(const pd_layer_cfg* cfg, int n_req, int max_kv_len) {
  return align_up(static_cast<size_t>(n_req) * cfg->n_kv_heads * max_kv_len * cfg->head_dim * sizeof(bf16), 256);
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_paged_decode_attention_workspace_bytes(const pd_layer_cfg* cfg, int32_t B, int32_t max_kv_len,
                                                               size_t* out_bytes) {
  PD_TRY(pd::check_paged_heads(cfg));
  if (!out_bytes || B < 0 || max_kv_len < 0) return PD_ERR_INVALID_ARG;
  const int splits = pd::paged_decode_splits(B, cfg->n_kv_heads, max_kv_len);
  *out_bytes = splits > 1 ? pd::align_up(static_cast<size_t>(B) * cfg->n_q_heads * splits * (cfg->head_dim + 2) * 4, 256) : 0;
  return PD_OK;
}

extern "C" pd_status pd_paged_decode_attention(const pd_layer_cfg* cfg, const void* q, int32_t ldq, void* out,
                                               const int32_t* kv_len_dev, int32_t B, int32_t max_kv_len,
                                               const pd_paged_kv_cache* cache, void* workspace, size_t workspace_bytes,
                                               int32_t* err_word, void* stream) {
  using namespace pd;
  PD_TRY(check_paged_heads(cfg));
  PagedDecodeArgs a{};
  PD_TRY(paged_cache_view(cache, &a.c));
  if (B < 0 || B > cache->n_seqs) return PD_ERR_INVALID_ARG;
  if (B > 65535) return PD_ERR_UNSUPPORTED_SHAPE;
  if (B == 0) return PD_OK;
  if (!q || !out || !kv_len_dev || ldq < cfg->n_q_heads * cfg->head_dim || ldq % 8 != 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) & 15u) || (reinterpret_cast<uintptr_t>(out) & 1u)) return PD_ERR_INVALID_ARG;
  if (max_kv_len <= 0 || max_kv_len > (cache->table_ld << a.c.log2_page)) return PD_ERR_INVALID_ARG;
  a.n_splits = paged_decode_splits(B, cfg->n_kv_heads, max_kv_len);
  if (a.n_splits > 1) {
    size_t need = 0;
    PD_TRY(pd_paged_decode_attention_workspace_bytes(cfg, B, max_kv_len, &need));
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PD_ERR_INVALID_ARG;
    if (workspace_bytes < need) return PD_ERR_WORKSPACE_TOO_SMALL;
  }
  a.q = static_cast<const bf16*>(q); a.o = static_cast<bf16*>(out); a.kv_len = kv_len_dev;
  a.partial = static_cast<float*>(workspace); a.err_word = err_word;
  a.ldq = ldq; a.batch = B; a.n_q_heads = cfg->n_q_heads; a.n_kv_heads = cfg->n_kv_heads;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_ATTN_DECODE, st);
  const bool wide = cfg->n_q_heads / cfg->n_kv_heads > 8;
  if (cfg->head_dim == 128) return wide ? launch_decode<128, true>(a, st) : launch_decode<128, false>(a, st);
  return wide ? launch_decode<64, true>(a, st) : launch_decode<64, false>(a, st);
}

extern "C" pd_status pd_paged_prefill_attention_workspace_bytes(const pd_layer_cfg* cfg, int32_t n_req, int32_t max_kv_len,
                                                                size_t* out_bytes) {
  PD_TRY(pd::check_paged_heads(cfg));
  if (!out_bytes || n_req < 0 || max_kv_len < 0) return PD_ERR_INVALID_ARG;
  *out_bytes = 2 * pd::prefill_scratch_half(cfg, n_req, max_kv_len);
  return PD_OK;
}

extern "C" pd_status pd_paged_prefill_attention(const pd_layer_cfg* cfg, const void* q, int32_t ldq, void* out,
                                                const int32_t* cu_dev, const int32_t* cu_host, int32_t n_req,
                                                const int32_t* prefix_dev, const int32_t* prefix_host,
                                                const pd_paged_kv_cache* cache, void* workspace, size_t workspace_bytes,
                                                int32_t* err_word, void* stream) {
  using namespace pd;
  PD_TRY(check_paged_heads(cfg));
  GatherArgs ga{};
  PD_TRY(paged_cache_view(cache, &ga.c));
  if (!cu_host || n_req < 0 || n_req > 4095 || n_req > cache->n_seqs || (prefix_dev == nullptr) != (prefix_host == nullptr))
    return PD_ERR_INVALID_ARG;
  if (cu_host[0] != 0) return PD_ERR_INVALID_ARG;
  const int cap = cache->table_ld << ga.c.log2_page;
  int max_len = 0, max_kv = 0;
  for (int r = 0; r < n_req; ++r) {
    const long long len = 1ll * cu_host[r + 1] - cu_host[r];
    const int pre = prefix_host ? prefix_host[r] : 0;
    if (len < 0 || pre < 0 || pre + len > cap) return PD_ERR_INVALID_ARG;
    if (len > max_len) max_len = static_cast<int>(len);
    if (len > 0 && pre + len > max_kv) max_kv = static_cast<int>(pre + len);
  }
  const int tokens = cu_host[n_req];
  if (tokens == 0) return PD_OK;
  if (!q || !out || !cu_dev || ldq < cfg->n_q_heads * cfg->head_dim || ldq % 8 != 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) & 15u) || (reinterpret_cast<uintptr_t>(out) & 31u)) return PD_ERR_INVALID_ARG;
  const size_t half = prefill_scratch_half(cfg, n_req, max_kv);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PD_ERR_INVALID_ARG;
  if (workspace_bytes < 2 * half) return PD_ERR_WORKSPACE_TOO_SMALL;
  // cache rows are addressed with 32-bit row numbers
  if (1ll * n_req * cfg->n_kv_heads * max_kv > 0x7fffffffll - 256) return PD_ERR_UNSUPPORTED_SHAPE;
  ga.k = static_cast<bf16*>(workspace);
  ga.v = reinterpret_cast<bf16*>(static_cast<uint8_t*>(workspace) + half);
  ga.cu_seqlens = cu_dev; ga.prefix = prefix_dev; ga.err_word = err_word;
  ga.n_kv_heads = cfg->n_kv_heads; ga.head_dim = cfg->head_dim; ga.len_cap = max_kv;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_ATTN_PREFILL, st);
  const int pages = (max_kv + (1 << ga.c.log2_page) - 1) >> ga.c.log2_page;
  PD_CUDA_TRY(launch_pdl(gather_pages_kernel, dim3(pages, cfg->n_kv_heads, n_req), dim3(256), 0, st, ga));
  count_launch();
  PrefillAttnArgs a{};
  a.q = static_cast<const bf16*>(q); a.ldq = ldq;
  a.k_cache = ga.k; a.v_cache = ga.v;
  a.o = static_cast<bf16*>(out); a.cu_seqlens = cu_dev; a.prefix = prefix_dev;
  a.n_req = n_req; a.n_tokens = tokens; a.max_len = max_len;
  a.n_q_heads = cfg->n_q_heads; a.n_kv_heads = cfg->n_kv_heads; a.head_dim = cfg->head_dim;
  a.len_cap = max_kv; a.batch_cap = n_req;
  return launch_prefill_attention_tc(a, err_word, st);
}
