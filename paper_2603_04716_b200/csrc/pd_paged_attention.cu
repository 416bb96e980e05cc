// Attention over the 8-bit paged KV cache for few query rows: one token per sequence (pd_paged_decode_attention) or short runs
// of tokens (one of the kernels behind pd_paged_prefill_attention).
//
// o = softmax(q K^T / sqrt(hd)) V per query head over the sequence's pages; K and V of a page are E4M3 codes times
// one power of two.  HBM-bound: every code byte is read once (by every block of tokens of a run).  One block per (part of the
// key range, KV head, sequence or block of tokens); every warp streams its own 16-key tiles through a private cp.async ring (a
// tile never crosses a page, so it has one page number and one pair of scales).
//   S^T = K Q^T    m16n8k16 in f16: rows are 16 keys, columns 8 (token, head of the group) pairs.
//   O^T = V^T P^T  m16n8k16: rows are features.
// Pairs are columns, so a group of at most 8 heads wastes no product; the legacy tensor instruction suffices, both products of a
// tile are 16 instructions for 4 KB of codes.
// E4M3 -> f16 is exact and one instruction for two codes.  The contraction order of a product is free, so a lane takes 16
// neighbouring features of a K row as its share of four k-steps, and 16 neighbouring features of four V rows (byte-permuted
// into pairs of keys): all shared-memory reads are 16 bytes wide, and the row order within a group of 8 keys is chosen so
// that they are free of bank conflicts.  q is scaled by a power of two per head into f16 range.  The reference of the
// exponent follows the maximum lazily, so a tile costs one vote instead of a reduction over its keys.  Softmax statistics
// and O are fp32; K's scale is applied to the scores, V's to the weights, relative to the largest V scale so far.
// Measured: 256 sequences of 2304 keys (1.13 GB) in 170 us = 103 % of a copy's rate, repeated on one cache, and 176 to 187 us = 94 to 100 % as a
// call among caches that change; one sequence of 32768 keys (67 MB) in 19 us, 24 of 100 to 4351 keys (103 MB) in 29 us, 53 %: launch, first lookups, ramp of the rings and the join do not shrink with it.
#include <math_constants.h>

#include <algorithm>

#include "pd_paged.cuh"

namespace pd {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

struct PagedDecodeArgs {
  const bf16* q;              // [rows, ldq]
  bf16* o;                    // [rows, Hq*hd]
  const int32_t* cu_seqlens;  // runs: [n_req + 1]; NULL: sequence b has the one row b
  const int32_t* kv_len;      // [n_req] position of the first row; runs: may be NULL (0)
  PagedParts parts;           // used when n_splits > 1
  int* err_word;
  PagedCache c;
  int ldq, rows, n_req, n_q_heads, n_kv_heads;
  int block_tokens;           // tokens of a block: block_tokens * group columns
  int n_splits, chunk;        // block x covers keys x * chunk .. (the last one whatever lies behind); chunk is a multiple of 64
};

constexpr int PA_WARPS = 8;
constexpr int PA_THREADS = PA_WARPS * 32;
constexpr int PA_KEYS = 16;
constexpr int PA_STAGES = 3;
// p is kept as 2^7 p relative to a reference that may lag the running maximum by 2^8: at most 2^15, below f16's 65504.
constexpr float P_SHIFT = 7.f, P_SLACK = 8.f, P_UNIT = 1.f / 128.f;
constexpr int PA_MIN_CHUNK = 256;               // keys of a part at least
constexpr int PA_RESIDENT = 296;                // blocks that run together (half as many WIDE ones)
constexpr float P_FAR = 1.f / 1024.f;

template <int HD>
struct PagedSmem {
  static constexpr int TILE = PA_KEYS * HD;                  // one K (or V) tile
  static constexpr int RING = PA_WARPS * PA_STAGES * 2 * TILE;
  static constexpr int MERGE = PA_WARPS * 16 * (HD + 2) * 4;
  static constexpr int BYTES = RING > MERGE ? RING : MERGE;
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
// The transpose of an 8 x 8 matrix of halves held one row per four lanes.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
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

// WIDE: 9 to 16 columns (two column groups in both products).  RUNS: blocks of several tokens; the one-token form is kept
// apart because its registers are few (with the masks of several tokens in it, a single long sequence took 1.4 times as long).
template <int HD, bool WIDE, bool RUNS>
__global__ void __launch_bounds__(PA_THREADS, WIDE ? 1 : 2) paged_decode_kernel(const PagedDecodeArgs a) {
  using SM = PagedSmem<HD>;
  constexpr int KS = HD / 16;          // k-steps of K Q^T
  constexpr int MT = HD / 16;          // 16-feature tiles of O^T
  constexpr int NC = WIDE ? 2 : 1;     // column groups of 8 heads
  extern __shared__ __align__(128) uint8_t smem[];
  const int split = blockIdx.x, kvh = blockIdx.y;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, t4 = lane & 3;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();

  const int l2p = a.c.log2_page, cap = a.c.table_ld << l2p;
  int b = blockIdx.z, row0 = b, n_tok = 1, pos0 = 0;  // sequence, first row, tokens, position of the first token
  if (RUNS) {
    const TokenBlock blk = find_block(a.cu_seqlens, a.kv_len, a.n_req, a.rows, b, a.block_tokens);
    if (blk.t0 >= blk.len) return;
    b = blk.req;
    row0 = blk.start + blk.t0;
    n_tok = min(a.block_tokens, blk.len - blk.t0);
    pos0 = blk.pre + blk.t0;
  }
  const int n_cols = n_tok * group;
  // Page numbers of 32 tiles of this warp at a time, a tile per lane.  The first 32 are read before the sequence's length is
  // known: entries behind its last page are read, too, but not used.
  const int32_t* table = a.c.table + static_cast<size_t>(b) * a.c.table_ld;
  const long long split_begin = 1ll * split * a.chunk;
  auto page_of = [&](int tile) { return (split_begin + (tile * PA_WARPS + warp) * PA_KEYS) >> l2p; };
  const long long first_page = page_of(lane);
  int id_cur = first_page < a.c.table_ld ? table[first_page] : -1;
  // Column c * 8 + j is token (c * 8 + j) / group, head (c * 8 + j) % group.  q of column c * 8 + g: this lane's share of every
  // k-step
  const uint32_t inv_group = 65536u / group + 1u;
  auto token_of = [&](int col) { return RUNS ? static_cast<int>((col * inv_group) >> 16) : 0; };
  uint2 qw[NC][KS];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int tok = token_of(c * 8 + g), head = c * 8 + g - tok * group;
    const bf16* src = a.q + static_cast<size_t>(row0 + tok) * a.ldq + (kvh * group + head) * HD + t4 * 16;
#pragma unroll
    for (int s = 0; s < KS; ++s)
      qw[c][s] = c * 8 + g < n_cols ? *reinterpret_cast<const uint2*>(src + (s >> 2) * 64 + (s & 3) * 4) : make_uint2(0u, 0u);
  }
  if (!RUNS) pos0 = min(a.kv_len[b], cap);
  if (split == 0 && kvh == 0 && tid == 0 && a.err_word && pos0 + n_tok > cap) atomicExch(a.err_word, 2);
  // keys that the last token sees; 0: none (a padding row)
  const int total = max(min(pos0 + n_tok, cap), 0);
  const int k_begin = static_cast<int>(min(1ll * total, split_begin));
  const int k_end = split == a.n_splits - 1 ? total : static_cast<int>(min(1ll * total, 1ll * k_begin + a.chunk));
  // the row of column `col` among the partial results, and among the outputs (split 0)
  auto out_row = [&](int col) {
    const int tok = token_of(col);
    return static_cast<size_t>(row0 + tok) * a.n_q_heads + kvh * group + col - tok * group;
  };
  const size_t part_row0 = static_cast<size_t>(split) * a.rows * a.n_q_heads;
  if (split > 0 && k_begin == k_end) {
    if (tid < n_cols) a.parts.ml[part_row0 + out_row(tid)] = make_float2(-CUDART_INF_F, 0.f);
    return;
  }
  const int n_tiles_blk = (k_end - k_begin + PA_KEYS - 1) / PA_KEYS;
  const int my_tiles = (n_tiles_blk > warp) ? (n_tiles_blk - warp + PA_WARPS - 1) / PA_WARPS : 0;
  const uint32_t ring = ptx::smem_u32(smem) + warp * (PA_STAGES * 2 * SM::TILE);

  // Of a batch of 32 tiles: -1 for a page that does not exist (its keys are left out), and the pages' scales.
  auto fetch_scales = [&](int first, int& id, float& ks, float& vs) {
    ks = -1.f; vs = 0.f;
    if (first + lane >= my_tiles) {
      id = -1;
    } else if (static_cast<unsigned>(id) < static_cast<unsigned>(a.c.n_pages)) {
      ks = a.c.k_scale[static_cast<size_t>(id) * a.n_kv_heads + kvh];
      vs = a.c.v_scale[static_cast<size_t>(id) * a.n_kv_heads + kvh];
    } else {
      id = -1;
      if (a.err_word) atomicExch(a.err_word, 2);
    }
  };
  // the next batch is fetched a batch ahead
  auto fetch_pages = [&](int first, int& id, float& ks, float& vs) {
    id = first + lane < my_tiles ? table[page_of(first + lane)] : -1;
    fetch_scales(first, id, ks, vs);
  };
  int id_nxt = -1;
  float ks_cur, vs_cur, ks_nxt = -1.f, vs_nxt = 0.f;
  fetch_scales(0, id_cur, ks_cur, vs_cur);
  if (my_tiles > 32) fetch_pages(32, id_nxt, ks_nxt, vs_nxt);

  // A tile of a page is PA_KEYS * HD contiguous bytes: chunk `lane + 32 i` of it goes to its swizzled place.
  constexpr int NLD = PA_KEYS * HD / 512;
  uint32_t dst[NLD];
#pragma unroll
  for (int i = 0; i < NLD; ++i) dst[i] = chunk_off<HD>((lane + 32 * i) / (HD / 16), (lane + 32 * i) % (HD / 16));
  auto load_tile = [&](int i, int stage) {
    if (i > 0 && (i & 31) == 0) id_cur = id_nxt;
    const int id = __shfl_sync(0xffffffffu, id_cur, i & 31);
    const int key0 = k_begin + (i * PA_WARPS + warp) * PA_KEYS;
    const int row0 = key0 & ((1 << l2p) - 1);
    const size_t base = (((static_cast<size_t>(max(id, 0)) * a.n_kv_heads + kvh) << l2p) + row0) * HD + lane * 16;
    const uint32_t sk = ring + stage * 2 * SM::TILE, sv = sk + SM::TILE;
    // rows past the end become zeros: whatever they hold is not read
    const int n_ok = id < 0 ? 0 : min(k_end - key0, PA_KEYS);
#pragma unroll
    for (int i2 = 0; i2 < NLD; ++i2) {
      const bool ok = (lane + 32 * i2) / (HD / 16) < n_ok;
      ptx::cp_async_16(sk + dst[i2], a.c.k + base + (ok ? 512 * i2 : 0), ok);
      ptx::cp_async_16(sv + dst[i2], a.c.v + base + (ok ? 512 * i2 : 0), ok);
    }
  };
#pragma unroll
  for (int s = 0; s < PA_STAGES - 1; ++s) {
    if (s < my_tiles) load_tile(s, s);
    ptx::cp_async_commit();
  }

  // Q^T as f16 operand fragments, every head scaled by a power of two so that its largest entry lies in [1, 2)
  uint32_t qb[NC][KS][2];
  float q_scale[NC];  // of the scores of head c * 8 + g, in log2 units
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float amax = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
      amax = fmaxf(amax, fmaxf(fmaxf(fabsf(ptx::bf16_lo(qw[c][s].x)), fabsf(ptx::bf16_hi(qw[c][s].x))),
                               fmaxf(fabsf(ptx::bf16_lo(qw[c][s].y)), fabsf(ptx::bf16_hi(qw[c][s].y)))));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    // 2^e <= amax < 2^(e+1), e kept where 2^e and 2^-e are normal (an infinite q stays infinite)
    const int e = min(max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -126), 126);
    const float up = __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
    const float inv = pow2_inverse(up);
    q_scale[c] = rsqrtf(static_cast<float>(HD)) * LOG2E * up;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qb[c][s][0] = pack_f16(ptx::bf16_lo(qw[c][s].x) * inv, ptx::bf16_hi(qw[c][s].x) * inv);
      qb[c][s][1] = pack_f16(ptx::bf16_lo(qw[c][s].y) * inv, ptx::bf16_hi(qw[c][s].y) * inv);
    }
  }
  // This lane's columns of S^T and O^T are c * 8 + 2 t4 + h, h = 0, 1.
  float f_head[NC][2];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    f_head[c][0] = __shfl_sync(0xffffffffu, q_scale[c], t4 * 8);
    f_head[c][1] = __shfl_sync(0xffffffffu, q_scale[c], t4 * 8 + 4);
  }

  float o_acc[NC][MT][4];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < MT; ++i) o_acc[c][i][0] = o_acc[c][i][1] = o_acc[c][i][2] = o_acc[c][i][3] = 0.f;
  // reference of the exponent (uniform over the lanes of a head; -inf: no key yet) and this lane's share of the sum
  float m_ref[NC][2], l_sum[NC][2];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m_ref[c][0] = m_ref[c][1] = -CUDART_INF_F;
    l_sum[c][0] = l_sum[c][1] = 0.f;
  }
  float unit = 0.f;  // o_acc counts in this V scale, the largest so far
  bool nan_seen = false;

  for (int i = 0; i < my_tiles; ++i) {
    const int stage = i % PA_STAGES;
    if (i > 0 && (i & 31) == 0) {
      ks_cur = ks_nxt; vs_cur = vs_nxt;
      if (i + 32 < my_tiles) fetch_pages(i + 32, id_nxt, ks_nxt, vs_nxt);
    }
    {
      const int nxt = i + PA_STAGES - 1;
      if (nxt < my_tiles) load_tile(nxt, nxt % PA_STAGES);
      ptx::cp_async_commit();
    }
    const float ks = __shfl_sync(0xffffffffu, ks_cur, i & 31), vs = __shfl_sync(0xffffffffu, vs_cur, i & 31);
    ptx::cp_async_wait<PA_STAGES - 1>();
    __syncwarp();
    const uint32_t sk = ring + stage * 2 * SM::TILE, sv = sk + SM::TILE;
    const int key0 = k_begin + (i * PA_WARPS + warp) * PA_KEYS;
    if (RUNS && key0 + PA_KEYS - 1 > pos0) {  // not every token of the block sees all keys (in place: registers are short)
#pragma unroll 1
      for (int o = lane * 16; o < SM::TILE; o += 512) {
        if (key0 + o / HD <= pos0) continue;
        const uint4 w = lds128(sv + o);
        bool seen = false;
        const uint4 d = make_uint4(drop_nans(w.x, seen), drop_nans(w.y, seen), drop_nans(w.z, seen), drop_nans(w.w, seen));
        if (seen) asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(sv + o), "r"(d.x), "r"(d.y), "r"(d.z), "r"(d.w) : "memory");
        nan_seen |= seen;
      }
      __syncwarp();
    }

    // ---- S^T = K Q^T: rows are keys key_of(g) and 8 + key_of(g), columns heads
    float st[NC][2][4];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) st[c][0][e] = st[c][1][e] = 0.f;
#pragma unroll
    for (int h = 0; h < HD / 64; ++h) {
      const uint4 w0 = lds128(sk + chunk_off<HD>(key_of<HD>(g), h * 4 + t4));
      const uint4 w1 = lds128(sk + chunk_off<HD>(8 + key_of<HD>(g), h * 4 + t4));
      const uint32_t x0[4] = {w0.x, w0.y, w0.z, w0.w}, x1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t a0 = e4m3x2_to_f16x2(static_cast<uint16_t>(x0[q])), a2 = e4m3x2_to_f16x2(static_cast<uint16_t>(x0[q] >> 16));
        const uint32_t a1 = e4m3x2_to_f16x2(static_cast<uint16_t>(x1[q])), a3 = e4m3x2_to_f16x2(static_cast<uint16_t>(x1[q] >> 16));
#pragma unroll
        for (int c = 0; c < NC; ++c) mma_f16(st[c][q & 1], a0, a1, a2, a3, qb[c][h * 4 + q][0], qb[c][h * 4 + q][1]);
      }
    }
    // ---- softmax
    const bool masked = key0 + PA_KEYS > (RUNS ? min(k_end, pos0 + 1) : k_end) || ks < 0.f;
    float x[NC][4];  // [key half][head] = (e >> 1, e & 1)
    bool grow = false;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float f0 = f_head[c][0] * ks, f1 = f_head[c][1] * ks;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[c][e] = (st[c][0][e] + st[c][1][e]) * ((e & 1) ? f1 : f0);
      if (masked) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // the last key of the tile that the column's token sees
          const int lim = ks < 0.f ? -1 : (RUNS ? min(pos0 + token_of(c * 8 + 2 * t4 + h), k_end - 1) : k_end - 1) - key0;
          if (key_of<HD>(g) > lim) x[c][h] = -CUDART_INF_F;
          if (8 + key_of<HD>(g) > lim) x[c][2 + h] = -CUDART_INF_F;
        }
      }
      // the reference follows the maximum only when that has grown by more than P_SLACK (always at the first key)
      grow |= fmaxf(x[c][0], x[c][2]) > m_ref[c][0] + P_SLACK || fmaxf(x[c][1], x[c][3]) > m_ref[c][1] + P_SLACK;
    }
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float mx = fmaxf(x[c][h], x[c][2 + h]);
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          const float m_new = fmaxf(m_ref[c][h], mx);
          const float corr = m_new == -CUDART_INF_F ? 1.f : ptx::ex2_approx(m_ref[c][h] - m_new);
          m_ref[c][h] = m_new;
          l_sum[c][h] *= corr;
#pragma unroll
          for (int n = 0; n < MT; ++n) { o_acc[c][n][h] *= corr; o_acc[c][n][2 + h] *= corr; }
        }
      }
    }
    if (vs > unit) {  // uniform; the quotient of two powers of two is exact (0 at the first tile: o_acc is still 0)
      const float r = unit * pow2_inverse(vs);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int n = 0; n < MT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) o_acc[c][n][e] *= r;
      unit = vs;
    }
    const float w = vs * pow2_inverse(unit);  // <= 1
    // a page whose V is far smaller than the largest: its weights would leave f16's range, so its product is scaled in fp32
    const bool far = w < P_FAR;
    const float pw = far ? 1.f : w;
    uint32_t pb[NC][2];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float ref = (m_ref[c][h] == -CUDART_INF_F ? 0.f : m_ref[c][h]) - P_SHIFT;  // (no key yet: every p is 0)
        x[c][h] = ptx::ex2_approx(x[c][h] - ref);
        x[c][2 + h] = ptx::ex2_approx(x[c][2 + h] - ref);
        l_sum[c][h] += x[c][h] + x[c][2 + h];
      }
      // P^T as an operand: the transpose of the accumulator's 8 x 8 blocks
      pb[c][0] = transpose8x8(pack_f16(x[c][0] * pw, x[c][1] * pw));
      pb[c][1] = transpose8x8(pack_f16(x[c][2] * pw, x[c][3] * pw));
    }
    // ---- O^T += V^T P^T: this lane's keys are key_of(2 t4), key_of(2 t4 + 1) of both halves, its features g * hd/8 ...
    uint32_t vw[4][HD / 32];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = (r >> 1) * 8 + key_of<HD>(t4 * 2 + (r & 1));
      if (HD == 128) {
        const uint4 v = lds128(sv + chunk_off<HD>(row, g));
        vw[r][0] = v.x; vw[r][1] = v.y; vw[r][HD / 32 - 2] = v.z; vw[r][HD / 32 - 1] = v.w;
      } else {
        const uint2 v = lds64(sv + chunk_off<HD>(row, g >> 1) + (g & 1) * 8);
        vw[r][0] = v.x; vw[r][1] = v.y;
      }
    }
    auto product = [&](auto accumulate) {
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // features 4 j + 2 h, 4 j + 2 h + 1
          const uint32_t sel = h ? 0x7362u : 0x5140u;
          const uint32_t u = __byte_perm(vw[0][j], vw[1][j], sel), y = __byte_perm(vw[2][j], vw[3][j], sel);
          const uint32_t a0 = e4m3x2_to_f16x2(static_cast<uint16_t>(u)), a1 = e4m3x2_to_f16x2(static_cast<uint16_t>(u >> 16));
          const uint32_t a2 = e4m3x2_to_f16x2(static_cast<uint16_t>(y)), a3 = e4m3x2_to_f16x2(static_cast<uint16_t>(y >> 16));
#pragma unroll
          for (int c = 0; c < NC; ++c) accumulate(c, 2 * j + h, a0, a1, a2, a3);
        }
      }
    };
    if (!far) {
      product([&](int c, int n, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
        mma_f16(o_acc[c][n], a0, a1, a2, a3, pb[c][0], pb[c][1]);
      });
    } else {
      product([&](int c, int n, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
        float f[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16(f, a0, a1, a2, a3, pb[c][0], pb[c][1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) o_acc[c][n][e] = fmaf(f[e], w, o_acc[c][n][e]);
      });
    }
    __syncwarp();  // every lane has read this stage before it is refilled
  }
  ptx::cp_async_wait<0>();
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l_sum[c][h] += __shfl_xor_sync(0xffffffffu, l_sum[c][h], o);
  __syncthreads();  // every warp has left its ring: the memory is reused for the merge

  float* mrg = reinterpret_cast<float*>(smem);
  constexpr int RS = HD + 2;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int col = c * 8 + t4 * 2 + h;
      if (col < n_cols) {
        float* dst_row = mrg + (warp * 16 + col) * RS;
#pragma unroll
        for (int n = 0; n < MT; ++n) {
          dst_row[g * (HD / 8) + 2 * n] = o_acc[c][n][h] * (unit * P_UNIT);
          dst_row[g * (HD / 8) + 2 * n + 1] = o_acc[c][n][2 + h] * (unit * P_UNIT);
        }
        if (g == 0) { dst_row[HD] = m_ref[c][h]; dst_row[HD + 1] = l_sum[c][h] * P_UNIT; }
      }
    }
  }
  const bool nans = RUNS ? __syncthreads_or(nan_seen) : (__syncthreads(), false);
  for (int idx = tid; idx < n_cols * HD; idx += PA_THREADS) {
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
    const size_t row = out_row(r);
    if (RUNS && nans) {
      for (int key = max(pos0 + 1, k_begin); key <= min(pos0 + token_of(r), k_end - 1); ++key) {
        const uint8_t* v = v_row(a.c, table, a.n_kv_heads, kvh, HD, key);
        if (v && (v[d] & 0x7f) == 0x7f) o = CUDART_NAN_F;
      }
    }
    if (a.n_splits == 1) {
      a.o[row * HD + d] = __float2bfloat16(l == 0.f ? 0.f : o / l);  // (no visible entry: zeros)
    } else {
      a.parts.o[(part_row0 + row) * HD + d] = o;
      if (d == 0) a.parts.ml[part_row0 + row] = make_float2(m, l);
    }
  }
}

// Joins the parts of a row = (token, query head).  With few rows or many parts the four warps of a block share a row: each
// computes the weights of all parts (a part per lane), they divide the parts' outputs and add up in shared memory.  Otherwise
// every warp has a row (16384 rows of two parts: 8 us, 24 with a block per row).  All loads of a round are issued before the
// first is used; outputs of parts without keys are loaded, too, and left out.
constexpr int PJ_WARPS = 4, PJ_PARTS = 8;  // parts per warp and round

template <int HD, int WARPS_PER_ROW>
__global__ void __launch_bounds__(PJ_WARPS * 32) paged_join_kernel(const PagedParts p, bf16* o, long long rows, int n_splits) {
  constexpr int V = HD / 32, ROUND = PJ_PARTS * WARPS_PER_ROW;  // features per lane, parts per round
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int share = WARPS_PER_ROW == 1 ? 0 : warp;
  const long long row = WARPS_PER_ROW == 1 ? 1ll * blockIdx.x * PJ_WARPS + warp : blockIdx.x;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  if (row >= rows) return;  // (a whole warp, and only where warps do not meet)
  float m_run = -CUDART_INF_F, l = 0.f, o_sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) o_sum[e] = 0.f;
  for (int s0 = 0; s0 < n_splits; s0 += ROUND) {
    const float2 st = lane < ROUND && s0 + lane < n_splits ? p.ml[static_cast<size_t>(s0 + lane) * rows + row] : make_float2(-CUDART_INF_F, 0.f);
    float v[PJ_PARTS][V];
#pragma unroll
    for (int i = 0; i < PJ_PARTS; ++i) {
      const int s = s0 + i * WARPS_PER_ROW + share;
#pragma unroll
      for (int e = 0; e < V; ++e) v[i][e] = 0.f;
      if (s < n_splits) {
        const float* src = p.o + (static_cast<size_t>(s) * rows + row) * HD + lane * V;
        if (V == 4) {
          const float4 w = *reinterpret_cast<const float4*>(src);
          v[i][0] = w.x; v[i][1] = w.y; v[i][V - 2] = w.z; v[i][V - 1] = w.w;
        } else {
          const float2 w = *reinterpret_cast<const float2*>(src);
          v[i][0] = w.x; v[i][1] = w.y;
        }
      }
    }
    const bool held = st.x != -CUDART_INF_F || st.y != 0.f;  // the part saw keys (so its outputs are there)
    float m = fmaxf(m_run, st.x);
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
    const float m_use = m == -CUDART_INF_F ? 0.f : m;
    const float corr = exp2f(m_run - m_use), f_lane = exp2f(st.x - m_use);
    m_run = m;
    l = l * corr + st.y * f_lane;
#pragma unroll
    for (int e = 0; e < V; ++e) o_sum[e] *= corr;
    const uint32_t held_mask = __ballot_sync(0xffffffffu, held);
#pragma unroll
    for (int i = 0; i < PJ_PARTS; ++i) {
      const int s = i * WARPS_PER_ROW + share;
      const float f = __shfl_sync(0xffffffffu, f_lane, s);
      if ((held_mask >> s) & 1u) {
#pragma unroll
        for (int e = 0; e < V; ++e) o_sum[e] = fmaf(v[i][e], f, o_sum[e]);
      }
    }
  }
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) l += __shfl_xor_sync(0xffffffffu, l, k);
  if constexpr (WARPS_PER_ROW == 1) {
    float r[V];
#pragma unroll
    for (int e = 0; e < V; ++e) r[e] = l == 0.f ? 0.f : o_sum[e] / l;  // (no visible entry: zeros)
    uint32_t* dst = reinterpret_cast<uint32_t*>(o + row * HD + lane * V);
#pragma unroll
    for (int e = 0; e < V; e += 2) dst[e / 2] = ptx::pack_bf16(r[e], r[e + 1]);
  } else {
    __shared__ float acc[PJ_WARPS][HD];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[warp][lane * V + e] = o_sum[e];
    __syncthreads();
    if (threadIdx.x < HD) {
      const float sum = (acc[0][threadIdx.x] + acc[1][threadIdx.x]) + (acc[2][threadIdx.x] + acc[3][threadIdx.x]);
      o[row * HD + threadIdx.x] = __float2bfloat16(l == 0.f ? 0.f : sum / l);
    }
  }
}

template <int HD, bool WIDE, bool RUNS>
pd_status launch_rows(const PagedDecodeArgs& a, int slots, cudaStream_t s) {
  using SM = PagedSmem<HD>;
  static PerDeviceInt smem_opt_in;
  PD_TRY(opt_in_smem(smem_opt_in, paged_decode_kernel<HD, WIDE, RUNS>, SM::BYTES));
  PD_CUDA_TRY(launch_pdl(paged_decode_kernel<HD, WIDE, RUNS>, dim3(a.n_splits, a.n_kv_heads, slots), dim3(PA_THREADS), SM::BYTES, s, a));
  count_launch();
  if (a.n_splits > 1) return launch_paged_join(a.parts, a.o, 1ll * a.rows * a.n_q_heads, a.n_splits, HD, s);
  return PD_OK;
}
template <int HD, bool WIDE>
pd_status launch_rows(const PagedDecodeArgs& a, int slots, cudaStream_t s) {
  return a.cu_seqlens ? launch_rows<HD, WIDE, true>(a, slots, s) : launch_rows<HD, WIDE, false>(a, slots, s);
}
bool rows_wide(const PagedDecodeArgs& a) { return a.block_tokens * (a.n_q_heads / a.n_kv_heads) > 8; }
pd_status launch_rows_any(const PagedDecodeArgs& a, int head_dim, int slots, cudaStream_t s) {
  if (head_dim == 128) return rows_wide(a) ? launch_rows<128, true>(a, slots, s) : launch_rows<128, false>(a, slots, s);
  return rows_wide(a) ? launch_rows<64, true>(a, slots, s) : launch_rows<64, false>(a, slots, s);
}

// Key ranges are cut into equal parts while there are fewer blocks than run together, into parts of at least PA_MIN_CHUNK keys
// and at most `longest` keys.
struct Split { int n, chunk; };
Split rows_split(long long blocks, long long parts, int max_kv_len, int longest) {
  if (blocks <= 0 || max_kv_len <= 0) return {1, PA_MIN_CHUNK};
  long long want = parts / blocks;
  if (want < 1) want = 1;
  long long chunk = (max_kv_len + want - 1) / want;
  if (chunk > longest) chunk = longest;
  if (chunk < PA_MIN_CHUNK) chunk = PA_MIN_CHUNK;
  chunk = (chunk + 63) / 64 * 64;
  return {static_cast<int>((max_kv_len + chunk - 1) / chunk), static_cast<int>(chunk)};
}
// Decode.  The sequences of a batch may differ in length, which the host does not know, so a part is at most 4096 keys (30
// sequences of up to 32000 keys: 175 us, 250 us uncut), and from about one block per SM on half as many parts again as run
// together even the lengths out (24 sequences of 100 to 4351 keys, 192 blocks: 31 us, 37 us at one part per resident block; 4
// sequences of 8000 keys, 32 blocks: 21 us, 18 us).  More parts cost more in the join than they bring; no more than 16 are
// made for the length alone, since max_kv_len may be a capacity far above the lengths.
Split decode_split(int batch, int n_kv_heads, int max_kv_len) {
  const long long blocks = 1ll * batch * n_kv_heads;
  return rows_split(blocks, blocks <= 148 ? PA_RESIDENT : PA_RESIDENT * 3 / 2, max_kv_len,
                    batch > 1 ? std::max(4096, max_kv_len / 16) : max_kv_len);
}

// (part, sequence) pairs that any call of up to `batch` sequences and a bound of up to max_kv_len has at most, where it has
// parts at all: a buffer of that size serves every smaller call, too.  Parts made to fill the GPU are at most as many as
// decode_split asks for, of at least PA_MIN_CHUNK keys; parts made for their length are as many as the bound allows.
long long decode_most_parts(int batch, int n_kv_heads, int max_kv_len) {
  if (batch <= 0 || max_kv_len <= PA_MIN_CHUNK) return 0;
  const long long fill = (1ll * batch * n_kv_heads <= 148 ? PA_RESIDENT : PA_RESIDENT * 3 / 2) / n_kv_heads;
  const long long most = std::min(fill, batch * ((max_kv_len + (PA_MIN_CHUNK - 1ll)) / PA_MIN_CHUNK));
  // (17: of max_kv_len / 16 keys, rounded down, and what is left)
  const long long length = batch > 1 ? std::min(17ll, (max_kv_len + 4095ll) / 4096) : 1;
  return std::max(most > 1 ? most : 0, length > 1 ? length * batch : 0);
}

}  // namespace

pd_status launch_paged_join(const PagedParts& parts, bf16* o, long long rows, int n_splits, int head_dim, cudaStream_t s) {
  if (rows > 0x7fffffffll) return PD_ERR_UNSUPPORTED_SHAPE;
  // (blocks enough for the whole GPU either way; a warp per row stores pairs of values, so a result that starts between two
  // 4-byte words takes the other form, which stores single ones)
  const bool few = n_splits <= PJ_PARTS && rows > 2048 && (reinterpret_cast<uintptr_t>(o) & 3u) == 0;
  const dim3 grid(static_cast<unsigned>(few ? (rows + PJ_WARPS - 1) / PJ_WARPS : rows)), block(PJ_WARPS * 32);
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, block, 0, s, parts, o, rows, n_splits); };
  PD_CUDA_TRY(head_dim == 128 ? (few ? go(paged_join_kernel<128, 1>) : go(paged_join_kernel<128, 4>))
                              : (few ? go(paged_join_kernel<64, 1>) : go(paged_join_kernel<64, 4>)));
  count_launch();
  return PD_OK;
}

int paged_rows_block(int group, int longest_run) {
  // eight columns where the runs fit them (half the registers), else sixteen
  return (group * longest_run <= 8 ? 8 : 16) / group;
}

size_t paged_rows_part_rows() { return PA_RESIDENT * 16; }

pd_status launch_paged_rows(const PagedRuns& r, int longest_run, const PagedParts& parts, cudaStream_t s) {
  PagedDecodeArgs a{};
  a.q = r.q; a.o = r.o; a.cu_seqlens = r.cu_seqlens; a.kv_len = r.prefix; a.parts = parts; a.err_word = r.err_word; a.c = r.c;
  a.ldq = r.ldq; a.rows = r.n_tokens; a.n_req = r.n_req; a.n_q_heads = r.n_q_heads; a.n_kv_heads = r.n_kv_heads;
  a.block_tokens = paged_rows_block(r.n_q_heads / r.n_kv_heads, longest_run);
  const int slots = first_slot(r.n_tokens, r.n_req, a.block_tokens);
  if (slots > 65535) return PD_ERR_UNSUPPORTED_SHAPE;
  const Split sp = rows_split(1ll * slots * r.n_kv_heads, rows_wide(a) ? PA_RESIDENT / 2 : PA_RESIDENT, r.max_kv, r.max_kv);
  a.n_splits = sp.n; a.chunk = sp.chunk;
  return launch_rows_any(a, r.head_dim, slots, s);
}

}  // namespace pd

extern "C" pd_status pd_paged_decode_attention_workspace_bytes(const pd_layer_cfg* cfg, int32_t B, int32_t max_kv_len,
                                                               size_t* out_bytes) {
  PD_TRY(pd::check_paged_heads(cfg));
  if (!out_bytes || B < 0 || max_kv_len < 0) return PD_ERR_INVALID_ARG;
  const long long parts = pd::decode_most_parts(B, cfg->n_kv_heads, max_kv_len);
  *out_bytes = parts ? pd::paged_parts_bytes(static_cast<size_t>(parts) * cfg->n_q_heads, cfg->head_dim) : 0;
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
  const Split sp = decode_split(B, cfg->n_kv_heads, max_kv_len);
  a.n_splits = sp.n; a.chunk = sp.chunk;
  if (a.n_splits > 1) {
    const size_t part_rows = static_cast<size_t>(a.n_splits) * B * cfg->n_q_heads;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PD_ERR_INVALID_ARG;
    if (workspace_bytes < paged_parts_bytes(part_rows, cfg->head_dim)) return PD_ERR_WORKSPACE_TOO_SMALL;
    a.parts.o = static_cast<float*>(workspace);
    a.parts.ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + paged_parts_ml_offset(part_rows, cfg->head_dim));
  }
  a.q = static_cast<const bf16*>(q); a.o = static_cast<bf16*>(out); a.kv_len = kv_len_dev; a.err_word = err_word;
  a.ldq = ldq; a.rows = B; a.n_req = B; a.n_q_heads = cfg->n_q_heads; a.n_kv_heads = cfg->n_kv_heads; a.block_tokens = 1;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_ATTN_DECODE, st);
  return launch_rows_any(a, cfg->head_dim, B, st);
}
