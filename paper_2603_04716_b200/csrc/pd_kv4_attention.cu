// Attention over the 4-bit paged KV cache for one or a few query tokens per sequence (pd_paged_kv4_decode_attention).
//
// o = softmax(q K^T / sqrt(hd)) V per query head over the sequence's pages; K and V are E2M1 codes times an E4M3 scale per 16
// features.  HBM-bound: 0.5625 bytes per element, read once (by every block of tokens).  One block per (part of the key range,
// KV head, sequence and block of tokens); parts join in a cluster or in a kernel of their own; every
// warp streams its own 32-key tiles through a private cp.async ring.
//   S^T = K Q^T    m16n8k16 in f16: rows are 16 keys, columns 8 (token, head of the group) pairs.
//   O^T = V^T P^T  m16n8k16: rows are features.
// A code times its scale has six significant bits and lies in 2^-10 .. 2688: exact in f16.  The contraction order of a product
// is free, so a lane takes hd / 4 neighbouring features of a K row as its share of all k-steps and hd / 8 neighbouring features of
// four V rows per 16 keys: its scales are a byte or two per row.  Features of two V rows are paired by shifts and masks on whole
// words before they are converted.  q is scaled by a power of two per head into f16 range.  The reference of the exponent
// follows the maximum lazily, so a tile costs one vote instead of a reduction over its keys.  Softmax statistics and O are fp32; weights
// are f16 in the second product, the operand's type, which is 2^-11 of a weight, an eighth of the result's own rounding (bf16 results
// differ from those of fp32 weights by 2.4e-4 in norm, and from 64 bits by 1.4e-3 either way).
// A tile of 32 keys costs a warp 565 instructions (128 conversions, 128 products with scales, 32 MMAs), a warp 660 more at both ends:
// instructions and their latency bind as much as HBM.  Measured, heads of 128: 256 sequences of 2,304 keys, 32 / 8 heads (640 MB)
// 118 us in bursts of a few milliseconds at an SM clock of 1,965 MHz (5.4 TB/s), 137 us where calls go on and the power cap holds the
// clock at 1,690 MHz (4.7 TB/s): 232,000 cycles either way.  In bursts each 1,024 keys more cost 52 us (5.8 TB/s), and pages shared in L2
// take the same time.  24 sequences of 100 to 4,351 keys, two tokens, 64 / 8 heads 30 us; one of 32,768 keys 16.3.
#include <math_constants.h>

#include <algorithm>

#include "pd_kv4.cuh"
#include "pd_paged.cuh"

namespace pd {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

struct Kv4DecodeArgs {
  const bf16* q;              // [B * n_new, ldq]
  bf16* o;                    // [B * n_new, Hq*hd]
  const int32_t* kv_len;      // [B] position of the first row
  PagedParts parts;           // used when n_splits > 1
  int* err_word;
  Kv4Cache c;
  int ldq, rows, n_new, n_q_heads, n_kv_heads;
  int col_blocks;             // blocks of KA_COLS (token, head) pairs that a sequence and KV head has
  int n_splits, chunk;        // part x covers keys x * chunk .. (the last one whatever lies behind); chunk is a multiple of 64
};

constexpr int KA_KEYS = 32;                     // of a tile: two halves of 16, each within a page
constexpr int KA_STAGES = 3;
constexpr int KA_CLUSTER = 8;                   // parts that can meet in a cluster at most
// p is kept as 2^7 p relative to a reference that may lag the running maximum by 2^6: at most 2^13, with room below f16's 65504 for
// what 7 - reference loses to rounding where scores are very large.
constexpr float P_SHIFT = 7.f, P_SLACK = 6.f, P_UNIT = 1.f / 128.f;
constexpr int KA_MIN_CHUNK = 256;               // keys of a part at least
// (token, head) pairs, the columns of both products: one or two groups of 8 a block.  A second group shares the conversion of K and V,
// half of a tile's instructions, and costs registers: 12 warps of an SM run together instead of 16.
constexpr int ka_cols(int col_groups) { return 8 * col_groups; }
constexpr int ka_resident_warps(int col_groups) { return 148 * (col_groups == 1 ? 16 : 12); }

template <int HD, int WARPS, int NC>
struct Kv4Smem {
  static constexpr int CODES = KA_KEYS * HD / 2, SCALES = KA_KEYS * HD / 16;  // bytes of a tile's K (or V)
  static constexpr int STAGE = 2 * (CODES + SCALES);                          // K codes, V codes, K scales, V scales
  static constexpr int RING = WARPS * KA_STAGES * STAGE;
  static constexpr int MERGE_ROW = HD + 4;                                    // floats: a row of O, then l
  static constexpr int MERGE = (WARPS * (MERGE_ROW + 1) + 2) * ka_cols(NC) * 4;  // m of all rows behind, and (m, l) of the columns
  static constexpr int BYTES = RING > MERGE ? RING : MERGE;
};

// Key that row n of an 8-key group of S^T holds.  A lane reads V rows key_of(2 t), key_of(2 t + 1): four neighbouring rows each
// over the lanes.
__device__ __forceinline__ int key_of(int n) { return (n >> 1) | ((n & 1) << 2); }
// Where 16-byte chunk c of key r lies in a tile.  K rows lie in the order in which they are read (8 rows x 4 lanes side by
// side); V rows of 64 bytes swap their halves in every other pair, so that four rows x 32 bytes fill all banks.
template <int HD>
__device__ __forceinline__ uint32_t k_chunk(int r, int c) {
  return static_cast<uint32_t>(((r & ~7) | ((r & 3) << 1) | ((r >> 2) & 1)) * (HD / 2) + c * 16);
}
template <int HD>
__device__ __forceinline__ uint32_t v_chunk(int r, int c) {
  return static_cast<uint32_t>(r * (HD / 2) + (HD == 128 ? c ^ (r & 2) : c) * 16);
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same from an accumulator of zeros.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Eight E2M1 codes -> eight halves in order, exactly.
__device__ __forceinline__ void e2m1_to_f16(uint32_t codes, uint32_t (&h)[4]) {
  asm("{ .reg .b8 b0, b1, b2, b3; mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0; cvt.rn.f16x2.e2m1x2 %1, b1; cvt.rn.f16x2.e2m1x2 %2, b2; cvt.rn.f16x2.e2m1x2 %3, b3; }"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
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
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t addr) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// NC: groups of 8 columns.  MULTI: sequences with several tokens.  TOGETHER: the parts of a key range are a cluster, which joins them
// itself.
template <int HD, int KA_WARPS, int NC, bool MULTI, bool TOGETHER>
__global__ void __launch_bounds__(KA_WARPS * 32, ka_resident_warps(NC) / 148 / KA_WARPS) kv4_decode_kernel(const Kv4DecodeArgs a) {
  using SM = Kv4Smem<HD, KA_WARPS, NC>;
  constexpr int KA_COLS = ka_cols(NC);
  constexpr int KA_THREADS = KA_WARPS * 32;
  constexpr int KS = HD / 16;          // k-steps of K Q^T
  constexpr int MT = HD / 16;          // 16-feature tiles of O^T
  constexpr int W = HD / 32;           // words of codes a lane has of a K row, and 2 W of V rows
  extern __shared__ __align__(128) uint8_t smem[];
  // The blocks that read the same keys are neighbours, so that all but one of them find them in L2.  Parts come last: what starts
  // late is what few sequences are long enough for, and ends of sequences.
  const int kvh = blockIdx.x / a.col_blocks, col0 = (blockIdx.x - kvh * a.col_blocks) * KA_COLS, b = blockIdx.y, split = blockIdx.z;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, t4 = lane & 3;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();

  const int l2p = a.c.log2_page, cap = a.c.table_ld << l2p;
  // Column c of the block is pair col0 + c of the sequence: token (col0 + c) / group, head (col0 + c) % group
  const int n_cols = min(KA_COLS, a.n_new * group - col0);
  const int tok0 = MULTI ? col0 / group : 0, skew = col0 - tok0 * group;  // the first column is head `skew` of token tok0
  const uint32_t inv_group = 65536u / group + 1u;
  auto token_of = [&](int col) { return MULTI ? static_cast<int>(((col + skew) * inv_group) >> 16) : 0; };  // relative to tok0
  auto head_of = [&](int col) { return col + skew - token_of(col) * group; };
  const int n_tok = token_of(n_cols - 1) + 1, row0 = b * a.n_new + tok0;
  // Page numbers of the halves of 32 tiles of this warp at a time, a tile per lane.  The first 32 are read before the sequence's
  // length is known: entries behind its last page are read, too, but not used.
  const int32_t* table = a.c.table + static_cast<size_t>(b) * a.c.table_ld;
  const long long split_begin = 1ll * split * a.chunk;
  auto fetch_pages = [&](int first, int (&id)[2]) {
    const long long key = split_begin + (1ll * (first + lane) * KA_WARPS + warp) * KA_KEYS;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const long long page = (key + 16 * h) >> l2p;
      id[h] = (h == 1 && l2p > 4) ? id[0] : page < a.c.table_ld ? table[page] : -1;
    }
  };
  int id_cur[2], id_nxt[2] = {-1, -1};
  fetch_pages(0, id_cur);
  // q of column 8 c + g: this lane's share of all k-steps, features t4 * hd / 4 ..
  uint4 qw[NC][KS / 2];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = 8 * c + g;
    const bf16* src = a.q + static_cast<size_t>(row0 + token_of(col)) * a.ldq + (kvh * group + head_of(col)) * HD + t4 * (HD / 4);
#pragma unroll
    for (int s = 0; s < KS / 2; ++s) qw[c][s] = col < n_cols ? *reinterpret_cast<const uint4*>(src + s * 8) : make_uint4(0u, 0u, 0u, 0u);
  }
  const int len = a.kv_len[b];
  // position of the block's first token; a negative length: a padding sequence, none of its rows sees a key
  const int pos0 = len < 0 ? -0x40000000 : static_cast<int>(min(1ll * len + tok0, static_cast<long long>(cap)));
  if (split == 0 && kvh == 0 && tid == 0 && a.err_word && 1ll * len + tok0 + n_tok > cap) atomicExch(a.err_word, 2);
  const int total = static_cast<int>(max(min(1ll * pos0 + n_tok, static_cast<long long>(cap)), 0ll));  // keys that the last token sees
  const int k_begin = static_cast<int>(min(1ll * total, split_begin));
  const int k_end = split == a.n_splits - 1 ? total : static_cast<int>(min(1ll * total, 1ll * k_begin + a.chunk));
  // the row of column `col` among the partial results, and among the outputs (split 0)
  auto out_row = [&](int col) {
    return static_cast<size_t>(row0 + token_of(col)) * a.n_q_heads + kvh * group + head_of(col);
  };
  const size_t part_row0 = static_cast<size_t>(split) * a.rows * a.n_q_heads;
  if (split > 0 && k_begin == k_end) {
    if (!TOGETHER && tid < n_cols) a.parts.ml[part_row0 + out_row(tid)] = make_float2(-CUDART_INF_F, 0.f);
    return;
  }
  const int n_tiles_blk = static_cast<int>((static_cast<uint32_t>(k_end - k_begin) + KA_KEYS - 1) / KA_KEYS);
  const int my_tiles = (n_tiles_blk > warp) ? (n_tiles_blk - warp + KA_WARPS - 1) / KA_WARPS : 0;
  const uint32_t ring = ptx::smem_u32(smem) + warp * (KA_STAGES * SM::STAGE);
  auto key_begin = [&](int tile) { return k_begin + (tile * KA_WARPS + warp) * KA_KEYS; };
  // Of a batch of 32 tiles: -1 for a half behind the end or on a page that does not exist (its keys are left out).
  auto check_pages = [&](int first, int (&id)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (first + lane >= my_tiles || key_begin(first + lane) + 16 * h >= k_end) {
        id[h] = -1;
      } else if (static_cast<unsigned>(id[h]) >= static_cast<unsigned>(a.c.n_pages)) {
        id[h] = -1;
        if (a.err_word) atomicExch(a.err_word, 2);
      }
    }
  };
  check_pages(0, id_cur);
  // the next batch is fetched a batch ahead
  if (my_tiles > 32) { fetch_pages(32, id_nxt); check_pages(32, id_nxt); }

  // The codes of 16 keys of a page are HD * 8 contiguous bytes, their scales HD; a tile lies in one page unless pages have 16
  // keys.  All rows of a page can be read, and page 0 stands in for one that does not exist: keys that do not count are masked
  // later.  Rows of the pool are numbered in 32 bits, so an address is one multiplication.
  constexpr int NLD = HD / 64;
  const uint32_t dst_k = k_chunk<HD>(lane / (HD / 32), lane % (HD / 32));
  const uint32_t dst_v = SM::CODES + v_chunk<HD>(lane / (HD / 32), lane % (HD / 32));
  const uint32_t page_rows = static_cast<uint32_t>(a.n_kv_heads) << l2p, head_row = static_cast<uint32_t>(kvh) << l2p;
  const uint8_t* const k_base = a.c.k + lane * 16;
  const uint8_t* const v_base = a.c.v + lane * 16;
  // scales: a chunk of 16 bytes per lane, [K or V][chunk]
  constexpr int SC = HD / 8;
  const int sc_kv = (lane / SC) & 1, sc_chunk = lane % SC, sc_half = sc_chunk / (SC / 2);
  const uint8_t* const s_base = (sc_kv ? a.c.v_scale : a.c.k_scale) + sc_chunk * 16 - (l2p > 4 ? 0 : sc_half * HD);
  const uint32_t dst_s = 2 * SM::CODES + sc_kv * SM::SCALES + sc_chunk * 16;
  uint32_t valid = 0;  // of the tiles in flight, two bits each (the newest in bits 0-1): halves with keys
  auto load_tile = [&](int i, uint32_t to) {
    if (i > 0 && (i & 31) == 0) { id_cur[0] = id_nxt[0]; id_cur[1] = id_nxt[1]; }
    const int id0 = __shfl_sync(0xffffffffu, id_cur[0], i & 31), id1 = __shfl_sync(0xffffffffu, id_cur[1], i & 31);
    valid = (valid << 2) | (id0 >= 0 ? 1u : 0u) | (id1 >= 0 ? 2u : 0u);
    const uint32_t row = static_cast<uint32_t>(max(id0, 0)) * page_rows + head_row + (key_begin(i) & ((1 << l2p) - 1));
    const uint32_t to_k = to + dst_k, to_v = to + dst_v;
    const uint8_t* const k0 = k_base + static_cast<uint64_t>(row) * (HD / 2);
    const uint8_t* const v0 = v_base + static_cast<uint64_t>(row) * (HD / 2);
    if (l2p > 4) {
#pragma unroll
      for (int n = 0; n < 2 * NLD; ++n) {
        cp_async(to_k + 512 * n, k0 + 512 * n);
        cp_async(to_v + 512 * n, v0 + 512 * n);
      }
      if (lane < 2 * SC) cp_async(to + dst_s, s_base + static_cast<uint64_t>(row) * (HD / 16));
    } else {
      const uint32_t row1 = static_cast<uint32_t>(max(id1, 0)) * page_rows + head_row;
      const uint8_t* const k1 = k_base + static_cast<uint64_t>(row1) * (HD / 2);
      const uint8_t* const v1 = v_base + static_cast<uint64_t>(row1) * (HD / 2);
#pragma unroll
      for (int n = 0; n < NLD; ++n) {
        cp_async(to_k + 512 * n, k0 + 512 * n);
        cp_async(to_k + HD * 8 + 512 * n, k1 + 512 * n);
        cp_async(to_v + 512 * n, v0 + 512 * n);
        cp_async(to_v + HD * 8 + 512 * n, v1 + 512 * n);
      }
      if (lane < 2 * SC) cp_async(to + dst_s, s_base + static_cast<uint64_t>(sc_half ? row1 : row) * (HD / 16));
    }
  };
  uint32_t stage_in = ring, stage_out = ring;  // where the next tile goes, and the next one is taken from
  auto next_stage = [&](uint32_t& at) { at = at == ring + (KA_STAGES - 1) * SM::STAGE ? ring : at + SM::STAGE; };
#pragma unroll
  for (int s = 0; s < KA_STAGES - 1; ++s) {
    if (s < my_tiles) load_tile(s, stage_in); else valid <<= 2;
    next_stage(stage_in);
    ptx::cp_async_commit();
  }

  // Q^T as f16 operand fragments, every head scaled by a power of two so that its largest entry lies in [1, 2).  With two groups of
  // columns they stay in shared memory, the same for all warps.
  __shared__ __align__(16) uint4 q_frag[NC == 1 ? 1 : NC][KS / 2][NC == 1 ? 1 : 32];  // of a pair of k-steps
  uint4 qb[KS / 2];
  uint64_t f_pair[NC];  // of the scores of this lane's columns of S^T and O^T, 8 c + 2 t4 and the next, in log2 units
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float x[KS / 2][8], amax = 0.f;
#pragma unroll
    for (int s = 0; s < KS / 2; ++s) {
      unpack8(qw[c][s], x[s]);
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[s][e]));
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    // 2^e <= amax < 2^(e+1), e kept where 2^e and 2^-e are normal (an infinite q stays infinite)
    const int e = min(max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -126), 126);
    const float inv = pow2f(-e);
    const float scale = rsqrtf(static_cast<float>(HD)) * LOG2E * pow2f(e) * pow2f(kv4_exp(a.c.k_exp, kvh));
#pragma unroll
    for (int s = 0; s < KS / 2; ++s) {
      qb[s] = make_uint4(pack_f16(x[s][0] * inv, x[s][1] * inv), pack_f16(x[s][2] * inv, x[s][3] * inv),
                         pack_f16(x[s][4] * inv, x[s][5] * inv), pack_f16(x[s][6] * inv, x[s][7] * inv));
      if (NC > 1 && warp == 0) q_frag[c][s][lane] = qb[s];
    }
    f_pair[c] = ptx::pack_f32x2(__shfl_sync(0xffffffffu, scale, t4 * 8), __shfl_sync(0xffffffffu, scale, t4 * 8 + 4));
  }
  const uint32_t q_at = NC > 1 ? ptx::smem_u32(&q_frag[0][0][NC == 1 ? 0 : lane]) : 0;
  if (NC > 1) __syncthreads();

  float o_acc[NC][MT][4];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < MT; ++i) o_acc[c][i][0] = o_acc[c][i][1] = o_acc[c][i][2] = o_acc[c][i][3] = 0.f;
  // Per column pair: reference of the exponent (uniform over the lanes of a head; -inf: no key yet), what is added to a score for
  // it, and this lane's share of the sum
  float m_ref[NC][2];
  uint64_t shift[NC], l_sum[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m_ref[c][0] = m_ref[c][1] = -CUDART_INF_F;
    shift[c] = ptx::pack_f32x2(P_SHIFT, P_SHIFT);  // (no key yet: every p is 0)
    l_sum[c] = ptx::pack_f32x2(0.f, 0.f);
  }
  bool nan_seen = false;

  for (int i = 0; i < my_tiles; ++i) {
    if (i > 0 && (i & 31) == 0 && i + 32 < my_tiles) { fetch_pages(i + 32, id_nxt); check_pages(i + 32, id_nxt); }
    if (i + KA_STAGES - 1 < my_tiles) load_tile(i + KA_STAGES - 1, stage_in); else valid <<= 2;
    next_stage(stage_in);
    ptx::cp_async_commit();
    ptx::cp_async_wait<KA_STAGES - 1>();
    __syncwarp();
    const uint32_t sk = stage_out, sv = sk + SM::CODES, ssk = sv + SM::CODES, ssv = ssk + SM::SCALES;
    const int key0 = key_begin(i), halves = static_cast<int>((valid >> (2 * (KA_STAGES - 1))) & 3u);
    const bool masked = (MULTI ? min(k_end, pos0 + 1) : k_end) - key0 < KA_KEYS || halves != 3;
    if (masked) {
      // V of keys that do not count is multiplied with weights of 0, and 0 * NaN is NaN: their scales become 0.  Of keys that
      // some tokens of the block see and others do not, scales that are NaN do, and the rows that see the key are given their NaN
      // at the end.  A key per lane.
      const bool counts = key0 + lane < k_end && (halves >> (lane >> 4)) & 1;
#pragma unroll
      for (int n = 0; n < HD / 64; ++n) {
        const uint32_t at = ssv + lane * (HD / 16) + 4 * n, w = lds32(at);
        bool seen = false;
        const uint32_t d = !counts ? 0u : MULTI && key0 + lane > pos0 ? drop_nans(w, seen) : w;
        if (d != w) asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(d) : "memory");
        nan_seen |= seen;
      }
      __syncwarp();
    }

    // ---- S^T = K Q^T: rows are keys key_of(g) and 8 + key_of(g) of each half, columns (token, head) pairs
    float x[2][NC][4];  // [half][column group][key half][column] = (e >> 1, e & 1)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float st[NC][2][4];
      uint32_t w[2][W], sc[2][2];  // rows g, g + 8: codes and scales (as pairs of equal halves)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t row = sk + (16 * h + 8 * r + g) * (HD / 2), srow = ssk + (16 * h + 8 * r + key_of(g)) * (HD / 16);
        if (HD == 128) {
          const uint4 v = lds128(row + t4 * 16);
          w[r][0] = v.x; w[r][1] = v.y; w[r][W - 2] = v.z; w[r][W - 1] = v.w;
          const uint32_t s2 = e4m3x2_to_f16x2(static_cast<uint16_t>(lds16(srow + t4 * 2)));
          sc[r][0] = __byte_perm(s2, 0, 0x1010);
          sc[r][1] = __byte_perm(s2, 0, 0x3232);
        } else {
          const uint2 v = lds64(row + t4 * 8);
          w[r][0] = v.x; w[r][1] = v.y;
          const uint32_t s1 = lds8(srow + t4);
          sc[r][0] = sc[r][1] = e4m3x2_to_f16x2(static_cast<uint16_t>(s1 | (s1 << 8)));
        }
      }
#pragma unroll
      for (int j = 0; j < W; ++j) {
        uint32_t a0[4], a1[4];
        e2m1_to_f16(w[0][j], a0);
        e2m1_to_f16(w[1][j], a1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a0[e] = mul_f16x2(a0[e], sc[0][j / 2]);
          a1[e] = mul_f16x2(a1[e], sc[1][j / 2]);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const uint4 b = NC > 1 ? lds128(q_at + (c * (KS / 2) + j) * 512) : qb[j];
          if (j == 0) {
            mma_f16_first(st[c][0], a0[0], a1[0], a0[1], a1[1], b.x, b.y);
            mma_f16_first(st[c][1], a0[2], a1[2], a0[3], a1[3], b.z, b.w);
          } else {
            mma_f16(st[c][0], a0[0], a1[0], a0[1], a1[1], b.x, b.y);
            mma_f16(st[c][1], a0[2], a1[2], a0[3], a1[3], b.z, b.w);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; e += 2)
          ptx::unpack_f32x2(ptx::mul_f32x2(ptx::add_f32x2(ptx::pack_f32x2(st[c][0][e], st[c][0][e + 1]),
                                                          ptx::pack_f32x2(st[c][1][e], st[c][1][e + 1])), f_pair[c]),
                            x[h][c][e], x[h][c][e + 1]);
    }
    // ---- softmax
    if (masked) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          // the last key of the tile that the column's token sees
          const int last = (MULTI ? min(pos0 + token_of(8 * c + 2 * t4 + e), k_end - 1) : k_end - 1) - key0;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int lim = (halves >> h) & 1 ? last - 16 * h : -1;
            if (key_of(g) > lim) x[h][c][e] = -CUDART_INF_F;
            if (8 + key_of(g) > lim) x[h][c][2 + e] = -CUDART_INF_F;
          }
        }
      }
    }
    // the reference follows the maximum only when that has grown by more than P_SLACK (always at the first key)
    float mx[NC][2];
    bool grow = false;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mx[c][e] = fmaxf(ptx::fmax3(x[0][c][e], x[0][c][2 + e], x[1][c][e]), x[1][c][2 + e]);
        grow |= mx[c][e] > m_ref[c][e] + P_SLACK;
      }
    }
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float corr[2], add[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float m = mx[c][e];
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
          const float m_new = fmaxf(m_ref[c][e], m);
          corr[e] = m_new == -CUDART_INF_F ? 1.f : ptx::ex2_approx(m_ref[c][e] - m_new);
          add[e] = P_SHIFT - (m_new == -CUDART_INF_F ? 0.f : m_new);
          m_ref[c][e] = m_new;
#pragma unroll
          for (int n = 0; n < MT; ++n) { o_acc[c][n][e] *= corr[e]; o_acc[c][n][2 + e] *= corr[e]; }
        }
        shift[c] = ptx::pack_f32x2(add[0], add[1]);
        l_sum[c] = ptx::mul_f32x2(l_sum[c], ptx::pack_f32x2(corr[0], corr[1]));
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t pb[NC][2];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float y0, y1;
          // (the rounded score, which is what the reference was taken from: very large ones would not cancel otherwise)
          ptx::unpack_f32x2(ptx::add_f32x2(ptx::pack_f32x2(x[h][c][2 * k], x[h][c][2 * k + 1]), shift[c]), y0, y1);
          y0 = ptx::ex2_approx(y0);
          y1 = ptx::ex2_approx(y1);
          l_sum[c] = ptx::add_f32x2(l_sum[c], ptx::pack_f32x2(y0, y1));
          // P^T as an operand: the transpose of the accumulator's 8 x 8 blocks
          pb[c][k] = transpose8x8(pack_f16(y0, y1));
        }
      }
      // ---- O^T += V^T P^T: this lane's keys are key_of(2 t4), key_of(2 t4 + 1) = t4, t4 + 4 of both 8-key groups, its features
      // g * hd / 8 ..; two keys share a word's nibbles, low and high
      uint32_t vw[4][W / 2], sv2[2], sb[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * h + (r >> 1) * 8 + t4 + (r & 1) * 4;
        if (HD == 128) {
          const uint2 v = lds64(sv + v_chunk<HD>(row, g >> 1) + (g & 1) * 8);
          vw[r][0] = v.x; vw[r][W / 2 - 1] = v.y;
        } else {
          vw[r][0] = lds32(sv + row * (HD / 2) + g * 4);
        }
        sb[r] = lds8(ssv + row * (HD / 16) + (HD == 128 ? g : g >> 1));
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) sv2[k] = e4m3x2_to_f16x2(static_cast<uint16_t>(sb[2 * k] | (sb[2 * k + 1] << 8)));
#pragma unroll
      for (int j = 0; j < W / 2; ++j) {
        uint32_t even[2][4], odd[2][4];  // [8-key group]: features 8 j + 2 n and 8 j + 2 n + 1 of two keys
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t w0 = vw[2 * k][j], w1 = vw[2 * k + 1][j];
          e2m1_to_f16((w0 & 0x0f0f0f0fu) | ((w1 << 4) & 0xf0f0f0f0u), even[k]);
          e2m1_to_f16(((w0 >> 4) & 0x0f0f0f0fu) | (w1 & 0xf0f0f0f0u), odd[k]);
#pragma unroll
          for (int n = 0; n < 4; ++n) { even[k][n] = mul_f16x2(even[k][n], sv2[k]); odd[k][n] = mul_f16x2(odd[k][n], sv2[k]); }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int c = 0; c < NC; ++c) mma_f16(o_acc[c][4 * j + n], even[0][n], odd[0][n], even[1][n], odd[1][n], pb[c][0], pb[c][1]);
      }
    }
    next_stage(stage_out);
    __syncwarp();  // every lane has read this stage before it is refilled
  }
  ptx::cp_async_wait<0>();
  float l_col[NC][2];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    ptx::unpack_f32x2(l_sum[c], l_col[c][0], l_col[c][1]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l_col[c][h] += __shfl_xor_sync(0xffffffffu, l_col[c][h], o);
  }
  // Merge: the warps agree on the maximum of every column, scale what they have to it, and add up in shared memory.
  constexpr int RS = SM::MERGE_ROW;
  float* const mrg = reinterpret_cast<float*>(smem);
  float* const m_all = mrg + KA_WARPS * KA_COLS * RS;  // [column][warp]
  float2* const ml = reinterpret_cast<float2*>(m_all + KA_WARPS * KA_COLS);
  __syncthreads();  // every warp has left its ring: the memory is reused
  if (g == 0) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      m_all[(8 * c + t4 * 2) * KA_WARPS + warp] = m_ref[c][0];
      m_all[(8 * c + t4 * 2 + 1) * KA_WARPS + warp] = m_ref[c][1];
    }
  }
  __syncthreads();
  auto column_max = [&](int col) {
    float m = m_all[col * KA_WARPS];
#pragma unroll
    for (int w = 1; w < KA_WARPS; ++w) m = fmaxf(m, m_all[col * KA_WARPS + w]);
    return m;
  };
  const float o_unit = P_UNIT * pow2f(kv4_exp(a.c.v_exp, kvh));
#pragma unroll
  for (int c = 0; c < NC; ++c) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int col = 8 * c + t4 * 2 + h;
      if (col < n_cols) {
        const float m = column_max(col);
        const float f = m == -CUDART_INF_F ? 1.f : ptx::ex2_approx(m_ref[c][h] - m), fo = f * o_unit;  // 0 for a warp that saw no key
        float* const dst_row = mrg + (warp * KA_COLS + col) * RS;
#pragma unroll
        for (int n = 0; n < MT; ++n)
          *reinterpret_cast<float2*>(dst_row + g * (HD / 8) + 2 * n) = make_float2(o_acc[c][n][h] * fo, o_acc[c][n][2 + h] * fo);
        if (g == 0) dst_row[HD] = l_col[c][h] * (f * P_UNIT);
      }
    }
  }
  const bool nans = MULTI ? __syncthreads_or(nan_seen) : (__syncthreads(), false);
  const bool pairs = (reinterpret_cast<uintptr_t>(a.o) & 3u) == 0;
  auto store_out = [&](size_t row, int d, const float4& o, float l) {
    const float inv = l == 0.f ? 0.f : 1.f / l;  // (no visible entry: zeros)
    const uint32_t lo = ptx::pack_bf16(o.x * inv, o.y * inv), hi = ptx::pack_bf16(o.z * inv, o.w * inv);
    bf16* const dst = a.o + row * HD + d;
    if (pairs) {
      reinterpret_cast<uint32_t*>(dst)[0] = lo;
      reinterpret_cast<uint32_t*>(dst)[1] = hi;
    } else {  // results that start between two words
      uint16_t* const dst16 = reinterpret_cast<uint16_t*>(dst);
      dst16[0] = static_cast<uint16_t>(lo); dst16[1] = static_cast<uint16_t>(lo >> 16);
      dst16[2] = static_cast<uint16_t>(hi); dst16[3] = static_cast<uint16_t>(hi >> 16);
    }
  };
  for (int idx = tid * 4; idx < n_cols * HD; idx += KA_THREADS * 4) {  // four neighbouring features of a column
    const int r = idx / HD, d = idx - r * HD;
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < KA_WARPS; ++w) {
      const float* src = mrg + (w * KA_COLS + r) * RS;
      const float4 v = *reinterpret_cast<const float4*>(src + d);
      l += src[HD];
      o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
    }
    const size_t row = out_row(r);
    if (MULTI && nans) {
      for (int key = max(pos0 + 1, k_begin); key <= min(pos0 + token_of(r), k_end - 1); ++key) {
        const int id = table[key >> l2p];
        if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.c.n_pages)) continue;
        const size_t at = ((static_cast<size_t>(id) * a.n_kv_heads + kvh) << l2p) + (key & ((1 << l2p) - 1));
        if ((a.c.v_scale[at * (HD / 16) + d / 16] & 0x7f) == 0x7f) o = make_float4(CUDART_NAN_F, CUDART_NAN_F, CUDART_NAN_F, CUDART_NAN_F);
      }
    }
    if (!TOGETHER && a.n_splits == 1) {
      store_out(row, d, o, l);
    } else if (TOGETHER) {
      *reinterpret_cast<float4*>(mrg + r * RS + d) = o;  // (the first warp's row: read by this thread alone, but for l behind it)
      if (d == 0) ml[r] = make_float2(column_max(r), l);
    } else {
      *reinterpret_cast<float4*>(a.parts.o + (part_row0 + row) * HD + d) = o;
      if (d == 0) a.parts.ml[part_row0 + row] = make_float2(column_max(r), l);
    }
  }
  if (!TOGETHER) return;
  // The parts that have keys meet (those without have left: a barrier does not wait for them), and each joins a share of the rows
  // over all of them.
  const int n_parts = min(a.n_splits, max(1, static_cast<int>((static_cast<uint32_t>(total) + a.chunk - 1) / a.chunk)));
  __syncwarp();
  ptx::cluster_sync_all();
  for (int idx = (split * KA_THREADS + tid) * 4; idx < n_cols * HD; idx += n_parts * KA_THREADS * 4) {
    const int r = idx / HD, d = idx - r * HD;
    const uint32_t ml_at = ptx::smem_u32(ml + r), o_at = ptx::smem_u32(mrg + r * RS + d);
    float m[KA_CLUSTER], ls[KA_CLUSTER], m_max = -CUDART_INF_F;
    float4 v[KA_CLUSTER];
#pragma unroll
    for (int x = 0; x < KA_CLUSTER; ++x) {
      m[x] = -CUDART_INF_F; ls[x] = 0.f; v[x] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (x < n_parts) {
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m[x]), "=f"(ls[x]) : "r"(ptx::map_to_cta(ml_at, x)) : "memory");
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(v[x].x), "=f"(v[x].y), "=f"(v[x].z), "=f"(v[x].w) : "r"(ptx::map_to_cta(o_at, x)) : "memory");
      }
    }
#pragma unroll
    for (int x = 0; x < KA_CLUSTER; ++x) m_max = fmaxf(m_max, m[x]);
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int x = 0; x < KA_CLUSTER; ++x) {
      if (x < n_parts) {
        const float f = m_max == -CUDART_INF_F ? 1.f : ptx::ex2_approx(m[x] - m_max);
        l = fmaf(ls[x], f, l);
        o.x = fmaf(v[x].x, f, o.x); o.y = fmaf(v[x].y, f, o.y); o.z = fmaf(v[x].z, f, o.z); o.w = fmaf(v[x].w, f, o.w);
      }
    }
    store_out(out_row(r), d, o, l);
  }
  __syncwarp();
  ptx::cluster_sync_all();  // nobody leaves before its rows are read
}

template <int HD, int WARPS, int NC, bool MULTI, bool TOGETHER>
pd_status launch_kv4(const Kv4DecodeArgs& a, int batch, cudaStream_t s) {
  using SM = Kv4Smem<HD, WARPS, NC>;
  const auto kernel = kv4_decode_kernel<HD, WARPS, NC, MULTI, TOGETHER>;
  static PerDeviceInt smem_opt_in;
  PD_TRY(opt_in_smem(smem_opt_in, kernel, SM::BYTES));
  const dim3 grid(a.col_blocks * a.n_kv_heads, batch, a.n_splits), block(WARPS * 32);
  if (TOGETHER) {
    PD_CUDA_TRY(launch_pdl_cluster(kernel, grid, block, dim3(1, 1, a.n_splits), SM::BYTES, s, a));
  } else {
    PD_CUDA_TRY(launch_pdl(kernel, grid, block, SM::BYTES, s, a));
  }
  count_launch();
  if (!TOGETHER && a.n_splits > 1) return launch_paged_join(a.parts, a.o, 1ll * a.rows * a.n_q_heads, a.n_splits, HD, s);
  return PD_OK;
}
template <int HD, int WARPS, int NC>
pd_status launch_kv4(const Kv4DecodeArgs& a, int batch, bool together, cudaStream_t s) {
  if (a.n_new > 1) return together ? launch_kv4<HD, WARPS, NC, true, true>(a, batch, s) : launch_kv4<HD, WARPS, NC, true, false>(a, batch, s);
  return together ? launch_kv4<HD, WARPS, NC, false, true>(a, batch, s) : launch_kv4<HD, WARPS, NC, false, false>(a, batch, s);
}
struct Split { int n, chunk, warps; bool together; };
template <int HD>
pd_status launch_kv4(const Kv4DecodeArgs& a, int batch, int col_groups, const Split& sp, cudaStream_t s) {
  if (col_groups == 2) return launch_kv4<HD, 4, 2>(a, batch, sp.together, s);
  return sp.warps == 4 ? launch_kv4<HD, 4, 1>(a, batch, sp.together, s) : launch_kv4<HD, 8, 1>(a, batch, sp.together, s);
}

// Key ranges are cut into equal parts while there are fewer blocks than run together, into parts of at least KA_MIN_CHUNK keys.
// The sequences of a batch may differ in length, which the host does not know, so a part is at most 4096 keys, and from 149
// blocks on more parts than would run together even the lengths out.  With 16 equal sequences and two tokens, 128 blocks, these cost more than
// they bring (28 us, 20 without), with 16 ragged ones of up to 4,000 keys less (26 and 29).  They are half as many again, or, for bounds of 4096
// keys on, twice as many, in us:
//   bounds of 4,096 keys and more   24 ragged, two tokens 34 and 30   20 of 4,095 keys 32 and 29   40 of 4,095 keys 48 and 45
//   bounds below                    64 of 2,000 keys 36 and 41        64 of 3,900 keys 63 and 61   64 ragged, to 4,095 keys, 58 and 50
// so the border is drawn for the sake of short equal sequences.  No more than 16 parts (and what is left) are made for the length
// alone, since max_kv_len may be a capacity far above the lengths.  A capacity has its price all the same, for parts are cut by it and
// the join looks at all of them: 256 sequences of 2,304 keys 119 us with that bound, 125 with 4,096, 129 with 8,192 and 151 with
// 32,768; 24 ragged ones of up to 4,352 keys, two tokens, 31, 42 (8,192) and 62 (32,768); 8 of 2,000 keys 8.8, 12 (4,096) and 19 (32,768).
// Blocks have 4 warps, which costs a short stream of tiles less at both ends (256 sequences of 2,304 keys 117 to 126 us, 133 with 8; 20 of 4,095 29
// and 31; but 64 ragged ones 58 and 52), or 8 where the keys of a block are cut into many parts, of which there are half as many to join (one
// sequence of 32,768 keys 20 us with 4 and 16 with 8; 8 of 8,000 22.8 and 22.2).
// Up to KA_CLUSTER parts that all run at once, with some room (a cluster's blocks need places in one part of the GPU), are a cluster
// and join in shared memory instead of in a kernel of their own (8 sequences of 2,000 keys: 10.6 and 8.7 us; 16 of 1,000: 10.7 and 9.0; 18
// of 3,000, 97 % of what runs at once: 21.2 and 24.0), and nine or ten parts are made at most eight for it (4 of 4,000: 10.8 and 9.1; two of
// 4,000, sixteen made eight: 7.6 and 8.7).  Where more blocks than that wait for a place, blocks that end one by one are
// better (24 ragged sequences: 30 and 42 us).
// The kernel that joins reads KA_JOIN_ROUND parts at a time, so 33 to 40 are made that many at most: one sequence of 32,768 keys, 37
// parts 17.0 us, 32 parts 16.3; one of 64,000 with 64 / 8 heads 25.7 and 24.7.  (Parts are whole steps of 64 keys, so 36 parts of 256 become 29 of 320: one of
// 9,000 keys 9.0 us, 9.2 with 29.)
constexpr int KA_FEW_BLOCKS = 74, KA_MORE_PARTS = 2, KA_JOIN_ROUND = 32;
Split kv4_split(long long blocks, int col_groups, int batch, int max_kv_len) {
  Split sp;
  sp.warps = col_groups == 1 && blocks <= KA_FEW_BLOCKS ? 8 : 4;
  const long long resident = ka_resident_warps(col_groups) / sp.warps;
  const long long most = blocks <= 148 ? resident : max_kv_len >= 4096 ? resident * KA_MORE_PARTS : resident * 3 / 2;
  const long long want = std::max(1ll, most / blocks);
  long long chunk = (max_kv_len + want - 1) / want;
  chunk = std::min(chunk, batch > 1 ? std::max(4096ll, max_kv_len / 16ll) : static_cast<long long>(max_kv_len));
  auto in_steps = [](long long keys) { return std::min((std::max<long long>(keys, KA_MIN_CHUNK) + 63) / 64 * 64, 0x7fffffc0ll); };
  auto parts = [&] { return (max_kv_len + chunk - 1) / chunk; };
  chunk = in_steps(chunk);
  auto fits = [&](long long n) { return blocks * n * 8 <= resident * 7; };
  for (const int n : {KA_CLUSTER, KA_JOIN_ROUND})
    if (parts() > n && parts() <= n * 5 / 4 && (n > KA_CLUSTER || fits(n))) chunk = in_steps((max_kv_len + n - 1ll) / n);
  sp.n = static_cast<int>(parts());
  sp.chunk = static_cast<int>(chunk);
  sp.together = sp.n > 1 && sp.n <= KA_CLUSTER && fits(sp.n);
  return sp;
}
// (part, row) pairs, row = (token, query head), that any call of up to these sizes has at most, where it has parts at all: a
// buffer of that size serves every smaller call, too.  Parts made to fill the GPU are at most as many blocks of 16 rows as
// kv4_split asks for (two groups of columns; of one, fewer rows), of at least KA_MIN_CHUNK keys; parts made for their length are as many as the bound allows.
long long kv4_most_part_rows(int batch, int n_new, int n_q_heads, int max_kv_len) {
  if (batch <= 0 || n_new <= 0 || max_kv_len <= KA_MIN_CHUNK) return 0;
  const long long rows = 1ll * batch * n_new * n_q_heads;
  const long long fill = std::min(1ll * ka_resident_warps(2) / 4 * KA_MORE_PARTS * ka_cols(2), (max_kv_len + (KA_MIN_CHUNK - 1ll)) / KA_MIN_CHUNK * rows);
  // (17: of max_kv_len / 16 keys, rounded down, and what is left)
  const long long length = std::min(17ll, (max_kv_len + 4095ll) / 4096);
  return std::max(fill, length > 1 ? length * rows : 0);
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_paged_kv4_decode_attention_workspace_bytes(const pd_layer_cfg* cfg, int32_t B, int32_t n_new, int32_t max_kv_len,
                                                                   size_t* out_bytes) {
  PD_TRY(pd::check_kv4_heads(cfg));
  if (!out_bytes || B < 0 || n_new < 1 || max_kv_len < 0) return PD_ERR_INVALID_ARG;
  const long long rows = pd::kv4_most_part_rows(B, n_new, cfg->n_q_heads, max_kv_len);
  *out_bytes = rows ? pd::paged_parts_bytes(static_cast<size_t>(rows), cfg->head_dim) : 0;
  return PD_OK;
}

extern "C" pd_status pd_paged_kv4_decode_attention(const pd_layer_cfg* cfg, const void* q, int32_t ldq, void* out,
                                                   const int32_t* kv_len_dev, int32_t B, int32_t n_new, int32_t max_kv_len,
                                                   const pd_paged_kv4_cache* cache, void* workspace, size_t workspace_bytes,
                                                   int32_t* err_word, void* stream) {
  using namespace pd;
  PD_TRY(check_kv4_heads(cfg));
  Kv4DecodeArgs a{};
  PD_TRY(kv4_cache_view(cache, cfg->n_kv_heads, &a.c));
  if (B < 0 || B > cache->n_seqs || n_new < 1) return PD_ERR_INVALID_ARG;
  if (B == 0) return PD_OK;
  if (!q || !out || !kv_len_dev || ldq < 1ll * cfg->n_q_heads * cfg->head_dim || ldq % 8 != 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) & 15u) || (reinterpret_cast<uintptr_t>(out) & 1u)) return PD_ERR_INVALID_ARG;
  if (max_kv_len < n_new || max_kv_len > (cache->table_ld << a.c.log2_page)) return PD_ERR_INVALID_ARG;
  const long long pairs = 1ll * n_new * (cfg->n_q_heads / cfg->n_kv_heads);
  if (B > 65535 || n_new > 65535 || 1ll * B * n_new * cfg->n_q_heads > 0x7fffffffll) return PD_ERR_UNSUPPORTED_SHAPE;
  const int col_groups = pairs > 8 ? 2 : 1;
  a.col_blocks = static_cast<int>((pairs + ka_cols(col_groups) - 1) / ka_cols(col_groups));
  a.rows = B * n_new;
  const Split sp = kv4_split(1ll * B * a.col_blocks * cfg->n_kv_heads, col_groups, B, max_kv_len);
  a.n_splits = sp.n; a.chunk = sp.chunk;
  if (a.n_splits > 1) {
    const size_t part_rows = static_cast<size_t>(a.n_splits) * a.rows * cfg->n_q_heads;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PD_ERR_INVALID_ARG;
    if (workspace_bytes < paged_parts_bytes(part_rows, cfg->head_dim)) return PD_ERR_WORKSPACE_TOO_SMALL;
    a.parts.o = static_cast<float*>(workspace);
    a.parts.ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + paged_parts_ml_offset(part_rows, cfg->head_dim));
  }
  a.q = static_cast<const bf16*>(q); a.o = static_cast<bf16*>(out); a.kv_len = kv_len_dev; a.err_word = err_word;
  a.ldq = ldq; a.n_new = n_new; a.n_q_heads = cfg->n_q_heads; a.n_kv_heads = cfg->n_kv_heads;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_ATTN_DECODE, st);
  return cfg->head_dim == 128 ? launch_kv4<128>(a, B, col_groups, sp, st) : launch_kv4<64>(a, B, col_groups, sp, st);
}
