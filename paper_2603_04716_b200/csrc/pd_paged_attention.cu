// Attention over the 8-bit paged KV cache: one query token per sequence (pd_paged_decode_attention) and the fresh rows of
// ragged requests (pd_paged_prefill_attention).
//
// Decode.  o = softmax(q K^T / sqrt(hd)) V per query head over the sequence's pages; K and V of a page are E4M3 codes times
// one power of two.  HBM-bound: every code byte is read once.  One block per (split of the key range, KV head, sequence);
// every warp streams its own 16-key tiles through a private cp.async ring (a tile never crosses a page, so it has one page
// number and one pair of scales).
//   S^T = K Q^T    m16n8k16 in f16: rows are 16 keys, columns 8 heads of the group.
//   O^T = V^T P^T  m16n8k16: rows are features, columns 8 heads.  Heads are columns, so a group of at most 8 wastes no
//                  product (a legacy tensor instruction suffices: both products of a tile are 16 instructions for 4 KB).
// E4M3 -> f16 is exact and one instruction for two codes.  The contraction order of a product is free, so a lane takes 16
// neighbouring features of a K row as its share of four k-steps, and 16 neighbouring features of four V rows (byte-permuted
// into pairs of keys): all shared-memory reads are 16 bytes wide, and the row order within a group of 8 keys is chosen so
// that they are free of bank conflicts.  q is scaled by a power of two per head into f16 range.  The reference of the
// exponent follows the maximum lazily, so a tile costs one vote instead of a reduction over its keys.  Softmax statistics
// and O are fp32; K's scale is applied to the scores, V's to the weights, relative to the largest V scale so far.
#include <math_constants.h>

#include "pd_paged.cuh"

namespace pd {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

struct PagedDecodeArgs {
  const bf16* q;          // [B, ldq]
  bf16* o;                // [B, Hq*hd]
  const int32_t* kv_len;  // [B]
  float* partial;         // when n_splits > 1: outputs [B, Hkv, n_splits, G, hd], then (max, sum) pairs [B, Hkv, n_splits, G]
  int* err_word;
  PagedCache c;
  int ldq, batch, n_q_heads, n_kv_heads;
  int n_splits, chunk;    // block x covers keys x * chunk .. (the last one whatever lies behind); chunk is a multiple of 64
};

constexpr int PA_WARPS = 8;
constexpr int PA_THREADS = PA_WARPS * 32;
constexpr int PA_KEYS = 16;
constexpr int PA_STAGES = 3;
// p is kept as 2^7 p relative to a reference that may lag the running maximum by 2^8: at most 2^15, below f16's 65504.
constexpr float P_SHIFT = 7.f, P_SLACK = 8.f, P_UNIT = 1.f / 128.f;
constexpr int PA_MIN_CHUNK = 256;               // keys of a run at least
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
// Entries of sequence b that the call attends to.
__device__ __forceinline__ int visible_keys(const PagedDecodeArgs& a, int b) {
  const int cap = a.c.table_ld << a.c.log2_page, len = a.kv_len[b];
  return len >= cap ? cap : max(len + 1, 0);
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

// WIDE: groups of 9 to 16 query heads (two column groups in both products).
template <int HD, bool WIDE>
__global__ void __launch_bounds__(PA_THREADS, WIDE ? 1 : 2) paged_decode_kernel(const PagedDecodeArgs a) {
  using SM = PagedSmem<HD>;
  constexpr int KS = HD / 16;          // k-steps of K Q^T
  constexpr int MT = HD / 16;          // 16-feature tiles of O^T
  constexpr int NC = WIDE ? 2 : 1;     // column groups of 8 heads
  extern __shared__ __align__(128) uint8_t smem[];
  const int split = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, t4 = lane & 3;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();

  const int l2p = a.c.log2_page;
  // Page numbers of 32 tiles of this warp at a time, a tile per lane.  The first 32 are read before the sequence's length is
  // known: entries behind its last page are read, too, but not used.
  const int32_t* table = a.c.table + static_cast<size_t>(b) * a.c.table_ld;
  const long long split_begin = 1ll * split * a.chunk;
  auto page_of = [&](int tile) { return (split_begin + (tile * PA_WARPS + warp) * PA_KEYS) >> l2p; };
  const long long first_page = page_of(lane);
  int id_cur = first_page < a.c.table_ld ? table[first_page] : -1;
  // q of head c * 8 + g: this lane's share of every k-step
  uint2 qw[NC][KS];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int s = 0; s < KS; ++s)
      qw[c][s] = c * 8 + g < group
                     ? *reinterpret_cast<const uint2*>(a.q + static_cast<size_t>(b) * a.ldq + (kvh * group + c * 8 + g) * HD +
                                                       (s >> 2) * 64 + t4 * 16 + (s & 3) * 4)
                     : make_uint2(0u, 0u);
  if (split == 0 && kvh == 0 && tid == 0 && a.err_word && a.kv_len[b] >= (a.c.table_ld << l2p)) atomicExch(a.err_word, 2);
  const int total = visible_keys(a, b);
  const int k_begin = static_cast<int>(min(1ll * total, 1ll * split * a.chunk));
  const int k_end = split == a.n_splits - 1 ? total : static_cast<int>(min(1ll * total, 1ll * k_begin + a.chunk));
  if (split > 0 && k_begin == k_end) return;  // (the merge knows how many splits hold keys)
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
  // This lane's columns of S^T and O^T are heads c * 8 + 2 t4 + h, h = 0, 1.
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
    const bool masked = key0 + PA_KEYS > k_end || ks < 0.f;
    float x[NC][4];  // [key half][head] = (e >> 1, e & 1)
    bool grow = false;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float f0 = f_head[c][0] * ks, f1 = f_head[c][1] * ks;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[c][e] = (st[c][0][e] + st[c][1][e]) * ((e & 1) ? f1 : f0);
      if (masked) {
        const int lim = ks < 0.f ? -1 : k_end - 1 - key0;
        if (key_of<HD>(g) > lim) x[c][0] = x[c][1] = -CUDART_INF_F;
        if (8 + key_of<HD>(g) > lim) x[c][2] = x[c][3] = -CUDART_INF_F;
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
      const int head = c * 8 + t4 * 2 + h;
      if (head < group) {
        float* dst_row = mrg + (warp * 16 + head) * RS;
#pragma unroll
        for (int n = 0; n < MT; ++n) {
          dst_row[g * (HD / 8) + 2 * n] = o_acc[c][n][h] * (unit * P_UNIT);
          dst_row[g * (HD / 8) + 2 * n + 1] = o_acc[c][n][2 + h] * (unit * P_UNIT);
        }
        if (g == 0) { dst_row[HD] = m_ref[c][h]; dst_row[HD + 1] = l_sum[c][h] * P_UNIT; }
      }
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
      const size_t row = ((static_cast<size_t>(b) * a.n_kv_heads + kvh) * a.n_splits + split) * group + r;
      a.partial[row * HD + d] = o;
      if (d == 0)
        reinterpret_cast<float2*>(a.partial + static_cast<size_t>(a.batch) * a.n_q_heads * a.n_splits * HD)[row] = make_float2(m, l);
    }
  }
}

// Merge of the splits: one block per (query head, sequence).  Every warp computes the weights of all splits (a split per
// lane), the warps share the splits' rows and add up in shared memory.  All loads of up to 32 splits are issued before
// the first is used; rows of splits that hold no keys are loaded, too, and left out.
constexpr int PC_WARPS = 4;

template <int HD>
__global__ void __launch_bounds__(PC_WARPS * 32) paged_combine_kernel(const PagedDecodeArgs a) {
  constexpr int V = HD / 32, NR = 32 / PC_WARPS;  // features per lane, rows per warp and round
  const int b = blockIdx.y, hq = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int kvh = hq / group, r = hq - kvh * group;
  __shared__ float acc[PC_WARPS][HD];
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const size_t row0 = (static_cast<size_t>(b) * a.n_kv_heads + kvh) * a.n_splits * group + r;
  const float2* ml = reinterpret_cast<const float2*>(a.partial + static_cast<size_t>(a.batch) * a.n_q_heads * a.n_splits * HD);
  float m_run = -CUDART_INF_F, l = 0.f, o_sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) o_sum[e] = 0.f;
  const int total = visible_keys(a, b);
  for (int s0 = 0; s0 < a.n_splits; s0 += 32) {
    float2 st = s0 + lane < a.n_splits ? ml[row0 + static_cast<size_t>(s0 + lane) * group] : make_float2(0.f, 0.f);
    float v[NR][V];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int s = s0 + i * PC_WARPS + warp;
#pragma unroll
      for (int e = 0; e < V; ++e) v[i][e] = 0.f;
      if (s < a.n_splits) {
        const float* src = a.partial + (row0 + static_cast<size_t>(s) * group) * HD + lane * V;
        if (V == 4) {
          const float4 w = *reinterpret_cast<const float4*>(src);
          v[i][0] = w.x; v[i][1] = w.y; v[i][V - 2] = w.z; v[i][V - 1] = w.w;
        } else {
          const float2 w = *reinterpret_cast<const float2*>(src);
          v[i][0] = w.x; v[i][1] = w.y;
        }
      }
    }
    const bool held = 1ll * (s0 + lane) * a.chunk < total;  // the split holds keys (so its row was written)
    if (!held) st = make_float2(-CUDART_INF_F, 0.f);
    float m = fmaxf(m_run, st.x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float m_use = m == -CUDART_INF_F ? 0.f : m;
    const float corr = exp2f(m_run - m_use), f_lane = exp2f(st.x - m_use);
    m_run = m;
    l = l * corr + st.y * f_lane;
#pragma unroll
    for (int e = 0; e < V; ++e) o_sum[e] *= corr;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int s = i * PC_WARPS + warp;
      const float f = __shfl_sync(0xffffffffu, f_lane, s);
      if (1ll * (s0 + s) * a.chunk < total) {
#pragma unroll
        for (int e = 0; e < V; ++e) o_sum[e] = fmaf(v[i][e], f, o_sum[e]);
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
  for (int e = 0; e < V; ++e) acc[warp][lane * V + e] = o_sum[e];
  __syncthreads();
  if (threadIdx.x < HD) {
    const float o = (acc[0][threadIdx.x] + acc[1][threadIdx.x]) + (acc[2][threadIdx.x] + acc[3][threadIdx.x]);
    // no visible entry: zeros
    a.o[static_cast<size_t>(b) * (a.n_q_heads * HD) + hq * HD + threadIdx.x] = __float2bfloat16(l == 0.f ? 0.f : o / l);
  }
}

template <int HD, bool WIDE>
pd_status launch_decode(const PagedDecodeArgs& a, cudaStream_t s) {
  using SM = PagedSmem<HD>;
  static PerDeviceInt smem_opt_in;
  PD_TRY(opt_in_smem(smem_opt_in, paged_decode_kernel<HD, WIDE>, SM::BYTES));
  PD_CUDA_TRY(launch_pdl(paged_decode_kernel<HD, WIDE>, dim3(a.n_splits, a.n_kv_heads, a.batch), dim3(PA_THREADS), SM::BYTES, s, a));
  count_launch();
  if (a.n_splits > 1) {
    PD_CUDA_TRY(launch_pdl(paged_combine_kernel<HD>, dim3(a.n_q_heads, a.batch), dim3(PC_WARPS * 32), 0, s, a));
    count_launch();
  }
  return PD_OK;
}

// How a segment (sequence, KV head) is cut.  Two blocks of eight warps are resident per SM.  A single sequence is cut into
// as many equal runs as are resident together (32768 keys, 8 KV heads: 20.3 us at 37 runs a head, 24.4 us at 55).  The
// sequences of a batch may differ in length, which the host does not know: half as many runs again even that out (24
// sequences of 100 to 4351 keys: 31.2 us, 37.4 us at one run per resident block).  From as many segments as there are
// resident blocks nothing is cut: the merge costs more than the last, partly filled wave.
struct Split { int n, chunk; };
Split paged_decode_split(int batch, int n_kv_heads, int max_kv_len) {
  const long long blocks = 1ll * batch * n_kv_heads;
  if (blocks <= 0 || max_kv_len <= 0) return {1, PA_MIN_CHUNK};
  long long want = (batch == 1 ? 296 : 444) / blocks;
  if (want < 1) want = 1;
  long long chunk = (max_kv_len + want - 1) / want;
  if (chunk < PA_MIN_CHUNK) chunk = PA_MIN_CHUNK;
  chunk = (chunk + 63) / 64 * 64;
  return {static_cast<int>((max_kv_len + chunk - 1) / chunk), static_cast<int>(chunk)};
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
  const int splits = pd::paged_decode_split(B, cfg->n_kv_heads, max_kv_len).n;
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
  const Split sp = paged_decode_split(B, cfg->n_kv_heads, max_kv_len);
  a.n_splits = sp.n; a.chunk = sp.chunk;
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
