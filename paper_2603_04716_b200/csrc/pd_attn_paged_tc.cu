// Prefill attention over the 8-bit paged KV cache on the 5th-generation tensor cores (tcgen05 + tensor memory).
//
// The tile structure is that of pd_attn_prefill_tc.cu: a block works on two row tiles of 128 rows whose softmax and products
// ping-pong over key tiles of 128, S / P and O live in tensor memory.  What differs:
//   * Rows are (token, query head of the group) pairs, the head fastest: a key tile is read and decoded once for all heads
//     that share it, and a short run of tokens still fills the rows (16 tokens of a group of 8 are one row tile).
//   * S = Q K^T takes the K codes as they are: a key tile is copied from its pages by TMA and multiplied as E4M3.  q goes in
//     as the sum of two E4M3 numbers, scaled per row by a power of two to a largest entry in [128, 256): the products are
//     exact, the second number leaves an error of at most 2^-10, 2^-17 of the row's largest entry.  Two 8-bit products take
//     the time of one 16-bit product.  The K scales of the pages multiply the scores in the softmax, per 16 keys.
//   * O += P V has both operands in f16.  V codes come by TMA as well, four warps turn them into f16 operand rows (exact, one
//     instruction for two codes).  O counts in a unit per item, 2^7 below the largest V scale of its pages; a page's scale
//     relative to it multiplies the codes, exact down to 2^-15 of the unit.  An item with a page below that (2^22 below its largest)
//     is a far one: its operands are bf16, V exact down to 2^-117 of the unit, p the sum of two numbers and P V two products.  So what a
//     row gets does not depend on the size of pages that weigh nothing for it or that only other rows see.  Every role has a
//     second copy of its code (ANY) that takes items of either kind, with the same arithmetic, which a block goes on with from
//     its first far item to its end.  (Measured against the kernel without far items: calls of hundreds of us 1.5 to 3 %, of
//     25 us 1.4 us more; a branch per tile in one copy of the roles 5 to 9 %.  Far items take 1.3 to 1.7 times as long.)
//   * p is kept as 2^7 p; the row reference of the exponent may lag the maximum by 2^8.  There is no decoded copy of the cache in
//     global memory.
//   * When there are fewer items than SMs, or few left over behind the last full turn of the SMs, key ranges are cut into
//     equal parts (paged_tiles_plan); the parts write unnormalised fp32 rows with their maximum and sum, and a second kernel
//     joins them.
//   * Items are handed out by the hardware: the grid has one block per item, a resident block that is done takes over the
//     next block that has not been started (clusterlaunchcontrol), so there is no counter in memory to share or to reset.
//   * S, P and both products advance by half a key tile: S of a half is written over the P that a product has just consumed,
//     while the softmax works on the other half (a prompt of 4096 tokens: 167 us, 208 us by whole tiles).
//   * 2^x of one pair of scores in eight is computed with products and sums instead of the special-function unit, which the
//     rest keeps busy for half of a step (a prompt of 8192: 547 us, 560 without; one pair in four: 577).
//   warp 0        : producer     - takes items over, looks through their V scales, publishes them in a ring, starts the copies of
//                   Q, K and V tiles and publishes the scales of the pages
//   warps 1, 2    : MMA issuers of row tile 0, 1 - S = Q K^T, O += P V (P read from tensor memory)
//   warps 4-7, 8-11 : softmax of row tile 0, 1, one row per thread; they also store the output rows
//   warps 12-15   : 32 rows each - V tiles from codes to f16, Q into two codes (while the item before is finished)
// What bounds it: two chains of about equal length, the products and the softmax.  A half costs a row tile 12 products, 650 cycles of the
// tensor pipe when back to back (8 of S, each of which reads 6 KB of shared memory, 48 cycles where the arithmetic is 32; 4 of P V, 64
// each), 1300 for both tiles; their thread gets them out at 1000 to 1600 between the other warps of its scheduler, the period
// of a half is 2150.  So an issuer runs its code as a whole warp (uniform addresses: one lane alone 4 % slower), descriptors are a sum with
// a constant, and loops that every warp shares the instruction caches with are kept small (roles inlined: 1.4 times the time).
// (Counters at 4 x 1000 tokens over 5000 keys: tensor pipe 62 % of the cycles, special functions 42 %, issue slots 50 %.)
// Measured: 37 chunks, 358 Gflop, in 385 us = 0.93 Pflop/s, 56 % of a library product's rate; a prompt of 4096 tokens (137 Gflop)
// in 160 us, of 8192 in 533 us = 1.03 Pflop/s.
// Every wait is wall-clock bounded and leaves through the common teardown.
#include <math_constants.h>

#include <algorithm>
#include <cmath>

#include "pd_paged.cuh"

namespace pd {
namespace {

constexpr int TQ = 128;                    // rows per row tile
constexpr int TK = 128;                    // keys per key tile
constexpr int TH = TK / 2;                 // half a key tile: scores, weights and products advance by it
constexpr int THREADS = 512;
constexpr int SOFTMAX_REGS = 168, OTHER_REGS = 88;  // registers of 8 warps each: together what the block is launched with, 16 x 128
constexpr float LOG2E_F = 1.4426950408889634f;
constexpr float RESCALE_THRESHOLD = 8.f;   // log2 units
constexpr float P_SHIFT = 7.f;             // p is kept as 2^7 p: at most 2^15, below f16's 65504
constexpr int K_SLOTS = 4, V_SLOTS = 2, R_SLOTS = 2, ITEM_SLOTS = 4, INFO_SLOTS = 8;
constexpr int kNoPage = static_cast<int>(0x80000000u);  // beyond the keys of a tile
constexpr int kNoRows = -1000;
// exponents of page scales, relative to the unit of O, for which f16 holds codes times 2^x: 448 * 2^7 < 65504, 2^-9 * 2^-15 = 2^-24
constexpr int V_TOP = 7, V_LOW = -15;
constexpr int SMS = 148;
constexpr int MAX_PARTS = 2 * SMS;         // parts of key ranges that a call may have (sizes the workspace)

template <int HD>
struct Cfg {
  static constexpr int CODE_BYTES = TQ * HD;                // one tile of codes: K, or one of the two numbers of Q
  static constexpr int Q_BYTES = 2 * CODE_BYTES;
  static constexpr int V_BYTES = TK * HD * 2;
  static constexpr int V_SUB_BYTES = TK * 128;              // V: sub-tiles of 64 features
  static constexpr int Q_OFF = 0;                           // two Q tiles
  static constexpr int K_OFF = 2 * Q_BYTES;
  static constexpr int V_OFF = K_OFF + K_SLOTS * CODE_BYTES;
  static constexpr int R_OFF = V_OFF + V_SLOTS * V_BYTES;   // codes of V tiles
  static constexpr int AUX_OFF = R_OFF + R_SLOTS * CODE_BYTES;
  static constexpr int SMEM_BYTES_MIN = AUX_OFF + 2048 + 1024;  // (the last for the alignment of the tiles)
  // always more than half of the SM's shared memory, so that one block owns the SM and its 512 tensor-memory columns
  static constexpr int SMEM_BYTES = SMEM_BYTES_MIN > 120 * 1024 ? SMEM_BYTES_MIN : 120 * 1024;
  static constexpr int S_COL = 0, O_COL = 128, TILE_COLS = 256;  // tensor-memory columns of a row tile
};

// barrier indices
constexpr int B_QFULL = 0, B_QEMPTY = 2, B_KFULL = 4, B_KEMPTY = B_KFULL + K_SLOTS, B_VFULL = B_KEMPTY + K_SLOTS,
              B_VEMPTY = B_VFULL + V_SLOTS, B_SFULL = B_VEMPTY + V_SLOTS, B_PREADY = B_SFULL + 4, B_ODONE = B_PREADY + 4,
              B_OREAD = B_ODONE + 4, B_IFULL = B_OREAD + 2, B_IEMPTY = B_IFULL + ITEM_SLOTS, B_CLC = B_IEMPTY + ITEM_SLOTS,
              B_QRAW = B_CLC + 1, B_RFULL = B_QRAW + 2, B_REMPTY = B_RFULL + R_SLOTS, N_BARS = B_REMPTY + R_SLOTS;

struct PagedPrefillDev {
  const bf16* q;
  bf16* o;
  const int32_t* cu_seqlens;
  const int32_t* prefix;
  PagedParts parts;        // used when split_slots > 0
  int* err_word;
  PagedCache c;
  int ldq, n_req, n_tokens, n_q_heads, n_kv_heads;
  int tile_tokens;         // tokens of a row tile: 128 / group
  int n_slots;             // blocks of tokens
  int split_slots, n_splits;  // of these, the first split_slots are n_splits items per KV head, the others one
  long long part_rows;     // (token, head) rows of the split ones
  unsigned long long wait_limit_ns;
  int test_skip_arrive;    // test hook: the second V warp leaves out one arrival
};

// A work item as warp 0 publishes it.
struct Item {
  int kvh, start, len, t0, pre, req, jb;
  int split;      // part of the key range; -1: the whole
  int n_kv;       // key tiles; -1: no more items
  int halves[2];  // half key tiles that a row tile works on
  int v_exp, far; // unit of O; whether the operands of P V are bf16
};
// Per 16 keys of a tile: factor of the scores and exponent of V's page scale relative to the unit of O (<= V_TOP; kNoRows: no
// such page).
struct alignas(16) TileInfo { float k_mul[TK / 16]; int v_rel[TK / 16]; };
// What the warps of a role hand over from its copy for usual items to that for any (the producer has one for both).
struct ProducerState { int idx, published, act[2], asked, more, g, q_started; };
struct IssuerState { int seq, act, kg, vg; uint32_t p_ph; };
struct ConverterState { int seq, g, act[2]; };
struct SoftmaxState { uint32_t s_ph, o_ph; int act, seq, base; };  // phases of the s_full and o_done barriers; items with work for the row tile

struct Shared {
  uint64_t bars[N_BARS + 1];
  Item items[ITEM_SLOTS];
  TileInfo info[INFO_SLOTS];
  int8_t row_exp[2][2][TQ];   // [items with work & 1][row tile][row]: exponent that q of the row was divided by
  uint4 clc;                  // the answer to a request for another block
  uint32_t tmem;
  int v_nan[8];               // [item & 7]: number of an item with a NaN that not all its rows see
  int any;                    // the next item is a far one: every role goes on with its other copy
  ProducerState producer;
  IssuerState issuer[2];
  ConverterState converter[4];
  SoftmaxState softmax[8];
  int abort_flag;
};
static_assert(sizeof(Shared) <= 2048, "AUX area");
static_assert(Cfg<128>::SMEM_BYTES <= 227 * 1024, "shared memory");

__device__ __forceinline__ constexpr uint32_t idesc_f16(int m, int n) {  // f16 A and B, both K-major, fp32 accumulator
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t f16x2_to_e4m3x2(uint32_t v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float exp2_int(int e) {  // 2^e, e up to 127; 0 below -126
  return __uint_as_float(static_cast<uint32_t>(min(max(e, -127), 127) + 127) << 23);
}
__device__ __forceinline__ void sts64(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
// The first lane's value, which the compiler then knows to be the whole warp's.
template <typename T>
__device__ __forceinline__ T uniform(T v) { return __shfl_sync(0xffffffffu, v, 0); }
// A wait of a whole warp: one look and one vote where the phase is over, the bounded loop only where it is not.
__device__ __forceinline__ bool slow_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint64_t limit) {
  return ptx::mbar_wait_bounded(bar, parity, abort_flag, limit);
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint64_t limit) {
  if (__all_sync(0xffffffffu, ptx::mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, slow_wait(bar, parity, abort_flag, limit));
}
// 2^y of two numbers with the arithmetic of products and sums: 2^n times a polynomial in f = y - n, n the nearest integer
// (read off the sum with 1.5 * 2^23), of degree 4 with the smallest largest relative error on [-1/2, 1/2] (found by Remez
// exchange: 2^-18.5, 2^-7 of a rounding to f16).  Below 2^-126: 2^-126.  A NaN stays one.
__device__ __forceinline__ void exp2_poly(float y0, float y1, float& p0, float& p1) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(y0) : "f"(-126.f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(y1) : "f"(-126.f));
  auto both = [](float v) { return ptx::pack_f32x2(v, v); };
  const uint64_t y = ptx::pack_f32x2(y0, y1);
  const uint64_t r = ptx::add_f32x2(y, both(12582912.f));
  const uint64_t f = ptx::fma_f32x2(ptx::add_f32x2(r, both(-12582912.f)), both(-1.f), y);
  uint64_t v = ptx::fma_f32x2(f, both(0.009570102207f), both(0.05591785908f));
  v = ptx::fma_f32x2(f, v, both(0.2402474433f));
  v = ptx::fma_f32x2(f, v, both(0.6931217909f));
  v = ptx::fma_f32x2(f, v, both(0.9999992847f));
  float r0, r1;
  ptx::unpack_f32x2(r, r0, r1);
  const uint64_t n = ptx::pack_f32x2(__uint_as_float((__float_as_uint(r0) << 23) + 0x3f800000u),
                                     __uint_as_float((__float_as_uint(r1) << 23) + 0x3f800000u));
  ptx::unpack_f32x2(ptx::mul_f32x2(v, n), p0, p1);
}
// Byte offset of 16-byte chunk c (8 features) of a row of a V tile: sub-tiles of 64 features, 128-byte rows, swizzled.
template <int HD>
__device__ __forceinline__ uint32_t v_off(int row, int c) {
  return static_cast<uint32_t>((c >> 3) * Cfg<HD>::V_SUB_BYTES + row * 128 + (((c & 7) ^ (row & 7)) << 4));
}
// Byte offset of 8 codes (features 8 c ..) of a row of a code tile: rows of HD bytes, swizzled as TMA lays K out.
template <int HD>
__device__ __forceinline__ uint32_t code_off(int row, int c) {
  const int x = HD == 128 ? (row & 7) : ((row >> 1) & 3);
  return static_cast<uint32_t>(row * HD + (((c >> 1) ^ x) << 4) + (c & 1) * 8);
}
template <int HD>
__device__ __forceinline__ uint64_t code_desc(uint32_t addr) {
  return HD == 128 ? ptx::umma_desc_sw128(addr) : ptx::umma_desc_sw64(addr);
}

// ------------------------------------------------------------------------------------------------ items
// Item `idx` of the grid: KV head fastest, then the part of the key range where it is cut, then slots from the last one down
// (of a request the rows with the longest key ranges come first).  All lanes of a warp call; false: nothing to do.
__device__ __forceinline__ bool decode_item(const PagedPrefillDev& p, int idx, Item& it) {
  const int tb = 2 * p.tile_tokens, whole = (p.n_slots - p.split_slots) * p.n_kv_heads;
  int slot;
  if (idx < whole) {
    slot = p.n_slots - 1 - idx / p.n_kv_heads;
    it.split = -1;
  } else {
    const int per_slot = p.n_kv_heads * p.n_splits;
    slot = p.split_slots - 1 - (idx - whole) / per_slot;
    it.split = (idx - whole) % per_slot / p.n_kv_heads;
  }
  it.kvh = (idx < whole ? idx : idx - whole) % p.n_kv_heads;
  const TokenBlock b = find_block(p.cu_seqlens, p.prefix, p.n_req, p.n_tokens, slot, tb);
  it.req = b.req; it.start = b.start; it.len = b.len; it.pre = b.pre; it.t0 = b.t0;
  if (it.t0 >= it.len) return false;
  const int h0 = (it.pre + min(it.len, it.t0 + p.tile_tokens) + TH - 1) / TH;
  const int h1 = it.t0 + p.tile_tokens < it.len ? (it.pre + min(it.len, it.t0 + tb) + TH - 1) / TH : 0;
  const int n_all = (max(h0, h1) + 1) / 2;
  it.jb = it.split < 0 ? 0 : static_cast<int>(1ll * n_all * it.split / p.n_splits);
  const int je = it.split < 0 ? n_all : static_cast<int>(1ll * n_all * (it.split + 1) / p.n_splits);
  it.n_kv = je - it.jb;
  it.halves[0] = max(0, min(h0, 2 * je) - 2 * it.jb);
  it.halves[1] = max(0, min(h1, 2 * je) - 2 * it.jb);
  return true;
}

// Rows of row tile t of an item that hold a (token, head) pair.
__device__ __forceinline__ int tile_rows(const PagedPrefillDev& p, const Item& it, int t, int group) {
  return min(max(it.len - it.t0 - t * p.tile_tokens, 0), p.tile_tokens) * group;
}

// q of 32 rows of a row tile, in place: the buffer holds the bf16 rows as TMA has brought them, the first half of the
// features of a row where the first number of that row goes, the second half where the second goes; they become two E4M3
// numbers and the rows' exponents.  Four lanes share a row, eight rows at a time.  All lanes of a warp call.  A function of
// its own (never inlined), like the roles below, so that its registers are allocated apart from theirs.
template <int HD>
__device__ __noinline__ void convert_q(const uint32_t tile, const int first, int8_t* exps) {
  const int lane = threadIdx.x & 31, quarter = lane & 3;
  constexpr int NC = HD / 32;  // chunks of 8 features per lane
  const uint32_t raw = tile + (quarter >> 1) * Cfg<HD>::CODE_BYTES + (quarter & 1) * (HD / 2);
#pragma unroll 1
  for (int r0 = first; r0 < first + 32; r0 += 8) {
    const int r = r0 + (lane >> 2);
    const int turn = r & (NC - 1);  // rows take their chunks in different orders, so that eight lanes cover all banks
    uint32_t w[4 * NC], m2 = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * c]), "=r"(w[4 * c + 1]), "=r"(w[4 * c + 2]), "=r"(w[4 * c + 3])
                   : "r"(raw + r * HD + (c ^ turn) * 16));
#pragma unroll
    for (int e = 0; e < 4 * NC; ++e) m2 = __vmaxu2(m2, w[e] & 0x7fff7fffu);  // magnitudes compare as integers
    m2 = __vmaxu2(m2, __shfl_xor_sync(0xffffffffu, m2, 1));
    m2 = __vmaxu2(m2, __shfl_xor_sync(0xffffffffu, m2, 2));  // (also: the rows have been read whole)
    const uint32_t amax = max(m2 & 0xffffu, m2 >> 16);       // bits of the largest magnitude
    // 2^(e + 7) <= the largest < 2^(e + 8), e kept where 2^e and 2^-e are normal
    const int e2 = min(max(static_cast<int>(amax >> 7) - 127 - 7, -126), 120);
    const float inv = exp2_int(-e2);
    // a row with an infinity or a NaN: all its scores are NaN (E4M3 has no infinity, and the conversion would saturate)
    const uint32_t spoilt = amax >= 0x7f80u ? 0x7f7f7f7fu : 0u;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // at most 2^8 and of 8 significant bits: f16 holds it exactly down to 2^-14 and within 2^-25 below, and what the
        // first number leaves as well
        const uint32_t x = pack_f16(ptx::bf16_lo(w[4 * c + e]) * inv, ptx::bf16_hi(w[4 * c + e]) * inv);
        hi[e] = f16x2_to_e4m3x2(x);
        lo[e] = f16x2_to_e4m3x2(sub_f16x2(x, e4m3x2_to_f16x2(static_cast<uint16_t>(hi[e]))));
      }
      const uint32_t at = tile + code_off<HD>(r, quarter * NC + (c ^ turn));
      sts64(at, hi[0] | (hi[1] << 16) | spoilt, hi[2] | (hi[3] << 16) | spoilt);
      sts64(at + Cfg<HD>::CODE_BYTES, lo[0] | (lo[1] << 16), lo[2] | (lo[3] << 16));
    }
    if (quarter == 0) exps[r] = static_cast<int8_t>(e2);
    __syncwarp();
  }
  ptx::fence_proxy_async();
  __syncwarp();
}

// V codes of this warp's 32 rows of a tile of a far item times 2^(page exponent - unit) -> bf16 operand rows (exact).  Returns
// whether this lane left out a NaN.
template <int HD>
__device__ __noinline__ bool convert_v_far(const uint32_t src, const uint32_t dst, const TileInfo& info, const int row_lo, const int keys,
                                           const int seen_by_all) {
  constexpr int LPR = HD / 16, RPL = 32 / LPR;
  const int lane = threadIdx.x & 31, c = (lane % LPR) * 2;
  bool seen = false;
#pragma unroll 1
  for (int row = row_lo + lane / LPR; row < row_lo + TK / 4; row += RPL) {
    uint32_t w[4];
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(src + row * HD + (lane % LPR) * 16));
    const int d = info.v_rel[row >> 4];
    const float m = exp2_int(d);
    const bool valid = d != kNoRows && row < keys;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t out[4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint32_t x = w[2 * h + e];
        if (row > seen_by_all && valid) x = drop_nans(x, seen);
        if (!valid) x = 0u;
        const uint32_t lo = e4m3x2_to_f16x2(static_cast<uint16_t>(x)), hi = e4m3x2_to_f16x2(static_cast<uint16_t>(x >> 16));
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
        out[2 * e] = ptx::pack_bf16(a.x * m, a.y * m);
        out[2 * e + 1] = ptx::pack_bf16(b.x * m, b.y * m);
      }
      sts128(dst + v_off<HD>(row, c + h), out[0], out[1], out[2], out[3]);
    }
  }
  return seen;
}

// The weights of half a tile of a far item, from its scores again (keys beyond `lim` are not seen): 2^7 p as the sum of two bf16
// numbers, the second behind the first.  Returns their sum.  s0 .. s3: factors of the scores per 16 keys.
__device__ __noinline__ float far_weights(const uint32_t s_addr, const float s0, const float s1, const float s2, const float s3,
                                          const float neg_m, const int lim) {
  uint32_t sv[TH / 32][32], hi[32], lo[32];
#pragma unroll
  for (int c = 0; c < TH / 32; ++c) ptx::tmem_ld_32x32(s_addr + c * 32, sv[c]);
  ptx::tmem_ld_wait();
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 32; ++e) {
    const float sl = e < 8 ? s0 : e < 16 ? s1 : e < 24 ? s2 : s3;
    float p[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      p[k] = 2 * e + k > lim ? 0.f : ptx::ex2_approx(fmaf(__uint_as_float(sv[e >> 4][(2 * e + k) & 31]), sl, neg_m));
    sum += p[0] + p[1];
    hi[e] = ptx::pack_bf16(p[0], p[1]);
    lo[e] = ptx::pack_bf16(p[0] - ptx::bf16_lo(hi[e]), p[1] - ptx::bf16_hi(hi[e]));
  }
  ptx::tmem_st_32x32(s_addr, hi);
  ptx::tmem_st_32x32(s_addr + TH / 2, lo);
  return sum;
}

// NaN where a row sees a key (of first .. last) whose NaN codes were left out of the products.
template <int HD>
__device__ __noinline__ void put_nans(const PagedPrefillDev& p, int req, int kvh, int first, int last, bf16* out, float* part) {
  const int32_t* table = p.c.table + static_cast<size_t>(req) * p.c.table_ld;
  for (int key = first; key <= last; ++key) {
    const uint8_t* v = v_row(p.c, table, p.n_kv_heads, kvh, HD, key);
    if (!v) continue;
    for (int d = 0; d < HD; ++d) {
      if ((v[d] & 0x7f) != 0x7f) continue;
      if (out) out[d] = __float2bfloat16(CUDART_NAN_F);
      else part[d] = CUDART_NAN_F;
    }
  }
}

// --------------------------------------------------------------------------------------------- warp 0: producer
template <int HD>
__device__ __noinline__ void producer(const CUtensorMap* tmap_q, const CUtensorMap* tmap_k, const CUtensorMap* tmap_v,
                                      const PagedPrefillDev& p, const uint32_t smem_base, Shared* sh, const uint64_t limit, const bool any) {
  using C = Cfg<HD>;
  const uint32_t bar0 = ptx::smem_u32(sh->bars), clc = ptx::smem_u32(&sh->clc);
  auto bar = [&](int i) { return bar0 + 8u * i; };
  volatile int* abort_flag = &sh->abort_flag;
  const int lane = threadIdx.x & 31;
  const int group = p.n_q_heads / p.n_kv_heads;
  const int q_bytes = p.tile_tokens * group * HD;  // half of a Q tile
  const int l2p = p.c.log2_page, ppt = TK >> l2p;  // pages per key tile
  const uint32_t page_bytes = static_cast<uint32_t>(HD) << l2p;
  const ProducerState st = sh->producer;
  int published = uniform(st.published), act[2] = {uniform(st.act[0]), uniform(st.act[1])}, asked = uniform(st.asked);
  int idx = uniform(st.idx);
  bool ok = true, more = uniform(st.more);
  bool q_started = uniform(st.q_started);  // of the item at hand
  int g = uniform(st.g);                   // key tiles started so far
  auto wait = [&](int b, uint32_t parity) {
    ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar(b), parity, abort_flag, limit));
    return ok;
  };
  // the next block of the grid, if one is left that has not been started
  auto take = [&] {
    if (lane == 0) {
      ptx::mbar_arrive_expect_tx(bar(B_CLC), 16);
      ptx::clc_try_cancel(clc, bar(B_CLC));
    }
    __syncwarp();
    if (!wait(B_CLC, asked & 1)) return;
    ++asked;
    more = ptx::clc_answer(clc, idx);
    __syncwarp();
    ptx::fence_proxy_async();
  };
  Item it;
  it.far = 0;
  bool have = false;
  auto next_item = [&] {  // the first item with something to do
    have = decode_item(p, idx, it);
    while (!have && more) {
      take();
      if (!ok || !more) break;
      have = decode_item(p, idx, it);
    }
  };
  auto publish = [&] {
    const int s = published & (ITEM_SLOTS - 1);
    if (!wait(B_IEMPTY + s, ((published / ITEM_SLOTS) & 1) ^ 1u)) return;
    if (lane == 0) {
      sh->items[s] = it;
      ptx::mbar_arrive(bar(B_IFULL + s));  // release: the item is visible to whoever sees the phase flip
    }
    __syncwarp();
    ++published;
  };
  next_item();
  while (ok) {
    if (!have) break;
    const int n = it.n_kv;
    const int total = it.pre + it.len;  // keys that the request holds
    const int32_t* table = p.c.table + static_cast<size_t>(it.req) * p.c.table_ld;
    const int kvh = it.kvh, jb = it.jb, q_token = it.start + it.t0;

    // lane l < ppt holds page l of a tile: its number (-1: no such page, or no key in it), its K scale, the exponent of its
    // V scale.  Values are looked at a tile after they have been asked for, so that no load is waited for.
    auto fetch_ids = [&](int j) {
      const long long page = (static_cast<long long>(jb + j) * ppt) + lane;
      return j < n && lane < ppt && (page << l2p) < total && page < p.c.table_ld ? table[page] : kNoPage;
    };
    auto checked = [&](int id) {
      if (id != kNoPage && static_cast<unsigned>(id) >= static_cast<unsigned>(p.c.n_pages) && p.err_word) atomicExch(p.err_word, 2);
      return static_cast<unsigned>(id) < static_cast<unsigned>(p.c.n_pages) ? id : -1;
    };
    auto page_head = [&](int id) { return static_cast<size_t>(id) * p.n_kv_heads + kvh; };
    auto fetch_v_scale = [&](int id) { return id >= 0 ? __float_as_uint(p.c.v_scale[page_head(id)]) : 0u; };
    auto fetch_k_scale = [&](int id) { return id >= 0 ? p.c.k_scale[page_head(id)] : 1.f; };
    // copies the pages of tile g (a ring position) and publishes its scales.  (Rows of a page behind the last key hold
    // anything: their scores are masked, their V rows become zeros.)
    auto start_tile = [&](int ids, float ks, uint32_t vs) {
      const int ev = ids >= 0 ? static_cast<int>(vs >> 23) - 127 : kNoRows;
      const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, ids >= 0)) * page_bytes;
      const int row = static_cast<int>(page_head(ids) << l2p);
      const int s = g % K_SLOTS, r = g % R_SLOTS;
      if (!wait(B_KEMPTY + s, ((g / K_SLOTS) & 1) ^ 1u)) return;
      TileInfo& info = sh->info[g % INFO_SLOTS];
      const int page16 = (16 * (lane & 7)) >> l2p;  // the page of 16 keys
      const float mul = __shfl_sync(0xffffffffu, ks, page16);
      const int rel = __shfl_sync(0xffffffffu, ev, page16);
      if (lane < TK / 16) {
        info.k_mul[lane] = mul;
        info.v_rel[lane] = rel == kNoRows ? kNoRows : rel - it.v_exp;
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_expect_tx(bar(B_KFULL + s), bytes);
      __syncwarp();
      if (ids >= 0) ptx::tma_load_2d(smem_base + C::K_OFF + s * C::CODE_BYTES + lane * page_bytes, tmap_k, 0, row, bar(B_KFULL + s));
      if (!wait(B_REMPTY + r, ((g / R_SLOTS) & 1) ^ 1u)) return;
      if (lane == 0) ptx::mbar_arrive_expect_tx(bar(B_RFULL + r), bytes);
      __syncwarp();
      if (ids >= 0) ptx::tma_load_2d(smem_base + C::R_OFF + r * C::CODE_BYTES + lane * page_bytes, tmap_v, 0, row, bar(B_RFULL + r));
      ++g;
    };
    auto start_q = [&](int t) {
      if ((t == 0 ? it.halves[0] : it.halves[1]) == 0) return;
      // the tile's Q buffer is free once the last Q K^T of its previous item has been executed
      if (!wait(B_QEMPTY + t, (act[t] & 1) ^ 1u)) return;
      if (lane == 0) {
        // (tokens of the tile that belong to the next request, or zeros behind the last one, come along: they are not used)
        const uint32_t tile = smem_base + C::Q_OFF + t * C::Q_BYTES;
        ptx::mbar_arrive_expect_tx(bar(B_QRAW + t), 2 * q_bytes);
        for (int h = 0; h < 2; ++h)
          ptx::tma_load_3d(tile + h * C::CODE_BYTES, tmap_q, h * (HD / 2), kvh * group, q_token + t * p.tile_tokens, bar(B_QRAW + t));
      }
      __syncwarp();
      ++act[t];
    };

    // The unit of the item's O, and whether it is a far one, come from all its V scales (the first pages' numbers are asked for
    // together with those of the first tiles).
    constexpr int AHEAD = 4;  // pages per lane
    const int scan_end = static_cast<int>(min((min(static_cast<long long>(jb + n) * TK, static_cast<long long>(total)) + (1 << l2p) - 1) >> l2p,
                                              static_cast<long long>(p.c.table_ld)));
    int page = jb * ppt + lane, scan[AHEAD];
    auto scan_ids = [&] {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) scan[i] = page + 32 * i < scan_end ? table[page + 32 * i] : -1;
      page += 32 * AHEAD;
    };
    scan_ids();
    int ids0 = fetch_ids(0), ids1 = fetch_ids(1), raw2 = fetch_ids(2);
    if (published == 0 && !q_started) {  // the block's first item: the buffers are free
      start_q(0);
      start_q(1);
      q_started = true;
    }
    ids0 = checked(ids0); ids1 = checked(ids1);
    uint32_t vs0 = fetch_v_scale(ids0), vs1 = fetch_v_scale(ids1);
    float ks0 = fetch_k_scale(ids0), ks1 = fetch_k_scale(ids1);
    {
      int top = kNoRows, low = -kNoRows;
      while (true) {
        uint32_t vs[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) vs[i] = static_cast<unsigned>(scan[i]) < static_cast<unsigned>(p.c.n_pages) ? fetch_v_scale(scan[i]) : 0u;
        const bool last = page - lane >= scan_end;
        if (!last) scan_ids();
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const int e = static_cast<int>(vs[i] >> 23) - 127;
          if (vs[i] != 0u) { top = max(top, e); low = min(low, e); }  // (a scale is never 0)
        }
        if (last) break;
      }
      top = __reduce_max_sync(0xffffffffu, top);
      low = __reduce_min_sync(0xffffffffu, low);
      it.v_exp = top == kNoRows ? 0 : top - V_TOP;
      it.far = low < it.v_exp + V_LOW;
    }
    if (!any && it.far) break;
    if (ok) publish();
    if (!ok) break;
#pragma unroll 1
    for (int j = 0; j < n && ok; ++j) {
      const int raw3 = fetch_ids(j + 3), ids2 = checked(raw2);
      const uint32_t vs2 = fetch_v_scale(ids2);
      const float ks2 = fetch_k_scale(ids2);
      start_tile(ids0, ks0, vs0);
      // (a later item's q waits for the current one's last product: its first key tiles go before it)
      if (ok && !q_started && j == min(1, n - 1)) { start_q(0); if (ok) start_q(1); }
      ids0 = ids1; ids1 = ids2; raw2 = raw3; vs0 = vs1; vs1 = vs2; ks0 = ks1; ks1 = ks2;
      if (!ok) break;
      // Another block is taken over only when the copies of this item are nearly all under way: early enough to bring the next
      // one's operands in time, and no block waits here while another SM has nothing to do.
      if (j == max(n - 2, 0)) { if (more) take(); }
    }
    if (ok && n == 0 && more) take();  // (a part of a key range with no tile in it)
    if (!ok) break;
    q_started = have = false;
    if (more) next_item();
  }
  if (ok) {  // the end, or the first far item
    it.n_kv = -1;
    publish();
    if (!any && lane == 0) {
      sh->any = it.far;
      sh->producer = {idx, published, {act[0], act[1]}, asked, more, g, q_started};
    }
  }
  if (!ok) {
    // the answer to a request still out, and copies in flight, must land before the block's shared memory is released
#pragma unroll 1
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
}

// Issued by the lane whose predicate is set; the whole warp runs the code, so that addresses and descriptors are uniform.
__device__ __forceinline__ void umma_f8_if(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %5, 0;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ void umma_f16_ts_if(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %5, 0;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ void commit_if(uint32_t leader, uint32_t bar) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
               "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader) : "memory");
}
__device__ __forceinline__ void arrive_if(uint32_t leader, uint32_t bar) {
  __syncwarp();
  if (leader) ptx::mbar_arrive(bar);
  __syncwarp();
}
// A descriptor whose address lies `bytes` further (addresses stay below 2^18, so nothing carries out of the field).
__device__ __forceinline__ uint64_t desc_plus(uint64_t desc, uint32_t bytes) {
  return (desc & 0xffffffff00000000ull) | (static_cast<uint32_t>(desc) + (bytes >> 4));
}
// ------------------------------------------------------------------------- warps 1, 2: MMA issuers, one per row tile
// S of half a key tile, and P V of it, at a time: the half of S that a product has consumed is written again at once, while
// the softmax works on the other half.
template <int HD, bool ANY>
__device__ __noinline__ void mma_issuer(const int tile, const uint32_t smem_b, const uint32_t tmem_b, Shared* sh, const uint64_t limit) {
  using C = Cfg<HD>;
  const int t = uniform(tile);
  const uint32_t smem_base = uniform(smem_b), tmem_base = uniform(tmem_b);
  const uint32_t bar0 = ptx::smem_u32(sh->bars);
  auto bar = [&](int i) { return bar0 + 8u * i; };
  volatile int* abort_flag = &sh->abort_flag;
  constexpr uint32_t idesc_qk = ptx::umma_idesc_e4m3(TQ, TH);
  constexpr uint32_t idesc_near = idesc_f16(TQ, HD) | (1u << 16), idesc_far = ptx::umma_idesc_bf16_bmn(TQ, HD);  // V: MN-major
  const uint32_t s_col = tmem_base + t * C::TILE_COLS + C::S_COL, o_col = tmem_base + t * C::TILE_COLS + C::O_COL;
  const uint64_t desc_q = code_desc<HD>(smem_base + C::Q_OFF + t * C::Q_BYTES), desc_k = code_desc<HD>(smem_base + C::K_OFF);
  const uint64_t desc_v = ptx::umma_desc_mn_sw128(smem_base + C::V_OFF, C::V_SUB_BYTES);
  auto wait = [&](int b, uint32_t parity) { return warp_wait(bar(b), parity, abort_flag, limit); };
  const uint32_t leader = (threadIdx.x & 31) == 0;
  int seq = 0;            // items taken from the ring so far
  int act = 0;            // items with work for this row tile finished so far
  int kg = 0, vg = 0;     // ring positions of the next K tile and of the next V tile
  uint32_t p_ph = 0;      // phase of the p_ready barriers
  if constexpr (ANY) {
    const IssuerState st = sh->issuer[t];
    seq = uniform(st.seq); act = uniform(st.act); kg = uniform(st.kg); vg = uniform(st.vg); p_ph = uniform(st.p_ph);
  }
  const uint32_t sfull = bar(B_SFULL + 2 * t), odone = bar(B_ODONE + 2 * t), pready = B_PREADY + 2 * t;
  // S of a half = Q K^T (it overwrites the P that aliased it, which a product issued before has consumed)
  auto issue_s = [&](int h) {
    const uint64_t dk = desc_plus(desc_k, (kg % K_SLOTS) * C::CODE_BYTES);
#pragma unroll
    for (int part = 0; part < 2; ++part) {
#pragma unroll
      for (int kk = 0; kk < HD / 32; ++kk)
        umma_f8_if(leader, s_col + h * TH, desc_plus(desc_q, part * C::CODE_BYTES + kk * 32), desc_plus(dk, h * (TH * HD) + kk * 32), idesc_qk,
                   (part > 0 || kk > 0) ? 1u : 0u);
    }
    commit_if(leader, sfull + 8 * h);
  };
  bool far = false;  // the item's kind
  // O += P V of a half
  auto issue_pv = [&](int h, uint32_t accumulate) {
    const uint32_t idesc_pv = ANY && far ? idesc_far : idesc_near;
    const uint64_t dv = desc_plus(desc_v, (vg % V_SLOTS) * C::V_BYTES);
#pragma unroll
    for (int kk = 0; kk < TH / 16; ++kk) {
      // 16 keys = 16 rows of 128 bytes further into the V tile; 8 packed columns further into P
      umma_f16_ts_if(leader, o_col, s_col + h * TH + kk * 8, desc_plus(dv, h * (TH * 128) + kk * 2048), idesc_pv, kk > 0 ? 1u : accumulate);
    }
    if (ANY && far) {  // the second number of p, behind the first
#pragma unroll 1
      for (int kk = 0; kk < TH / 16; ++kk)
        umma_f16_ts_if(leader, o_col, s_col + h * TH + TH / 2 + kk * 8, desc_plus(dv, h * (TH * 128) + kk * 2048), idesc_pv, 1u);
    }
  };
  auto wait_k = [&] { return wait(B_KFULL + kg % K_SLOTS, (kg / K_SLOTS) & 1); };
  auto wait_v = [&] { return wait(B_VFULL + vg % V_SLOTS, (vg / V_SLOTS) & 1); };
  while (true) {
    const int s = seq & (ITEM_SLOTS - 1);
    if (!wait(B_IFULL + s, (seq / ITEM_SLOTS) & 1)) return;
    const int n_kv = uniform(sh->items[s].n_kv), nh = uniform(sh->items[s].halves[t]);
    if constexpr (ANY) far = __any_sync(0xffffffffu, sh->items[s].far);
    arrive_if(leader, bar(B_IEMPTY + s));
    ++seq;
    if (n_kv < 0) break;
    int left = nh;       // halves whose S has not been issued
    auto k_done = [&] {  // the tile's last S
      commit_if(leader, bar(B_KEMPTY + kg % K_SLOTS));
      if (left == 0) commit_if(leader, bar(B_QEMPTY + t));  // the tile's Q buffer may be refilled
      ++kg;
    };
    if (nh > 0) {
      if (!wait(B_QFULL + t, act & 1) || !wait_k()) return;
      ptx::tc_fence_after();
      issue_s(0);
      --left;
      if (left > 0) { issue_s(1); --left; }
      k_done();
    }
    // Per tile, and the half h of it: O += P V, then S of that half of the next tile.  As little as possible stands between
    // the products: one that is followed by an S has no barrier of its own.
#pragma unroll 1
    for (int todo = nh; todo > 0; todo -= 2) {
      if (!wait_v()) return;
      // the first product of an item overwrites O: the previous item's output must have been read out
      if (todo == nh && act > 0 && !wait(B_OREAD + t, (act - 1) & 1)) return;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (h < todo) {
          if (!wait(pready + h, (p_ph >> h) & 1)) return;
          p_ph ^= 1u << h;
          ptx::tc_fence_after();
          issue_pv(h, h == 0 && todo == nh ? 0u : 1u);
          if (h == 1 || todo == 1) commit_if(leader, bar(B_VEMPTY + vg % V_SLOTS));
          if (left > 0) {
            if (h == 0) {
              if (!wait_k()) return;
              ptx::tc_fence_after();
            }
            issue_s(h);
            --left;
            if (h == 1 || left == 0) k_done();
          } else {
            commit_if(leader, odone + 8 * h);
          }
        }
      }
      ++vg;
    }
    // tiles that only the other row tile works on
#pragma unroll 1
    for (int j = (nh + 1) / 2; j < n_kv; ++j) {
      if (!wait_k()) return;
      arrive_if(leader, bar(B_KEMPTY + kg % K_SLOTS));
      ++kg;
      if (!wait_v()) return;
      arrive_if(leader, bar(B_VEMPTY + vg % V_SLOTS));
      ++vg;
    }
    if (nh > 0) ++act;
  }
  if (!ANY && leader) sh->issuer[t] = {seq, act, kg, vg, p_ph};
}

// ------------------------------------------------------------------------------------------- warps 12-15: Q and V tiles
template <int HD, bool ANY>
__device__ __noinline__ void v_converter(const PagedPrefillDev& p, const uint32_t smem_base, Shared* sh, const int part,
                                         const uint64_t limit) {
  using C = Cfg<HD>;
  constexpr int LPR = HD / 16, RPL = 32 / LPR;     // lanes per row (16 codes each), rows at a time
  const uint32_t bar0 = ptx::smem_u32(sh->bars);
  auto bar = [&](int i) { return bar0 + 8u * i; };
  volatile int* abort_flag = &sh->abort_flag;
  const int lane = threadIdx.x & 31;
  const int row_lo = part * (TK / 4);              // this warp's rows of a tile
  // 16 codes are two chunks of a row; lanes of the second half of a 128-feature row store theirs in the other order, so
  // that eight lanes cover all banks
  const int c = (lane % LPR) * 2, odd = HD == 128 ? (lane >> 2) & 1 : 0;
  int seq = 0, g = 0;       // items taken, V tiles converted so far
  int act[2] = {0, 0};      // items with work for a row tile so far
  if constexpr (ANY) {
    const ConverterState st = sh->converter[part];
    seq = uniform(st.seq); g = uniform(st.g); act[0] = uniform(st.act[0]); act[1] = uniform(st.act[1]);
  }
  bool ok = true;
  while (ok) {
    int n, keys, seen_by_all, halves[2];
    bool far = false;
    {
      const int s = seq & (ITEM_SLOTS - 1);
      ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar(B_IFULL + s), (seq / ITEM_SLOTS) & 1, abort_flag, limit));
      if (!ok) break;
      const Item& it = sh->items[s];
      n = it.n_kv;
      halves[0] = it.halves[0]; halves[1] = it.halves[1];
      if (ANY) far = it.far;
      seen_by_all = it.pre + it.t0 - it.jb * TK;  // the last key that all rows see
      keys = it.pre + it.len - it.jb * TK;  // that the request holds, from the item's first tile on
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(B_IEMPTY + s));
      ++seq;
    }
    if (n < 0) break;
    // q, while the item before is still worked on: its copy started when the last Q K^T of that item had run
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (halves[t] == 0) continue;
      ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar(B_QRAW + t), act[t] & 1, abort_flag, limit));
      if (!ok) break;
      convert_q<HD>(smem_base + C::Q_OFF + t * C::Q_BYTES, part * 32, sh->row_exp[act[t] & 1][t]);
      if (lane == 0) ptx::mbar_arrive(bar(B_QFULL + t));
      ++act[t];
    }
    if (!ok) break;
#pragma unroll 1
    for (int j = 0; j < n; ++j, ++g, keys -= TK, seen_by_all -= TK) {
      const int s = g % V_SLOTS, r = g % R_SLOTS;
      ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar(B_RFULL + r), (g / R_SLOTS) & 1, abort_flag, limit));
      if (!ok) break;
      ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar(B_VEMPTY + s), ((g / V_SLOTS) & 1) ^ 1u, abort_flag, limit));
      if (!ok) break;
      const uint32_t src = smem_base + C::R_OFF + r * C::CODE_BYTES + lane * 16, dst = smem_base + C::V_OFF + s * C::V_BYTES;
      if (ANY && far) {
        if (convert_v_far<HD>(src - lane * 16, dst, sh->info[g % INFO_SLOTS], row_lo, keys, seen_by_all))
          *const_cast<volatile int*>(&sh->v_nan[seq & 7]) = seq;
      } else {
        // codes * 2^(page exponent - unit) -> f16 operand rows
#pragma unroll 1
        for (int r0 = row_lo; r0 < row_lo + TK / 4; r0 += 16) {
          uint4 v[16 / RPL];
#pragma unroll
          for (int q = 0; q < 16 / RPL; ++q)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[q].x), "=r"(v[q].y), "=r"(v[q].z), "=r"(v[q].w)
                         : "r"(src + (r0 + q * RPL) * HD));
          const int d = sh->info[g % INFO_SLOTS].v_rel[r0 >> 4];
          const float m = exp2_int(d);
          const uint32_t m2 = pack_f16(m, m);
          // rows past the last key, and rows of a page that does not exist, become zeros: 0 * (whatever) must stay 0
          const int valid = d == kNoRows ? 0 : keys;
          if (r0 + 15 > seen_by_all) {
            bool seen = false;
#pragma unroll
            for (int q = 0; q < 16 / RPL; ++q) {
              const int row = r0 + q * RPL + lane / LPR;
              if (row > seen_by_all && row < valid)
                v[q] = make_uint4(drop_nans(v[q].x, seen), drop_nans(v[q].y, seen), drop_nans(v[q].z, seen), drop_nans(v[q].w, seen));
            }
            if (seen) *const_cast<volatile int*>(&sh->v_nan[seq & 7]) = seq;
          }
#pragma unroll
          for (int q = 0; q < 16 / RPL; ++q) {
            const int row = r0 + q * RPL + lane / LPR;
            if (row >= valid) v[q] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const bool second = (h ^ odd) != 0;
              const uint32_t x = second ? v[q].z : v[q].x, y = second ? v[q].w : v[q].y;
              const uint32_t h0 = e4m3x2_to_f16x2(static_cast<uint16_t>(x)), h1 = e4m3x2_to_f16x2(static_cast<uint16_t>(x >> 16));
              const uint32_t h2 = e4m3x2_to_f16x2(static_cast<uint16_t>(y)), h3 = e4m3x2_to_f16x2(static_cast<uint16_t>(y >> 16));
              sts128(dst + v_off<HD>(row, c + (h ^ odd)), mul_f16x2(h0, m2), mul_f16x2(h1, m2), mul_f16x2(h2, m2), mul_f16x2(h3, m2));
            }
          }
        }
      }
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        ptx::mbar_arrive(bar(B_REMPTY + r));
        if (!(p.test_skip_arrive && part == 1 && g == 1)) ptx::mbar_arrive(bar(B_VFULL + s));
      }
    }
  }
  if (!ANY && lane == 0) sh->converter[part] = {seq, g, {act[0], act[1]}};
}

// ---------------------------------------------------------------------------------------------- warps 4-11: softmax
// An item's rows of this thread's row tile, one row per thread.  False: a wait gave up.
template <int HD, bool ANY>
__device__ __forceinline__ bool softmax_item(const PagedPrefillDev& p, Shared* sh, const Item& it, const uint32_t tmem_base, const int item_base,
                                             const int seq, SoftmaxState& st, const uint64_t limit) {
  using C = Cfg<HD>;
  const uint32_t bar0 = ptx::smem_u32(sh->bars);
  auto bar = [&](int i) { return bar0 + 8u * i; };
  volatile int* abort_flag = &sh->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = (warp - 4) >> 2;       // row tile of this warpgroup
  const int lane_group = warp & 3;     // tensor-memory lanes this warp may touch
  const int row = lane_group * 32 + lane;
  const uint32_t t_lane = tmem_base + (static_cast<uint32_t>(lane_group * 32) << 16) + t * C::TILE_COLS;
  const int group = p.n_q_heads / p.n_kv_heads;
  const int row_token = row / group, row_head = row - row_token * group;
  const int nh = t == 0 ? it.halves[0] : it.halves[1];
  const int token0 = it.t0 + t * p.tile_tokens;
  const bool mine = row < tile_rows(p, it, t, group);
  const size_t out_row = static_cast<size_t>(it.start + token0 + row_token) * p.n_q_heads + it.kvh * group + row_head;
  if (nh == 0) {  // no rows, or no keys in this part of the range
    if (it.split >= 0 && mine)
      p.parts.ml[it.split * p.part_rows + out_row] = make_float2(-CUDART_INF_F, 0.f);
    return true;
  }
  const int row_pos = it.pre + token0 + row_token;  // last key the row may see
  float m_used = -CUDART_INF_F, l_sum = 0.f, row_scale = 0.f;
  bool ok;
#pragma unroll 1
  for (int i = 0; i < nh; ++i) {
    const int h = i & 1;
    ok = warp_wait(bar(B_SFULL + 2 * t + h), (st.s_ph >> h) & 1, abort_flag, limit);
    if (!ok) return false;
    st.s_ph ^= 1u << h;
    ptx::tc_fence_after();
    // (written before the barriers that S waited for)
    if (i == 0) row_scale = mine ? rsqrtf(static_cast<float>(HD)) * LOG2E_F * exp2_int(sh->row_exp[st.act & 1][t][row]) : 1.f;
    const TileInfo& info = sh->info[(item_base + (i >> 1)) % INFO_SLOTS];
    // factor of the scores, per 16 keys (not 0: -inf * 0)
    float sl[TH / 16];
    {
      const float4 k_mul = *reinterpret_cast<const float4*>(&info.k_mul[h * (TH / 16)]);
      sl[0] = fmaxf(row_scale * k_mul.x, 1.17549435e-38f); sl[1] = fmaxf(row_scale * k_mul.y, 1.17549435e-38f);
      sl[2] = fmaxf(row_scale * k_mul.z, 1.17549435e-38f); sl[3] = fmaxf(row_scale * k_mul.w, 1.17549435e-38f);
    }
    const int k0 = it.jb * TK + i * TH;
    const uint32_t s_addr = t_lane + C::S_COL + h * TH;
    uint32_t sv[TH / 32][32];
#pragma unroll
    for (int c = 0; c < TH / 32; ++c) ptx::tmem_ld_32x32(s_addr + c * 32, sv[c]);
    ptx::tmem_ld_wait();
    if (k0 + TH - 1 > it.pre + token0) {  // warp-uniform: some row of the tile does not see all keys
      const int lim = row_pos - k0;
#pragma unroll
      for (int c = 0; c < TH / 32; ++c) {
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if (c * 32 + e > lim) sv[c][e] = 0xff800000u;  // -inf
      }
    }
    // row maximum: three-input maxima over 16 keys, scaled, over the groups
    float mx = -CUDART_INF_F;
#pragma unroll
    for (int c = 0; c < TH / 16; ++c) {
      const uint32_t(&v)[32] = sv[c >> 1];
      const int o = (c & 1) * 16;
      float m = fmaxf(__uint_as_float(v[o]), __uint_as_float(v[o + 1]));
#pragma unroll
      for (int e = 2; e < 16; e += 2) m = ptx::fmax3(m, __uint_as_float(v[o + e]), __uint_as_float(v[o + e + 1]));
      mx = fmaxf(mx, m * sl[c]);
    }
    // lazy reference: keep the old one unless this tile exceeds it by more than the threshold
    float factor = 1.f;
    bool grow = false;
    if (i == 0) {
      m_used = mx;
    } else if (mx > m_used + RESCALE_THRESHOLD) {
      factor = ptx::ex2_approx(m_used - mx);  // (0 if the row had seen no key)
      m_used = mx;
      l_sum *= factor;
      grow = true;
    }
    if (__any_sync(0xffffffffu, grow)) {
      // O must be stable: the P V product of the previous half has finished
      // (S of half i + 1 follows it, the last two products of an item have a barrier)
      const uint32_t b = i + 1 < nh ? bar(B_SFULL + 2 * t + (h ^ 1)) : bar(B_ODONE + 2 * t + (h ^ 1));
      ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(b, ((i + 1 < nh ? st.s_ph : st.o_ph) >> (h ^ 1)) & 1, abort_flag, limit));
      if (!ok) return false;
      ptx::tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {
        uint32_t ov[32];
        ptx::tmem_ld_32x32(t_lane + C::O_COL + c * 32, ov);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * factor);
        ptx::tmem_st_32x32(t_lane + C::O_COL + c * 32, ov);
      }
      ptx::tmem_st_wait();
    }
    // 2^7 p = 2^(s * scale - m + 7) for a pair of keys at a time
    const float neg_m = (m_used == -CUDART_INF_F ? 0.f : -m_used) + P_SHIFT;
    if (ANY && it.far) {
      l_sum += far_weights(s_addr, sl[0], sl[1], sl[2], sl[3], neg_m, k0 + TH - 1 > it.pre + token0 ? row_pos - k0 : TH);
    } else {
      const uint64_t negm_2 = ptx::pack_f32x2(neg_m, neg_m);
      uint64_t ps[4] = {0ull, 0ull, 0ull, 0ull}, sl2 = 0ull;
      uint32_t pk[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        // packed column e holds keys 2 e and 2 e + 1
        const uint64_t x2 = ptx::pack_f32x2(__uint_as_float(sv[e >> 4][(2 * e) & 31]), __uint_as_float(sv[e >> 4][(2 * e + 1) & 31]));
        if (e % 8 == 0) sl2 = ptx::pack_f32x2(sl[e / 8], sl[e / 8]);
        float y0, y1;
        ptx::unpack_f32x2(ptx::fma_f32x2(x2, sl2, negm_2), y0, y1);
        float p0, p1;
        if (e % 8 == 3) {  // (one pair in eight)
          exp2_poly(y0, y1, p0, p1);
        } else {
          p0 = ptx::ex2_approx(y0);
          p1 = ptx::ex2_approx(y1);
        }
        ps[e & 3] = ptx::add_f32x2(ps[e & 3], ptx::pack_f32x2(p0, p1));
        pk[e] = pack_f16(p0, p1);
      }
      ptx::tmem_st_32x32(s_addr, pk);
      {
        float a0, a1;
        ptx::unpack_f32x2(ptx::add_f32x2(ptx::add_f32x2(ps[0], ps[1]), ptx::add_f32x2(ps[2], ps[3])), a0, a1);
        l_sum += a0 + a1;
      }
    }
    ptx::tmem_st_wait();
    ptx::tc_fence_before();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(bar(B_PREADY + 2 * t + h));
  }
  if (!ok) return false;
  ++st.act;
  // ---- the last product: store the tile's rows
  {
    const int h = (nh - 1) & 1;
    ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar(B_ODONE + 2 * t + h), (st.o_ph >> h) & 1, abort_flag, limit));
    if (!ok) return false;
    st.o_ph ^= nh > 1 ? 3u : 1u;
  }
  ptx::tc_fence_after();
  // o = O 2^v_exp / (sum of 2^7 p); the two factors apart, so that neither leaves the normal range
  const float unit = exp2_int(it.v_exp), inv = l_sum == 0.f ? 0.f : 1.f / l_sum;
  const size_t part = max(it.split, 0) * p.part_rows + out_row;
#pragma unroll 1
  for (int c0 = 0; c0 < HD; c0 += 64) {
    uint32_t ov[2][32];
    ptx::tmem_ld_32x32(t_lane + C::O_COL + c0, ov[0]);
    ptx::tmem_ld_32x32(t_lane + C::O_COL + c0 + 32, ov[1]);
    ptx::tmem_ld_wait();
    if (c0 == HD - 64) {  // the next item's first product may overwrite O
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(B_OREAD + t));
    }
    if (mine && it.split < 0) {
      bf16* dst = p.o + out_row * HD + c0;
      // a thread owns a row, so every store of a warp touches 32 different lines: 32-byte stores halve their number
#pragma unroll
      for (int e = 0; e < 64; e += 16) {
        uint32_t w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q)
          w[q] = ptx::pack_bf16(__uint_as_float(ov[e >> 5][(e & 31) + 2 * q]) * inv * unit, __uint_as_float(ov[e >> 5][(e & 31) + 2 * q + 1]) * inv * unit);
        ptx::st_global_v8(dst + e, w);
      }
    } else if (mine) {
      float* dst = p.parts.o + part * HD + c0;
#pragma unroll
      for (int e = 0; e < 64; e += 8) {
        uint32_t w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = __float_as_uint(__uint_as_float(ov[e >> 5][(e & 31) + q]) * unit);
        ptx::st_global_v8(dst + e, w);
      }
    }
  }
  if (mine && it.split >= 0) p.parts.ml[part] = make_float2(m_used, l_sum);
  if (mine && *const_cast<volatile int*>(&sh->v_nan[seq & 7]) == seq)
    put_nans<HD>(p, it.req, it.kvh, max(it.pre + it.t0 + 1, it.jb * TK), min(row_pos, (it.jb + it.n_kv) * TK - 1), it.split < 0 ? p.o + out_row * HD : nullptr, p.parts.o + part * HD);
  return true;
}
template <int HD, bool ANY>
__device__ __forceinline__ void softmax(const PagedPrefillDev& p, Shared* sh, const uint32_t tmem_base, const uint64_t limit) {
  const uint32_t bar0 = ptx::smem_u32(sh->bars);
  const int lane = threadIdx.x & 31;
  SoftmaxState* const state = &sh->softmax[(threadIdx.x >> 5) - 4];
  SoftmaxState st = {};
  if (ANY) st = {uniform(state->s_ph), uniform(state->o_ph), uniform(state->act), uniform(state->seq), uniform(state->base)};
  int seq = st.seq;     // items taken from the ring so far
  int base = st.base;   // ring position of the current item's first key tile
  bool ok = true;
  while (ok) {
    Item it;
    {
      const int s = seq & (ITEM_SLOTS - 1);
      ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar0 + 8u * (B_IFULL + s), (seq / ITEM_SLOTS) & 1, &sh->abort_flag, limit));
      if (!ok) break;
      it = sh->items[s];
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar0 + 8u * (B_IEMPTY + s));
      ++seq;
    }
    if (it.n_kv < 0) break;  // no more items
    const int item_base = base;
    base += it.n_kv;
    ok = softmax_item<HD, ANY>(p, sh, it, tmem_base, item_base, seq, st, limit);
    __syncwarp();
  }
  if (!ANY && lane == 0) *state = {st.s_ph, st.o_ph, st.act, seq, base};
  __syncwarp();
}
template <int HD>
__device__ __noinline__ void softmax_any(const PagedPrefillDev& p, Shared* sh, const uint32_t tmem_base, const uint64_t limit) {
  softmax<HD, true>(p, sh, tmem_base, limit);
}

// All roles meet at the end, or in front of the first far item; whether that is it.
__device__ __forceinline__ bool any_next(Shared* sh) {
  __syncthreads();
  return sh->any && !*const_cast<volatile int*>(&sh->abort_flag);
}

template <int HD>
__global__ void __launch_bounds__(THREADS, 1) paged_prefill_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                     const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ PagedPrefillDev p) {
  using C = Cfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  Shared* sh = reinterpret_cast<Shared*>(smem_raw + (smem_base - ptx::smem_u32(smem_raw)) + C::AUX_OFF);
  const uint32_t bar0 = ptx::smem_u32(sh->bars);
  auto bar = [&](int i) { return bar0 + 8u * i; };
  const uint64_t limit = p.wait_limit_ns;
  volatile int* abort_flag = &sh->abort_flag;

  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    sh->any = 0;
    sh->producer = {static_cast<int>(blockIdx.x), 0, {0, 0}, 0, 1, 0, 0};
    for (int i = 0; i < 8; ++i) sh->v_nan[i] = 0;
    for (int i = 0; i < N_BARS; ++i) {
      int count = 1;
      if (i >= B_QFULL && i < B_QFULL + 2) count = 4;
      if (i >= B_VFULL && i < B_VFULL + V_SLOTS) count = 4;         // the four V warps
      if (i >= B_REMPTY && i < B_REMPTY + R_SLOTS) count = 4;
      if (i >= B_KEMPTY && i < B_KEMPTY + K_SLOTS) count = 2;       // the two row tiles
      if (i >= B_VEMPTY && i < B_VEMPTY + V_SLOTS) count = 2;
      if (i >= B_PREADY && i < B_PREADY + 4) count = 4;             // the four softmax warps of the tile
      if (i >= B_OREAD && i < B_OREAD + 2) count = 4;
      if (i >= B_IEMPTY && i < B_IEMPTY + ITEM_SLOTS) count = 14;   // eight softmax warps, two MMA threads, four V warps
      ptx::mbar_init(bar(i), count);
    }
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&tmap_q);
    ptx::prefetch_tensormap(&tmap_k);
    ptx::prefetch_tensormap(&tmap_v);
  }
  if (warp == 1) {
    ptx::tmem_alloc(ptx::smem_u32(&sh->tmem), 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = sh->tmem;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();

  if (warp < 4 || warp >= 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    if (warp == 0) {
      producer<HD>(&tmap_q, &tmap_k, &tmap_v, p, smem_base, sh, limit, false);
    } else if (warp == 1 || warp == 2) {
      mma_issuer<HD, false>(warp - 1, smem_base, tmem_base, sh, limit);
    } else if (warp >= 12) {
      v_converter<HD, false>(p, smem_base, sh, warp - 12, limit);
    }
    if (any_next(sh)) {
      if (warp == 0) {
        producer<HD>(&tmap_q, &tmap_k, &tmap_v, p, smem_base, sh, limit, true);
      } else if (warp == 1 || warp == 2) {
        mma_issuer<HD, true>(warp - 1, smem_base, tmem_base, sh, limit);
      } else if (warp >= 12) {
        v_converter<HD, true>(p, smem_base, sh, warp - 12, limit);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
    softmax<HD, false>(p, sh, tmem_base, limit);
    if (any_next(sh)) softmax_any<HD>(p, sh, tmem_base, limit);
  }

  ptx::tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && p.err_word) atomicExch(p.err_word, 1);
  if (warp == 1) {
    __syncwarp();
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, 512);
  }
}

template <int HD>
pd_status launch(const PagedPrefillDev& p, long long items, cudaStream_t s) {
  static PerDeviceInt smem_opt_in;
  PD_TRY(opt_in_smem(smem_opt_in, paged_prefill_kernel<HD>, Cfg<HD>::SMEM_BYTES));
  CUtensorMap tq, tk, tv;
  PD_TRY(make_tmap_heads(&tq, p.q, p.n_tokens, p.n_q_heads, HD, p.ldq, p.tile_tokens, p.n_q_heads / p.n_kv_heads, HD / 2));
  const uint64_t rows = (static_cast<uint64_t>(p.c.n_pages) * p.n_kv_heads) << p.c.log2_page;
  PD_TRY(make_tmap_u8(&tk, p.c.k, rows, HD, HD, 1u << p.c.log2_page, HD));
  PD_TRY(make_tmap_u8(&tv, p.c.v, rows, HD, HD, 1u << p.c.log2_page, 0));
  PD_CUDA_TRY(launch_pdl(paged_prefill_kernel<HD>, dim3(static_cast<unsigned>(items)), dim3(THREADS), Cfg<HD>::SMEM_BYTES, s, tq, tk, tv, p));
  count_launch();
  if (p.split_slots > 0) return launch_paged_join(p.parts, p.o, p.part_rows, p.n_splits, HD, s);
  return PD_OK;
}

}  // namespace

size_t paged_tiles_part_rows() { return static_cast<size_t>(MAX_PARTS) * 2 * TQ; }

// Up to half as many items as SMs: every key range is cut, as often as the parts still fit the SMs together, into parts of at
// least two key tiles.  Otherwise the items that are left over when every SM has had the same number may be cut in two to four:
// items of equal length would leave most SMs idle behind the last full turn.  It is done where the time saved (2.35 us a key
// tile, 0.7 of it for heads of 64) exceeds that of writing and joining the parts: 4 x 1000 tokens over 5000 keys 390 -> 381 us.
PagedTilesPlan paged_tiles_plan(const PagedRuns& r, const int32_t* cu, const int32_t* prefix) {
  const int group = r.n_q_heads / r.n_kv_heads, tb = 2 * (TQ / group);
  const long long items = r.tile_blocks * r.n_kv_heads, all_rows = 1ll * r.n_tokens * r.n_q_heads;
  const PagedTilesPlan uncut{0, 1, 0};
  if (items <= SMS / 2) {
    const int want = static_cast<int>(std::min<long long>(SMS / items, (r.max_kv + TK - 1) / TK / 2));
    return want > 1 ? PagedTilesPlan{first_slot(r.n_tokens, r.n_req, tb), want, all_rows} : uncut;
  }
  int blocks = static_cast<int>((items % SMS + r.n_kv_heads - 1) / r.n_kv_heads);  // per KV head
  if (blocks == 0) return uncut;
  const double cut_items = 1.0 * blocks * r.n_kv_heads;
  PagedTilesPlan plan = uncut;
  int steps = 0;  // key tiles of the longest of them
  for (int i = 0; i < r.n_req && blocks > 0; ++i) {
    const int len = cu[i + 1] - cu[i], pre = prefix ? prefix[i] : 0, take = std::min(blocks, (len + tb - 1) / tb);
    if (take == 0) continue;
    const int tokens = std::min(len, take * tb);
    steps = std::max(steps, (pre + tokens + TK - 1) / TK);
    plan.split_slots = first_slot(cu[i], i, tb) + take;
    plan.part_rows = 1ll * (cu[i] + tokens) * r.n_q_heads;
    blocks -= take;
  }
  const double step_us = r.head_dim == 128 ? 2.35 : 1.65;
  double best = 0;
  for (int k = 2; k <= 4; ++k) {
    if (cut_items * k > MAX_PARTS || steps / k < 4) continue;
    const double saved = (1 - std::ceil(cut_items * k / SMS) / k) * steps * step_us;
    const double gain = saved - 6 - cut_items * 2 * TQ * k * r.head_dim * 8 / 4e6;
    if (gain > best) { best = gain; plan.n_splits = k; }
  }
  return plan.n_splits > 1 ? plan : uncut;
}

pd_status launch_paged_tiles(const PagedRuns& r, const PagedTilesPlan& plan, const PagedParts& parts, cudaStream_t s) {
  // rows of K are addressed with 32-bit numbers
  if ((static_cast<long long>(r.c.n_pages) * r.n_kv_heads << r.c.log2_page) > 0x7fffffffll) return PD_ERR_UNSUPPORTED_SHAPE;
  PagedPrefillDev p{};
  p.q = r.q; p.o = r.o; p.cu_seqlens = r.cu_seqlens; p.prefix = r.prefix; p.parts = parts; p.err_word = r.err_word; p.c = r.c;
  p.ldq = r.ldq; p.n_req = r.n_req; p.n_tokens = r.n_tokens; p.n_q_heads = r.n_q_heads; p.n_kv_heads = r.n_kv_heads;
  p.tile_tokens = TQ / (r.n_q_heads / r.n_kv_heads);
  p.split_slots = plan.split_slots; p.n_splits = plan.n_splits; p.part_rows = plan.part_rows;
  p.n_slots = first_slot(r.n_tokens, r.n_req, 2 * p.tile_tokens);
  const long long items = (p.n_slots + 1ll * p.split_slots * (p.n_splits - 1)) * r.n_kv_heads;
  if (items > 0x3fffffffll) return PD_ERR_UNSUPPORTED_SHAPE;
  p.wait_limit_ns = 4000000000ull;
  {
    unsigned long long inj = 0;
    if (take_wait_injection(PD_INJECT_ATTN_PAGED, &inj)) { p.wait_limit_ns = inj; p.test_skip_arrive = 1; }
  }
  return r.head_dim == 128 ? launch<128>(p, items, s) : launch<64>(p, items, s);
}

}  // namespace pd
