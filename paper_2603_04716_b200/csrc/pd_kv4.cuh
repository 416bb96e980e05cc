// What the kernels of the 4-bit paged KV cache share: the cache as kernels see it, host-side argument checks, the transform of q
// and k heads (norm, rotation) and the quantiser.
#pragma once
#include "pd_common.cuh"
#include "pd_ptx.cuh"

namespace pd {

constexpr int kKv4Group = 16;   // features that share a scale
constexpr int kKv4MaxExp = 30;  // of the power of two per head

// Device view of a pd_paged_kv4_cache.
struct Kv4Cache {
  uint8_t* k;              // [n_pages, Hkv, page_len, hd / 2] E2M1 codes
  uint8_t* v;
  uint8_t* k_scale;        // [n_pages, Hkv, page_len, hd / 16] E4M3
  uint8_t* v_scale;
  const int32_t* k_exp;    // [Hkv] or NULL
  const int32_t* v_exp;
  const int32_t* table;    // [n_seqs, table_ld]
  int n_pages, log2_page, table_ld;
};

// Checks the description (not the device contents) and fills the device view.
inline pd_status kv4_cache_view(const pd_paged_kv4_cache* c, Kv4Cache* out) {
  if (!c || c->struct_size != sizeof(pd_paged_kv4_cache)) return PD_ERR_INVALID_ARG;
  if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales || !c->page_table) return PD_ERR_INVALID_ARG;
  if (c->n_pages <= 0 || c->n_seqs <= 0 || c->table_ld <= 0) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k_codes) | reinterpret_cast<uintptr_t>(c->v_codes) | reinterpret_cast<uintptr_t>(c->k_scales) |
       reinterpret_cast<uintptr_t>(c->v_scales)) & 15u)
    return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k_exp) | reinterpret_cast<uintptr_t>(c->v_exp) | reinterpret_cast<uintptr_t>(c->page_table)) & 3u)
    return PD_ERR_INVALID_ARG;
  int l2 = 0;
  switch (c->page_len) {
    case 16: l2 = 4; break;
    case 32: l2 = 5; break;
    case 64: l2 = 6; break;
    case 128: l2 = 7; break;
    default: return PD_ERR_UNSUPPORTED_SHAPE;
  }
  // positions are 32-bit: table_ld pages must not reach past them
  if (c->table_ld > (0x7fffffff >> l2)) return PD_ERR_UNSUPPORTED_SHAPE;
  out->k = static_cast<uint8_t*>(c->k_codes); out->v = static_cast<uint8_t*>(c->v_codes);
  out->k_scale = static_cast<uint8_t*>(c->k_scales); out->v_scale = static_cast<uint8_t*>(c->v_scales);
  out->k_exp = c->k_exp; out->v_exp = c->v_exp; out->table = c->page_table;
  out->n_pages = c->n_pages; out->log2_page = l2; out->table_ld = c->table_ld;
  return PD_OK;
}

// The head shape part of a layer configuration (d_model and d_ff play no role here).
inline pd_status check_kv4_heads(const pd_layer_cfg* cfg) {
  if (!cfg || cfg->struct_size != sizeof(pd_layer_cfg)) return PD_ERR_INVALID_ARG;
  if (cfg->n_q_heads <= 0 || cfg->n_kv_heads <= 0) return PD_ERR_INVALID_ARG;
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return PD_ERR_UNSUPPORTED_SHAPE;
  if (cfg->n_q_heads % cfg->n_kv_heads != 0 || cfg->n_q_heads / cfg->n_kv_heads > 16) return PD_ERR_UNSUPPORTED_SHAPE;
  if (cfg->n_kv_heads > 4096) return PD_ERR_UNSUPPORTED_SHAPE;
  return PD_OK;
}

// Device view of a pd_qk_transform.
struct QkTransform {
  const float2* table;     // [n_pos, rot / 2] (cos, sin) or NULL
  const bf16* q_gain;      // [hd] or NULL
  const bf16* k_gain;
  double eps;
  int n_pos, rot;          // rot = 0 without a table
};
inline pd_status qk_transform_view(const pd_qk_transform* t, const pd_layer_cfg* cfg, QkTransform* out) {
  if (!t || t->struct_size != sizeof(pd_qk_transform)) return PD_ERR_INVALID_ARG;
  if (t->layout != PD_ROPE_HALVES && t->layout != PD_ROPE_PAIRS) return PD_ERR_INVALID_ARG;
  if (!(t->eps >= 0.0) || t->eps > 1e30) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(t->table) | reinterpret_cast<uintptr_t>(t->q_gain) | reinterpret_cast<uintptr_t>(t->k_gain)) & 15u)
    return PD_ERR_INVALID_ARG;
  out->table = reinterpret_cast<const float2*>(t->table);
  out->q_gain = static_cast<const bf16*>(t->q_gain); out->k_gain = static_cast<const bf16*>(t->k_gain);
  out->eps = t->eps; out->n_pos = 0; out->rot = 0;
  if (t->table) {
    if (t->n_pos <= 0 || t->rot_dim <= 0 || t->rot_dim > cfg->head_dim) return PD_ERR_INVALID_ARG;
    if (t->rot_dim % 16 != 0) return PD_ERR_UNSUPPORTED_SHAPE;
    out->n_pos = t->n_pos; out->rot = t->rot_dim;
  }
  return PD_OK;
}

__device__ __forceinline__ int kv4_exp(const int32_t* e, int head) { return e ? min(max(e[head], -kKv4MaxExp), kKv4MaxExp) : 0; }
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
__device__ __forceinline__ void report_place(int* err_word) {
  if (err_word) atomicExch(err_word, 2);
}

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

// A head of one row is the work of hd / 16 neighbouring lanes, 16 features each: two chunks of 8 that start at a and b.  With
// halves paired, lane j < rot / 16 holds features 8 j .. and their partners rot / 2 + 8 j ..; every other lane 16 neighbours.
// Either way the lane's 8 pairs are pairs 8 j .. of the table's row.
template <bool PAIRS>
struct HeadShare {
  int a, b;
  bool turns;
  __device__ __forceinline__ HeadShare(int j, int rot) {
    turns = j < rot / 16;
    const bool split = !PAIRS && turns;
    a = split ? 8 * j : 16 * j;
    b = split ? rot / 2 + 8 * j : a + 8;
  }
};

__device__ __forceinline__ void load_share(const bf16* head, int a, int b, uint4 (&w)[2]) {
  w[0] = *reinterpret_cast<const uint4*>(head + a);
  w[1] = *reinterpret_cast<const uint4*>(head + b);
}
__device__ __forceinline__ void load_angles(const float2* row, int j, float (&cs)[16]) {
  const float4* p = reinterpret_cast<const float4*>(row + j * 8);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = p[i];
    cs[4 * i] = v.x; cs[4 * i + 1] = v.y; cs[4 * i + 2] = v.z; cs[4 * i + 3] = v.w;
  }
}
// (a, b) -> (a c - b s, b c + a s) of the lane's 8 pairs, in the precision of T.
template <bool PAIRS, class T>
__device__ __forceinline__ void turn(T (&f)[16], const float (&cs)[16]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const T c = static_cast<T>(cs[2 * e]), s = static_cast<T>(cs[2 * e + 1]);
    T& x = f[PAIRS ? 2 * e : e];
    T& y = f[PAIRS ? 2 * e + 1 : 8 + e];
    const T u = x * c - y * s, w = y * c + x * s;
    x = u; y = w;
  }
}
// RMSNorm (where there is a gain) and rotation of a lane's share of a head, in the precision of T, times `unit`.  The factor that
// the norm has in common comes last: x * gain is exact in fp32, and in double so are its products with cos and sin.  All
// lanes of a warp call it.
template <int HD, bool PAIRS, class T>
__device__ __forceinline__ void transform_share(const uint4 (&w)[2], bool norm, const uint4 (&gain)[2], double eps, bool turns,
                                                const float (&cs)[16], T unit, T (&f)[16]) {
  float x[16];
  unpack8(w[0], x);
  unpack8(w[1], x + 8);
#pragma unroll
  for (int e = 0; e < 16; ++e) f[e] = static_cast<T>(x[e]);
  if (norm) {  // (the same for all lanes)
    T sum[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[e & 3] = fma(f[e], f[e], sum[e & 3]);
    T all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
    for (int o = HD / 32; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    unit *= rsqrt(all * static_cast<T>(1.0 / HD) + static_cast<T>(eps));
    float g[16];
    unpack8(gain[0], g);
    unpack8(gain[1], g + 8);
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] *= static_cast<T>(g[e]);
  }
  if (turns) turn<PAIRS>(f, cs);
#pragma unroll
  for (int e = 0; e < 16; ++e) f[e] *= unit;
}
// NH heads (n_h of them there are) of one row in fp32, rounded to bf16 once.  The row is read before anything else is known
// (`there`: it exists); `live`, the angles' row and the rest of the work wait for the position.
template <int HD, bool PAIRS, int NH>
struct HeadsOfRow {
  uint4 w[NH][2];
  __device__ __forceinline__ HeadsOfRow(const bf16* src, int n_h, bool there, const HeadShare<PAIRS>& at) {
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      w[h][0] = w[h][1] = make_uint4(0, 0, 0, 0);
      if (there && h < n_h) load_share(src + h * HD, at.a, at.b, w[h]);
    }
  }
  __device__ __forceinline__ void transform(bf16* dst, int n_h, bool live, const HeadShare<PAIRS>& at, const bf16* gain, double eps,
                                            const float2* angles, int j) {
    uint4 g[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    float cs[16] = {};
    if (live && at.turns) load_angles(angles, j, cs);
    if (gain) load_share(gain, at.a, at.b, g);
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      float f[16];
      transform_share<HD, PAIRS>(w[h], gain != nullptr, g, eps, at.turns, cs, 1.f, f);
      if (live && h < n_h) {
        *reinterpret_cast<uint4*>(dst + h * HD + at.a) = pack8(f);
        *reinterpret_cast<uint4*>(dst + h * HD + at.b) = pack8(f + 8);
      }
    }
  }
};

// ------------------------------------------------------------------------------------------------------------ quantiser
// A double as the float that compares the same with every number of at most 23 significant bits: rounded toward zero, the last
// bit set if anything was lost.  Borders of the two formats times a scale have a handful of bits, so decisions are exact.
// (Below 2^-126 nothing is decided.)
__device__ __forceinline__ float sticky_float(double d) {
  const uint32_t lost = static_cast<uint32_t>(__double2loint(d)) & 0x1fffffffu;
  return __uint_as_float(__float_as_uint(__double2float_rz(d)) | (lost ? 1u : 0u));
}
// Largest magnitude of 8 values; NaN if one is infinite or NaN.
__device__ __forceinline__ float chunk_max(const float* t) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(fabsf(t[e])));
  return m <= 3.402823466e38f ? m : __int_as_float(0x7fc00000);
}
// t / d by an approximate reciprocal, corrected by the exact remainder: the float nearest to within 2^-20 of a step.  That cannot
// move it onto a border b of the formats that it does not lie on, or off one that it does: b * d is a float, t differs from it by
// one step at least, and d has at most four significant bits, so the quotients differ by more than half a step of b.
__device__ __forceinline__ float quotient(float t, float d, float inv) {
  const float p = __fmul_rn(t, inv);
  return __fmaf_rn(__fmaf_rn(-p, d, t), inv, p);
}
// The E4M3 scale of 16 values from their largest magnitude.
__device__ __forceinline__ uint32_t kv4_scale(float amax) {
  return amax == amax ? ptx::cvt_e4m3x2(quotient(amax, 6.f, 1.f / 6.f), 0.f) : 0x7fu;
}
__device__ __forceinline__ float e4m3_value(uint32_t code) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(code)));
  float f;
  asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.f32.f16 %0, lo; }" : "=f"(f) : "r"(h));
  return f;
}
// Eight values over a scale -> eight E2M1 codes, value i in bits 4 i .. 4 i + 3.
__device__ __forceinline__ uint32_t kv4_codes(const float* t, float scale) {
  float inv;
  asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(scale));
  if (!(scale > 0.f)) inv = 0.f;
  uint32_t r = 0;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float q[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) q[i] = quotient(t[e + i], scale, inv);
    uint32_t c;
    asm("{ .reg .b8 c; .reg .b16 h; cvt.rn.satfinite.e2m1x2.f32 c, %1, %2; cvt.u16.u8 h, c; cvt.u32.u16 %0, h; }"
        : "=r"(c) : "f"(q[1]), "f"(q[0]));
    r |= c << (4 * e);
  }
  return r;
}
// Stores a lane's share (16 values t in units of 2^exp) of one row: codes to row `codes`, scales to row `scales`.  The two
// chunks of 8 whose common scale it is lie with one lane or, where halves are paired, with two.  All lanes of a warp call it.
template <int HD, bool PAIRS>
__device__ __forceinline__ void store_kv4(const float (&t)[16], const HeadShare<PAIRS>& at, int j, int rot, bool live, uint8_t* codes,
                                          uint8_t* scales) {
  const float m[2] = {chunk_max(t), chunk_max(t + 8)};
  float group[2];
  if (PAIRS) {
    group[0] = group[1] = fmaxf(m[0], m[1]);
    if (m[0] != m[0] || m[1] != m[1]) group[0] = group[1] = __int_as_float(0x7fc00000);
  } else {
    const int lane0 = (threadIdx.x & 31) - j;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int other = ((i ? at.b : at.a) >> 3) ^ 1;  // the neighbouring chunk, its lane and its place there
      const bool split = other < rot / 8;
      const int lane = split ? (other < rot / 16 ? other : other - rot / 16) : other >> 1;
      const bool second = split ? other >= rot / 16 : other & 1;
      const float m0 = __shfl_sync(0xffffffffu, m[0], lane0 + lane), m1 = __shfl_sync(0xffffffffu, m[1], lane0 + lane);
      const float o = second ? m1 : m0;
      group[i] = fmaxf(m[i], o);
      if (m[i] != m[i] || o != o) group[i] = __int_as_float(0x7fc00000);
    }
  }
  if (!live) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int f = i ? at.b : at.a;
    const uint32_t s = kv4_scale(group[i]);
    *reinterpret_cast<uint32_t*>(codes + f / 2) = kv4_codes(t + 8 * i, e4m3_value(s));
    if ((f & 8) == 0) scales[f / 16] = static_cast<uint8_t>(s);
  }
}

}  // namespace pd
