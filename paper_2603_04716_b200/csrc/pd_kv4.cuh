// What the kernels of the 4-bit paged KV cache share: the cache as kernels see it, host-side argument checks, the transform of q
// and k heads (norm, rotation) and the quantiser.
#pragma once
#include <algorithm>
#include <limits>
#include <type_traits>

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

// Checks the description (not the device contents) and fills the device view; kv_heads: of the configuration, checked before.
inline pd_status kv4_cache_view(const pd_paged_kv4_cache* c, int kv_heads, Kv4Cache* out) {
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
  if ((1ll * c->n_pages * kv_heads) << l2 > 0xffffffffll) return PD_ERR_UNSUPPORTED_SHAPE;  // (so are rows of the pool)
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
  float eps_fast;          // of the fp32 transform: eps above 0 stays above 0, so that a head of zeros stays one
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
  out->eps = t->eps;
  out->eps_fast = t->eps > 0.0 ? std::max(static_cast<float>(t->eps), std::numeric_limits<float>::denorm_min()) : 0.f;
  out->n_pos = 0; out->rot = 0;
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

// Eight bf16 values, in memory order (of a share: of its chunks).
__device__ __forceinline__ void unpack8(const uint4& v, float* f) {
  f[0] = ptx::bf16_lo(v.x); f[1] = ptx::bf16_hi(v.x);
  f[2] = ptx::bf16_lo(v.y); f[3] = ptx::bf16_hi(v.y);
  f[4] = ptx::bf16_lo(v.z); f[5] = ptx::bf16_hi(v.z);
  f[6] = ptx::bf16_lo(v.w); f[7] = ptx::bf16_hi(v.w);
}

template <int LANES, class T>
__device__ __forceinline__ T lanes_sum(T v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ uint64_t dup_f32x2(float v) { return ptx::pack_f32x2(v, v); }

// A head of one row is the work of hd / 8 neighbouring lanes, 8 features each: two chunks of 4 that start at a and b.  With halves
// paired, lane j < rot / 8 holds features 4 j .. and their partners rot / 2 + 4 j ..; every other lane 8 neighbours.  Either way
// the lane's 4 pairs are pairs 4 j .. of the table's row.
template <bool PAIRS>
struct HeadShare {
  int a, b;
  bool turns;
  __device__ __forceinline__ HeadShare(int j, int rot) {
    turns = j < rot / 8;
    const bool split = !PAIRS && turns;
    a = split ? 4 * j : 8 * j;
    b = split ? rot / 2 + 4 * j : a + 4;
  }
  __device__ __forceinline__ uint4 load(const bf16* head) const {
    if (PAIRS) return *reinterpret_cast<const uint4*>(head + a);
    const uint2 x = *reinterpret_cast<const uint2*>(head + a), y = *reinterpret_cast<const uint2*>(head + b);
    return make_uint4(x.x, x.y, y.x, y.y);
  }
  __device__ __forceinline__ void store(bf16* head, const uint4& w) const {
    if (PAIRS) {
      *reinterpret_cast<uint4*>(head + a) = w;
    } else {
      *reinterpret_cast<uint2*>(head + a) = make_uint2(w.x, w.y);
      *reinterpret_cast<uint2*>(head + b) = make_uint2(w.z, w.w);
    }
  }
  // The first and the second features of the lane's pairs 2 i and 2 i + 1, packed.
  static __device__ __forceinline__ void unpack(const uint4& w, uint64_t (&u)[2], uint64_t (&v)[2]) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u[i] = PAIRS ? ptx::pack_f32x2(ptx::bf16_lo(x[2 * i]), ptx::bf16_lo(x[2 * i + 1])) : ptx::pack_f32x2(ptx::bf16_lo(x[i]), ptx::bf16_hi(x[i]));
      v[i] = PAIRS ? ptx::pack_f32x2(ptx::bf16_hi(x[2 * i]), ptx::bf16_hi(x[2 * i + 1])) : ptx::pack_f32x2(ptx::bf16_lo(x[2 + i]), ptx::bf16_hi(x[2 + i]));
    }
  }
  static __device__ __forceinline__ uint4 pack(const uint64_t (&u)[2], const uint64_t (&v)[2]) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float u0, u1, v0, v1;
      ptx::unpack_f32x2(u[i], u0, u1);
      ptx::unpack_f32x2(v[i], v0, v1);
      x[PAIRS ? 2 * i : i] = PAIRS ? ptx::pack_bf16(u0, v0) : ptx::pack_bf16(u0, u1);
      x[PAIRS ? 2 * i + 1 : 2 + i] = PAIRS ? ptx::pack_bf16(u1, v1) : ptx::pack_bf16(v0, v1);
    }
    return make_uint4(x[0], x[1], x[2], x[3]);
  }
};
// A warp has a row, 256 / hd heads of it at a time, and the loads of STEPS such groups go out before anything else is known.
template <int HD>
constexpr int heads_per_step() { return 256 / HD; }
template <int HD, bool PAIRS, int STEPS>
__device__ __forceinline__ void load_heads(uint4 (&w)[STEPS], const bf16* first_head, int n_heads, const HeadShare<PAIRS>& at) {
  const int mine = (threadIdx.x & 31) / (HD / 8);
  const bf16* const head = first_head + mine * HD;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    w[i] = make_uint4(0, 0, 0, 0);
    if (i * heads_per_step<HD>() + mine < n_heads) w[i] = at.load(head + i * 256);
  }
}
// Of the two kernels that read rows: whether there is a norm and whether whole heads are rotated is decided once per warp, not per head.
template <class F>
__device__ __forceinline__ void with_flags(bool norm, bool whole, F f) {
  if (norm) {
    if (whole) f(std::true_type(), std::true_type()); else f(std::true_type(), std::false_type());
  } else {
    if (whole) f(std::false_type(), std::true_type()); else f(std::false_type(), std::false_type());
  }
}

// ---- q, in fp32: n_heads heads of a row, rounded to bf16 once.  Gain and rotation are one product with a matrix of two by two
// per pair, the same for all heads of the row; the factor that the norm has in common comes last.
template <int HD, bool PAIRS, bool NORM, bool WHOLE>
struct FastTransform {
  uint64_t mu[2], mv[2], nu[2], nv[2];  // first = mu first + nu second, second = mv second + nv first
  bool turns;
  __device__ __forceinline__ FastTransform(const HeadShare<PAIRS>& at, const bf16* gain, const float2* angles, int j) {
    turns = WHOLE || at.turns;
    at.unpack(NORM ? at.load(gain) : make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), mu, mv);
    if (!turns) return;
    const float4* const cs = reinterpret_cast<const float4*>(angles + 4 * j);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 x = cs[i];
      const uint64_t c = ptx::pack_f32x2(x.x, x.z);
      nu[i] = ptx::mul_f32x2(mv[i], ptx::pack_f32x2(-x.y, -x.w));
      nv[i] = ptx::mul_f32x2(mu[i], ptx::pack_f32x2(x.y, x.w));
      mu[i] = ptx::mul_f32x2(mu[i], c);
      mv[i] = ptx::mul_f32x2(mv[i], c);
    }
  }
  template <int STEPS>
  __device__ __forceinline__ void operator()(const uint4 (&w)[STEPS], bf16* first_head, int n_heads, const HeadShare<PAIRS>& at, float eps) const {
    const int mine = (threadIdx.x & 31) / (HD / 8);
    bf16* const head = first_head + mine * HD;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      uint64_t u[2], v[2], x[2], y[2];
      at.unpack(w[s], u, v);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[i] = ptx::mul_f32x2(u[i], mu[i]);
        y[i] = ptx::mul_f32x2(v[i], mv[i]);
        if (turns) {
          x[i] = ptx::fma_f32x2(v[i], nu[i], x[i]);
          y[i] = ptx::fma_f32x2(u[i], nv[i], y[i]);
        }
      }
      if (NORM) {
        float lo, hi, r;
        ptx::unpack_f32x2(ptx::fma_f32x2(u[1], u[1], ptx::fma_f32x2(v[0], v[0], ptx::fma_f32x2(v[1], v[1], ptx::mul_f32x2(u[0], u[0])))), lo, hi);
        asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(fmaf(lanes_sum<HD / 8>(lo + hi), 1.f / HD, eps)));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          x[i] = ptx::mul_f32x2(x[i], dup_f32x2(r));
          y[i] = ptx::mul_f32x2(y[i], dup_f32x2(r));
        }
      }
      if (s * heads_per_step<HD>() + mine < n_heads) at.store(head + s * 256, at.pack(x, y));
    }
  }
};

// ---- k, in double.  A product of a gain and a cos or sin has 32 significant bits, its products with a feature 40: all of them are
// exact, and the factor of the norm comes last.
template <int HD, bool PAIRS, bool NORM, bool WHOLE>
struct ExactTransform {
  double m[8], n[8];  // feature = m feature + n partner
  bool turns;
  static __device__ __forceinline__ constexpr int first(int pair) { return PAIRS ? 2 * pair : pair; }
  static __device__ __forceinline__ constexpr int second(int pair) { return PAIRS ? 2 * pair + 1 : 4 + pair; }
  __device__ __forceinline__ ExactTransform(const HeadShare<PAIRS>& at, const bf16* gain, const float2* angles, int j) {
    turns = WHOLE || at.turns;
    float g[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (NORM) unpack8(at.load(gain), g);
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = static_cast<double>(g[e]);
    if (turns) {
      const float4* const cs = reinterpret_cast<const float4*>(angles + 4 * j);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 x = cs[i];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const double c = p ? x.z : x.x, s = p ? x.w : x.y;
          const int a = first(2 * i + p), b = second(2 * i + p);
          n[a] = -m[b] * s;
          n[b] = m[a] * s;
          m[a] *= c;
          m[b] *= c;
        }
      }
    }
  }
  // All lanes of a warp call it.
  __device__ __forceinline__ void operator()(const uint4& w, double eps, double (&f)[8]) const {
    float x[8];
    double v[8];
    unpack8(w, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<double>(x[e]);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = v[e] * m[e];
    if (turns) {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        f[first(p)] = fma(v[second(p)], n[first(p)], f[first(p)]);
        f[second(p)] = fma(v[first(p)], n[second(p)], f[second(p)]);
      }
    }
    if (NORM) {
      double sum[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e & 1] = fma(v[e], v[e], sum[e & 1]);
      const double r = rsqrt(lanes_sum<HD / 8>(sum[0] + sum[1]) * (1.0 / HD) + eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= r;
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
// Largest magnitude of 4 values; NaN if one of them is.
__device__ __forceinline__ float max_nan3(float a, float b, float c) {
  float m;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
  return m;
}
__device__ __forceinline__ float chunk_max(const float* t) {
  return max_nan3(max_nan3(fabsf(t[0]), fabsf(t[1]), fabsf(t[2])), fabsf(t[3]), 0.f);
}
// Quotients t / d are formed with an approximate reciprocal and corrected by the exact remainder, p + (t - p d) inv: the float
// nearest to within 2^-20 of a step.  That cannot move one onto a border b of the formats that it does not lie on, or off one that
// it does: b * d is a float, t differs from it by one step at least, and d has at most four significant bits, so the quotients
// differ by more than half a step of b.
// The E4M3 scale of 16 values from their largest magnitude; NaN if one of them is infinite or NaN.
__device__ __forceinline__ uint32_t kv4_scale(float amax) {
  const float inv = 1.f / 6.f, p = __fmul_rn(amax, inv);
  return amax <= 3.402823466e38f ? ptx::cvt_e4m3x2(__fmaf_rn(__fmaf_rn(p, -6.f, amax), inv, p), 0.f) : 0x7fu;
}
__device__ __forceinline__ float e4m3_value(uint32_t code) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(code)));
  float f;
  asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.f32.f16 %0, lo; }" : "=f"(f) : "r"(h));
  return f;
}
// Eight values over their scales (one of the first four, one of the others) -> eight E2M1 codes, value i in bits 4 i .. 4 i + 3.
__device__ __forceinline__ uint32_t kv4_codes(const float (&t)[8], float scale0, float scale1) {
  float q[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float scale = h ? scale1 : scale0;
    float inv;
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(scale));
    if (!(scale > 0.f)) inv = 0.f;
    const uint64_t inv2 = dup_f32x2(inv), neg2 = dup_f32x2(-scale);
#pragma unroll
    for (int e = 4 * h; e < 4 * h + 4; e += 2) {
      // (a zero added: 0 is +0 whatever the sign of t)
      const uint64_t v = ptx::pack_f32x2(t[e], t[e + 1]), p = ptx::fma_f32x2(v, inv2, dup_f32x2(0.f));
      ptx::unpack_f32x2(ptx::fma_f32x2(ptx::fma_f32x2(p, neg2, v), inv2, p), q[e], q[e + 1]);
    }
  }
  uint32_t r;
  asm("{ .reg .b8 c0, c1, c2, c3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c0, %2, %1; cvt.rn.satfinite.e2m1x2.f32 c1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c2, %6, %5; cvt.rn.satfinite.e2m1x2.f32 c3, %8, %7;\n\t"
      "mov.b32 %0, {c0, c1, c2, c3}; }"
      : "=r"(r) : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
  return r;
}
// Stores a lane's share (8 values t) of one row: codes to row `codes`, scales, in units of 2^exp, to row `scales`.  With neighbours
// in a lane the 16 that share a scale lie with two lanes.  Where halves are paired its four chunks of 4 may lie with four, in
// either place: their maxima meet in `maxima`, 64 floats of the warp's own in shared memory.  All lanes of a warp call it; j is
// the lane's place in its row.
template <int HD, bool PAIRS>
__device__ __forceinline__ void store_kv4(const float (&t)[8], int exp, const HeadShare<PAIRS>& at, int j, bool live, float* maxima,
                                          uint8_t* codes, uint8_t* scales) {
  float amax[2];
  if (PAIRS) {
    amax[0] = max_nan3(chunk_max(t), chunk_max(t + 4), 0.f);
    amax[0] = max_nan3(amax[0], __shfl_xor_sync(0xffffffffu, amax[0], 1), 0.f);
  } else {
    float* const row = maxima + ((threadIdx.x & 31) - j) * 2;
    row[at.a / 4] = chunk_max(t);
    row[at.b / 4] = chunk_max(t + 4);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 m = *reinterpret_cast<const float4*>(row + (i ? at.b : at.a) / 16 * 4);
      amax[i] = max_nan3(max_nan3(m.x, m.y, m.z), m.w, 0.f);
    }
    __syncwarp();  // (the next head's maxima go to the same place)
  }
  if (!live) return;
  const float unit = pow2f(exp), inv_unit = pow2f(-exp);
  // (toward zero: a finite value stays one, and an infinite one stays infinite)
  const uint32_t s0 = kv4_scale(__fmul_rz(amax[0], inv_unit)), s1 = PAIRS ? s0 : kv4_scale(__fmul_rz(amax[1], inv_unit));
  // Values beyond 8 times the largest scale have the largest code whatever they are.  They are held to that where their quotients
  // would leave fp32: the remainder of an infinite one is infinite with the other sign, and the code would lose it.
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = t[e];
  if (exp < -8) {
    const float most = 8.f * 448.f * unit;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fminf(fmaxf(v[e], -most), most);
  }
  const uint32_t c = kv4_codes(v, e4m3_value(s0) * unit, e4m3_value(s1) * unit);
  if (PAIRS) {
    *reinterpret_cast<uint32_t*>(codes + at.a / 2) = c;
    if ((j & 1) == 0) scales[j / 2] = static_cast<uint8_t>(s0);
  } else {
    *reinterpret_cast<uint16_t*>(codes + at.a / 2) = static_cast<uint16_t>(c);
    *reinterpret_cast<uint16_t*>(codes + at.b / 2) = static_cast<uint16_t>(c >> 16);
    if ((at.a & 12) == 0) scales[at.a / 16] = static_cast<uint8_t>(s0);
    if ((at.b & 12) == 0) scales[at.b / 16] = static_cast<uint8_t>(s1);
  }
}

}  // namespace pd
