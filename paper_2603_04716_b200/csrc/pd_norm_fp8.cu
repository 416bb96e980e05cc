// Residual addition, RMSNorm and FP8 quantisation of a row in one pass (pd_add_rmsnorm_fp8).
//
//   h = bf16(x + r),  n = h * rsqrt(mean(h^2) + eps) * g,  s = max|n| / 448 over 128 channels or the row,  code = E4M3(n / s)
//
// One block per row.  The row is read once, kept in registers as its bf16 sum, and written once as h, codes and scales:
// 2 + 2 bytes in, 2 + 1 bytes out per element, HBM-bound.  n is quantised from its fp32 value: the bf16 rounding that a
// separate norm and quantiser would put between the two is left out.  All loads of a row are in flight before the first is
// used, a block holds little else, so several rows per SM overlap.  Measured: 4099 x 4096 in 21 us = 5.6 TB/s, 87 % of a copy;
// 200 x 8192 (one wave of blocks) 5.2 us; one row 2.2 us.
#include "pd_common.cuh"
#include "pd_ptx.cuh"

namespace pd {
namespace {

constexpr int AN_THREADS = 256;
constexpr int AN_MAX_CHUNKS = 8;  // 8 chunks * 8 elements * 256 threads = d up to 16384

struct AddNormArgs {
  const bf16* x;
  const bf16* r;     // NULL: h = x
  const bf16* gain;
  bf16* sum_out;     // [rows, d] or NULL
  bf16* norm_out;    // [rows, d] or NULL
  uint8_t* codes;    // [rows, d] or NULL
  float* scales;     // [rows, d / 128] or [rows]
  int ldx, ldr, rows, d;
  float eps;
};

// Eight elements as four pairs: the packed fp32 instructions do two at a time.
__device__ __forceinline__ void unpack8(const uint4& v, uint64_t (&f)[4]) {
  f[0] = ptx::pack_f32x2(ptx::bf16_lo(v.x), ptx::bf16_hi(v.x));
  f[1] = ptx::pack_f32x2(ptx::bf16_lo(v.y), ptx::bf16_hi(v.y));
  f[2] = ptx::pack_f32x2(ptx::bf16_lo(v.z), ptx::bf16_hi(v.z));
  f[3] = ptx::pack_f32x2(ptx::bf16_lo(v.w), ptx::bf16_hi(v.w));
}
__device__ __forceinline__ uint32_t round2(uint64_t f) {
  float lo, hi;
  ptx::unpack_f32x2(f, lo, hi);
  return ptx::pack_bf16(lo, hi);
}
__device__ __forceinline__ uint4 pack8(const uint64_t (&f)[4]) {
  return make_uint4(round2(f[0]), round2(f[1]), round2(f[2]), round2(f[3]));
}
__device__ __forceinline__ float max_abs(const uint64_t (&f)[4]) {
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float lo, hi;
    ptx::unpack_f32x2(f[j], lo, hi);
    m = ptx::fmax3(m, fabsf(lo), fabsf(hi));
  }
  return m;
}
__device__ __forceinline__ uint32_t codes2(uint64_t f, uint64_t inv) {
  float lo, hi;
  ptx::unpack_f32x2(ptx::mul_f32x2(f, inv), lo, hi);
  return ptx::cvt_e4m3x2(lo, hi);
}

// max / 448, 1 for an all-zero block; kept at the smallest normal number so that its reciprocal is finite.  Product and
// approximate reciprocal (each within 1.5 units in the last place) instead of divisions, whose instructions had been a third
// of the kernel's: a code can then differ from that of the exact quotient only where the two lie 2^-22 from a tie.
__device__ __forceinline__ float scale_of(float amax) {
  return amax > 0.f ? fmaxf(amax * (1.f / 448.f), 1.17549435e-38f) : 1.f;
}
__device__ __forceinline__ float reciprocal(float s) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
  return r;
}

// NCH: 16-byte chunks per thread.  GROUPS: one scale per 128 channels (16 neighbouring threads) instead of one per row.
template <int NCH, bool GROUPS>
__global__ void __launch_bounds__(AN_THREADS) add_rmsnorm_fp8_kernel(const AddNormArgs a) {
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const size_t row = blockIdx.x;
  const int chunks = a.d / 8;
  __shared__ float red[2][AN_THREADS / 32];
  const uint4* xr = reinterpret_cast<const uint4*>(a.x + row * a.ldx);
  const uint4* rr = a.r ? reinterpret_cast<const uint4*>(a.r + row * a.ldr) : nullptr;
  const uint4* gr = reinterpret_cast<const uint4*>(a.gain);
  uint64_t f[NCH][4];  // the sum, then the norm
  uint4 g[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = threadIdx.x + i * AN_THREADS;
    uint4 h = make_uint4(0u, 0u, 0u, 0u);
    g[i] = h;
    if (c < chunks) {
      h = xr[c];
      if (rr) {
        uint64_t e[4];
        unpack8(rr[c], e);
        unpack8(h, f[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i][j] = ptx::add_f32x2(f[i][j], e[j]);
        h = pack8(f[i]);
      }
      g[i] = gr[c];
      if (a.sum_out) reinterpret_cast<uint4*>(a.sum_out + row * a.d)[c] = h;
    }
    unpack8(h, f[i]);  // the norm sees the stored (rounded) sum; chunks beyond the row are zero
  }
  uint64_t ss2 = 0ull;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) ss2 = ptx::fma_f32x2(f[i][j], f[i][j], ss2);
  float ss, ss_hi;
  ptx::unpack_f32x2(ss2, ss, ss_hi);
  ss += ss_hi;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if ((threadIdx.x & 31) == 0) red[0][threadIdx.x >> 5] = ss;
  __syncthreads();
  float tot = 0.f;
#pragma unroll
  for (int w = 0; w < AN_THREADS / 32; ++w) tot += red[0][w];
  const float rs = rsqrtf(tot / static_cast<float>(a.d) + a.eps);
  const uint64_t rs2 = ptx::pack_f32x2(rs, rs);
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    uint64_t e[4];
    unpack8(g[i], e);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[i][j] = ptx::mul_f32x2(ptx::mul_f32x2(f[i][j], rs2), e[j]);
  }

  float inv_row = 1.f;
  if (!GROUPS && a.codes) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) amax = fmaxf(amax, max_abs(f[i]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if ((threadIdx.x & 31) == 0) red[1][threadIdx.x >> 5] = amax;
    __syncthreads();
    float mx = 0.f;
#pragma unroll
    for (int w = 0; w < AN_THREADS / 32; ++w) mx = fmaxf(mx, red[1][w]);
    const float s = scale_of(mx);
    inv_row = reciprocal(s);
    if (threadIdx.x == 0) a.scales[row] = s;
  }
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = threadIdx.x + i * AN_THREADS;
    if (a.norm_out && c < chunks) reinterpret_cast<uint4*>(a.norm_out + row * a.d)[c] = pack8(f[i]);
    if (a.codes) {
      float inv = inv_row;
      if (GROUPS) {
        float amax = max_abs(f[i]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        const float s = scale_of(amax);
        inv = reciprocal(s);
        if ((threadIdx.x & 15) == 0 && c < chunks) a.scales[row * (a.d / 128) + (c >> 4)] = s;
      }
      if (c < chunks) {
        const uint64_t inv2 = ptx::pack_f32x2(inv, inv);
        uint2 o;
        o.x = codes2(f[i][0], inv2) | (codes2(f[i][1], inv2) << 16);
        o.y = codes2(f[i][2], inv2) | (codes2(f[i][3], inv2) << 16);
        reinterpret_cast<uint2*>(a.codes + row * a.d)[c] = o;
      }
    }
  }
}

template <bool GROUPS>
cudaError_t launch(const AddNormArgs& a, cudaStream_t s) {
  const int per_thread = (a.d / 8 + AN_THREADS - 1) / AN_THREADS;
  const dim3 g(a.rows), b(AN_THREADS);
  if (per_thread <= 1) return launch_pdl(add_rmsnorm_fp8_kernel<1, GROUPS>, g, b, 0, s, a);
  if (per_thread <= 2) return launch_pdl(add_rmsnorm_fp8_kernel<2, GROUPS>, g, b, 0, s, a);
  if (per_thread <= 4) return launch_pdl(add_rmsnorm_fp8_kernel<4, GROUPS>, g, b, 0, s, a);
  return launch_pdl(add_rmsnorm_fp8_kernel<8, GROUPS>, g, b, 0, s, a);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace pd

extern "C" pd_status pd_add_rmsnorm_fp8(const void* x, int32_t ldx, const void* residual, int32_t ldr, const void* gain,
                                        float eps, int32_t rows, int32_t d, int32_t group, void* sum_out, void* norm_out,
                                        void* codes, float* scales, void* stream) {
  using namespace pd;
  if (rows < 0 || d <= 0 || (group != 0 && group != 128) || !(eps >= 0.f)) return PD_ERR_INVALID_ARG;
  if (d % (group ? 128 : 16) != 0 || d > AN_THREADS * AN_MAX_CHUNKS * 8) return PD_ERR_UNSUPPORTED_SHAPE;
  if (rows == 0) return PD_OK;
  if (!x || !gain || (!norm_out && !codes) || (codes && !scales)) return PD_ERR_INVALID_ARG;
  // in place only over rows of the same pitch: a row is read whole before it is written, its neighbours are not
  if ((sum_out == x && ldx != d) || (sum_out && sum_out == residual && ldr != d)) return PD_ERR_INVALID_ARG;
  if (ldx < d || ldx % 8 != 0 || (residual && (ldr < d || ldr % 8 != 0))) return PD_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(gain) || !aligned16(sum_out) || !aligned16(norm_out) ||
      !aligned16(codes) || (reinterpret_cast<uintptr_t>(scales) & 3u))
    return PD_ERR_INVALID_ARG;
  AddNormArgs a{};
  a.x = static_cast<const bf16*>(x); a.r = static_cast<const bf16*>(residual); a.gain = static_cast<const bf16*>(gain);
  a.sum_out = static_cast<bf16*>(sum_out); a.norm_out = static_cast<bf16*>(norm_out);
  a.codes = static_cast<uint8_t*>(codes); a.scales = scales;
  a.ldx = ldx; a.ldr = ldr; a.rows = rows; a.d = d; a.eps = eps;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_RMSNORM, st);
  PD_CUDA_TRY(group ? launch<true>(a, st) : launch<false>(a, st));
  count_launch();
  return PD_OK;
}
