// Rotary positions scaled for long contexts (pd_rope_table_scaled) and the transform of q and k heads in front of attention
// (pd_qk_norm_rope).
#include <algorithm>
#include <cmath>

#include "pd_kv4.cuh"

namespace pd {
namespace {

// ------------------------------------------------------------------------------------------------------------------ table
// A thread computes `run` neighbouring positions of one pair: cos and sin of the first from the angle in half turns (product
// and reduction in double), the others by turning on, 4 fused operations instead of a reduction and two polynomials each.
// Angles are theirs to 2^-50 relative; 16 steps add 2^-48 at most, far below the final rounding to fp32.  A thread keeps its
// pair for all runs that it does: its three constants differ from lane to lane, and constant memory serves one address at a time
// (fetched for each run of 16, they cost 14.1 us instead of 13.0 for 131,072 positions of 64 pairs; 25 for runs of 8).  67 MB written at
// 5.2 TB/s; 1000 positions of 32 pairs take 2.3 us, mostly the launch and the first angle.
struct TableArgs {
  double half_turns[64], c[64], s[64];  // f_i / pi, cos f_i, sin f_i
  double magnitude;
  float2* out;  // [n_pos, pairs]
  int first, n_pos, pairs, run;
};
constexpr int TB_THREADS = 256;  // at most: as many as are a multiple of the pairs

__global__ void __launch_bounds__(TB_THREADS) rope_table_kernel(const __grid_constant__ TableArgs a) {
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int i = threadIdx.x % a.pairs, runs = blockDim.x / a.pairs;
  const double half_turns = a.half_turns[i], dc = a.c[i], ds = a.s[i];
  const long long step = 1ll * gridDim.x * runs * a.run;
  for (long long p0 = (1ll * blockIdx.x * runs + threadIdx.x / a.pairs) * a.run; p0 < a.n_pos; p0 += step) {
    const int n = static_cast<int>(min(1ll * a.run, a.n_pos - p0));
    double s, c;
    sincospi(static_cast<double>(a.first + p0) * half_turns, &s, &c);
    c *= a.magnitude;
    s *= a.magnitude;
    float2* out = a.out + p0 * a.pairs + i;
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
      out[static_cast<size_t>(k) * a.pairs] = make_float2(static_cast<float>(c), static_cast<float>(s));
      const double c1 = c * dc - s * ds;
      s = s * dc + c * ds;
      c = c1;
    }
  }
}

// Frequencies of the pairs, in radians per position.
void rope_frequencies(const pd_rope_cfg& r, double* f) {
  const int pairs = r.rot_dim / 2;
  const double pi = 3.14159265358979323846;
  double theta = r.theta;
  if (r.scaling == PD_ROPE_SCALE_BASE) theta *= std::pow(r.factor, r.rot_dim / (r.rot_dim - 2.0));
  double a = 0, b = 0;
  if (r.scaling == PD_ROPE_SCALE_INDEX) {
    auto pair_of = [&](double turns) { return r.rot_dim * std::log(r.trained_len / (2 * pi * turns)) / (2 * std::log(theta)); };
    a = std::fmax(std::floor(pair_of(r.high)), 0.0);
    b = std::fmin(std::ceil(pair_of(r.low)), r.rot_dim - 1.0);  // (behind the last pair: the slowest keeps a part)
  }
  for (int i = 0; i < pairs; ++i) {
    f[i] = std::pow(theta, -2.0 * i / r.rot_dim);
    double keep = 1.0;
    if (r.scaling == PD_ROPE_SCALE_LINEAR) keep = 0.0;
    if (r.scaling == PD_ROPE_SCALE_TURNS) keep = (r.trained_len * f[i] / (2 * pi) - r.low) / (r.high - r.low);
    if (r.scaling == PD_ROPE_SCALE_INDEX) keep = 1.0 - (i - a) / std::fmax(b - a, 1e-3);
    keep = std::fmin(std::fmax(keep, 0.0), 1.0);
    if (keep < 1.0) f[i] = keep * f[i] + (1.0 - keep) * f[i] / r.factor;
  }
}

// -------------------------------------------------------------------------------------------------------------- q and k
// HBM-bound at size, by launch and the latency of two loads (position, angles) below that.  A warp has a row and NR_STEPS * 256
// features of its heads, all loads in flight; what concerns the row (its position, the angles, their products with the gains) is
// done once for them.  Blocks along y are groups of heads, so that a small batch still covers the SMs.
// Measured: 4,099 rows of 32 + 8 heads of 128 (84 MB) 15.5 us, 5.5 TB/s; 200 rows of 64 + 8 heads 3.0 us.
struct NormArgs {
  const bf16* qkv;
  bf16* q_out;
  bf16* k_out;
  const int32_t* positions;
  int* err_word;
  QkTransform t;
  int ldqkv, ldq, ldk, rows, n_q_heads, n_kv_heads, q_blocks;
};
constexpr int NR_WARPS = 4;
constexpr int NR_STEPS = 4;

template <int HD, bool PAIRS>
__global__ void __launch_bounds__(NR_WARPS * 32, 8) qk_norm_rope_kernel(const NormArgs a) {
  constexpr int J = HD / 8, HEADS = NR_STEPS * heads_per_step<HD>();
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int row = blockIdx.x * NR_WARPS + __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), j = (threadIdx.x & 31) % J;
  if (row >= a.rows) return;
  const HeadShare<PAIRS> at(j, a.t.rot);
  const bool is_q = static_cast<int>(blockIdx.y) < a.q_blocks;
  const int h0 = (is_q ? blockIdx.y : blockIdx.y - a.q_blocks) * HEADS, n_heads = min((is_q ? a.n_q_heads : a.n_kv_heads) - h0, HEADS);
  uint4 w[NR_STEPS];
  load_heads<HD, PAIRS>(w, a.qkv + static_cast<size_t>(row) * a.ldqkv + (is_q ? h0 : a.n_q_heads + h0) * HD, n_heads, at);
  const int pos = a.positions[row];
  if (pos < 0) return;
  if (a.t.rot > 0 && pos >= a.t.n_pos) {
    report_place(a.err_word);
    return;
  }
  bf16* dst = is_q ? a.q_out + static_cast<size_t>(row) * a.ldq + h0 * HD : a.k_out + static_cast<size_t>(row) * a.ldk + h0 * HD;
  const bf16* const gain = is_q ? a.t.q_gain : a.t.k_gain;
  with_flags(gain != nullptr, a.t.rot == HD, [&](auto norm, auto whole) {
    constexpr bool NORM = decltype(norm)::value, WHOLE = decltype(whole)::value;
    const FastTransform<HD, PAIRS, NORM, WHOLE> transform(at, gain, a.t.table + static_cast<size_t>(pos) * (a.t.rot / 2), j);
    transform(w, dst, n_heads, at, a.t.eps_fast);
  });
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_rope_table_scaled(const pd_rope_cfg* rope, int32_t first_pos, int32_t n_pos, float* table, void* stream) {
  using namespace pd;
  if (!rope || rope->struct_size != sizeof(pd_rope_cfg)) return PD_ERR_INVALID_ARG;
  if (rope->rot_dim <= 0 || rope->scaling < PD_ROPE_SCALE_NONE || rope->scaling > PD_ROPE_SCALE_INDEX) return PD_ERR_INVALID_ARG;
  if (rope->rot_dim % 16 != 0 || rope->rot_dim > 128) return PD_ERR_UNSUPPORTED_SHAPE;
  if (!(rope->theta > 1.0) || !std::isfinite(rope->theta) || !(rope->magnitude > 0.0) || !std::isfinite(rope->magnitude)) return PD_ERR_INVALID_ARG;
  if (rope->scaling != PD_ROPE_SCALE_NONE && (!(rope->factor >= 1.0) || !std::isfinite(rope->factor))) return PD_ERR_INVALID_ARG;
  if (rope->scaling >= PD_ROPE_SCALE_TURNS &&
      (!(rope->low > 0.0) || !(rope->high > rope->low) || !std::isfinite(rope->high) || rope->trained_len < 1))
    return PD_ERR_INVALID_ARG;
  if (first_pos < 0 || n_pos < 0 || n_pos > 0x7fffffff - first_pos) return PD_ERR_INVALID_ARG;
  if (n_pos == 0) return PD_OK;
  if (!table || (reinterpret_cast<uintptr_t>(table) & 7u)) return PD_ERR_INVALID_ARG;
  TableArgs a{};
  double f[64];
  rope_frequencies(*rope, f);
  a.pairs = rope->rot_dim / 2;
  for (int i = 0; i < a.pairs; ++i) {
    a.half_turns[i] = f[i] / 3.14159265358979323846;
    a.c[i] = std::cos(f[i]);
    a.s[i] = std::sin(f[i]);
  }
  a.magnitude = rope->magnitude; a.out = reinterpret_cast<float2*>(table);
  a.first = first_pos; a.n_pos = n_pos;
  // long runs where there are threads enough for every SM all the same
  a.run = 1ll * n_pos * a.pairs >= (1ll << 22) ? 16 : 4;
  const int runs = TB_THREADS / a.pairs;
  const long long blocks = std::min((n_pos + (1ll * a.run * runs - 1)) / (1ll * a.run * runs), 148ll * 8);
  PD_CUDA_TRY(launch_pdl(rope_table_kernel, dim3(static_cast<unsigned>(blocks)), dim3(runs * a.pairs), 0, static_cast<cudaStream_t>(stream), a));
  count_launch();
  return PD_OK;
}

extern "C" pd_status pd_qk_norm_rope(const pd_layer_cfg* cfg, const pd_qk_transform* transform, const void* qkv, int32_t ldqkv,
                                     void* q_out, int32_t ldq_out, void* k_out, int32_t ldk_out, const int32_t* positions, int32_t T,
                                     int32_t* err_word, void* stream) {
  using namespace pd;
  PD_TRY(check_kv4_heads(cfg));
  NormArgs a{};
  PD_TRY(qk_transform_view(transform, cfg, &a.t));
  if (T < 0) return PD_ERR_INVALID_ARG;
  if (T == 0 || (!q_out && !k_out)) return PD_OK;
  const int hd = cfg->head_dim;
  if (1ll * (cfg->n_q_heads + cfg->n_kv_heads) * hd > 0x7fffffffll) return PD_ERR_UNSUPPORTED_SHAPE;
  if (!qkv || !positions || ldqkv < (cfg->n_q_heads + cfg->n_kv_heads) * hd || ldqkv % 8 != 0) return PD_ERR_INVALID_ARG;
  if (q_out && (ldq_out < cfg->n_q_heads * hd || ldq_out % 8 != 0)) return PD_ERR_INVALID_ARG;
  if (k_out && (ldk_out < cfg->n_kv_heads * hd || ldk_out % 8 != 0)) return PD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(qkv) | reinterpret_cast<uintptr_t>(q_out) | reinterpret_cast<uintptr_t>(k_out)) & 15u)
    return PD_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(positions) & 3u) return PD_ERR_INVALID_ARG;
  a.qkv = static_cast<const bf16*>(qkv); a.q_out = static_cast<bf16*>(q_out); a.k_out = static_cast<bf16*>(k_out);
  a.positions = positions; a.err_word = err_word;
  a.ldqkv = ldqkv; a.ldq = ldq_out; a.ldk = ldk_out; a.rows = T; a.n_q_heads = cfg->n_q_heads; a.n_kv_heads = cfg->n_kv_heads;
  const int heads = NR_STEPS * (256 / hd);
  a.q_blocks = q_out ? (cfg->n_q_heads + heads - 1) / heads : 0;
  const int y = a.q_blocks + (k_out ? (cfg->n_kv_heads + heads - 1) / heads : 0);
  const dim3 grid((T + (NR_WARPS - 1ll)) / NR_WARPS, y), block(NR_WARPS * 32);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TraceScope ts(PD_K_RMSNORM, st);
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, block, 0, st, a); };
  const bool pairs = transform->layout == PD_ROPE_PAIRS;
  PD_CUDA_TRY(hd == 128 ? (pairs ? go(qk_norm_rope_kernel<128, true>) : go(qk_norm_rope_kernel<128, false>))
                        : (pairs ? go(qk_norm_rope_kernel<64, true>) : go(qk_norm_rope_kernel<64, false>)));
  count_launch();
  return PD_OK;
}
