// Losses of a language model's head and their gradients with respect to its
// logits, the G operand of the head's norm and clipped sum (part of misc.hip).
//
// A row of logits z has lse = log sum_v exp(z_v) and gives its target y the
// log-probability z_y - lse; d(-log p_y)/dz_v = p_v - [v = y], p = exp(z - lse).
// Cross-entropy weights that with w per token. The preference loss of a pair of
// answers (R. Rafailov et al., "Direct Preference Optimization", 2023, with
// label smoothing) is a function of the two sums of log-ratios
//   r = beta sum_t (log p_t - log ref_t):  m = r_chosen - r_rejected,
//   loss = -(1 - eps) log sigma(m) - eps log sigma(-m),
// so every scored token of the chosen answer has the weight
// beta ((1 - eps) sigma(-m) - eps sigma(m)), and of the rejected one its negative.
//
// All of it is bound by HBM: a logit costs one exponential (three in the
// passes that write gradients twice over) and moves 2 to 8 bytes. Cross-entropy
// keeps its row in registers between the sum and the gradient, so the logits
// are read once (a row of 50257 is 98 KB in bf16: 8 octets a thread of
// 1024). A pair's weight needs the last row's log p before the first row's
// gradient, so there the logits are passed twice.
//
// Sums are fp32 from the row's largest logit; the logarithm, and the sums of
// log-ratios over an answer's tokens, are in double: a margin is a small
// difference of long sums. Exponents are formed as (z - top) log2 e, not as two
// products, which would overflow for logits near the type's ends. -inf logits
// have p = 0; a row of nothing else has log p = -inf and a zero gradient. NaN
// and +inf make the row's outputs NaN. Ignored rows are not read.
#pragma once
#include "rows.hpp"

namespace dpg {

constexpr float LOWEST = -FLT_MAX;   // running maximum of no logits (finite: -inf - it is -inf)

template <int DT>
constexpr uint32_t NEG_INF = DT == DT_BF16 ? 0xFF80FF80u : 0xFF800000u;

__device__ __forceinline__ float exp_from(float z, float top) {
  return __builtin_amdgcn_exp2f((z - top) * LOG2E);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, WAVE));
  return v;
}

// Largest value over a team (see team_sum2).
template <int W>
__device__ __forceinline__ float team_max(float v, float* red) {
  v = wave_max(v);
  if constexpr (W > 1) {
    const int w = (int)threadIdx.x / WAVE;
    __syncthreads();
    if (threadIdx.x % WAVE == 0) red[w] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v = fmaxf(v, red[i]);
  }
  return v;
}

template <int W>
struct LossTeam {
  static constexpr int THREADS = W == 1 ? 4 * WAVE : W * WAVE;
  static constexpr int TEAMS = W == 1 ? 4 : 1;
};

// Running maximum and sum of exponentials of the lane's logits: octets `lane`,
// `lane` + LANES, ... of the row, U of them in flight.
template <int DT, int W, int U>
__device__ __forceinline__ void row_sum(const char* z, int V, int lane, float& top, float& sum) {
  constexpr int LANES = W * WAVE;
  top = LOWEST;
  sum = 0.f;
  for (int o = lane; o * 8 < V; o += U * LANES) {
    Oct<DT> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (o + u * LANES) * 8;
      v[u].load(z + (int64_t)col * Oct<DT>::ES, V - col, NEG_INF<DT>);
    }
    float m = top;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, v[u].at(e));
    sum *= exp_from(top, m);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += exp_from(v[u].at(e), m);
    top = m;
  }
}

// The team's: every thread gets the row's maximum and sum.
template <int W>
__device__ __forceinline__ void team_row(float& top, float& sum, float* red) {
  const float m = team_max<W>(top, red);
  float s = sum * exp_from(top, m), none = 0.f;
  team_sum2<W>(s, none, red);
  top = m;
  sum = s;
}

__device__ __forceinline__ double row_logp(float zt, float top, float sum) {
  return sum == 0.f ? -__builtin_inf() : (double)zt - (double)top - log((double)sum);
}

template <int DT>
__device__ __forceinline__ float logit_at(const char* z, int col) {
  if constexpr (DT == DT_BF16) return bf16_to_f32(((const uint16_t*)z)[col]);
  else return ((const float*)z)[col];
}

template <int DT, int W>
__global__ __launch_bounds__(LossTeam<W>::THREADS) void token_logprobs_kernel(LossArgs a) {
  __shared__ float red[2 * W];
  const int lane = (int)threadIdx.x % (W * WAVE), team = (int)threadIdx.x / (W * WAVE);
  const int64_t r = (int64_t)blockIdx.x * LossTeam<W>::TEAMS + team;
  if (r >= a.rows) return;
  const int64_t row = a.row0 + r;
  const int y = a.targets[row];
  if (y < 0 || y >= a.V) {
    if (lane == 0) {
      if (a.logp) a.logp[row] = 0.f;
      if (a.lse) a.lse[row] = 0.f;
      if (a.logp64) a.logp64[row] = 0.0;
      if (a.stat) a.stat[row] = RowStat{0.f, 0.f};
    }
    return;
  }
  const char* z = (const char*)a.Z + row * a.ldz * Oct<DT>::ES;
  const float zt = logit_at<DT>(z, y);
  float top, sum;
  row_sum<DT, W, 4>(z, a.V, lane, top, sum);
  team_row<W>(top, sum, red);
  if (lane == 0) {
    const double logp = row_logp(zt, top, sum);
    if (a.logp) a.logp[row] = (float)logp;
    if (a.lse) a.lse[row] = sum == 0.f ? -__builtin_inff() : (float)((double)top + log((double)sum));
    if (a.logp64) a.logp64[row] = logp;
    if (a.stat) a.stat[row] = RowStat{top, sum == 0.f ? 0.f : 1.f / sum};
  }
}

// Eight gradients w (p - onehot) of an octet that starts at column col.
template <int DT>
__device__ __forceinline__ void grad_octet(Oct<DT>& v, float top, float f, float w, int rel) {
  float o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = fmaf(exp_from(v.at(e), top), f, e == rel ? -w : 0.f);
  v.set(o);
}

// Rows that give no gradient: octets from `lane` on, LANES apart.
template <int DT>
__device__ __forceinline__ void zero_row(char* g, int V, int lane, int lanes) {
  Oct<DT> v;
  const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  v.set(none);
  for (int col = lane * 8; col < V; col += lanes * 8) v.store(g + (int64_t)col * Oct<DT>::ES, V - col);
}

// NV > 0: the row stays in registers, NV octets a lane. NV = 0: rows longer than
// that are read again for the gradient.
template <int DT, int W, int NV>
__global__ __launch_bounds__(LossTeam<W>::THREADS) void cross_entropy_kernel(LossArgs a) {
  __shared__ float red[2 * W];
  __shared__ float zt_s[LossTeam<W>::TEAMS];
  constexpr int LANES = W * WAVE, ES = Oct<DT>::ES;
  const int lane = (int)threadIdx.x % LANES, team = (int)threadIdx.x / LANES;
  const int64_t row = (int64_t)blockIdx.x * LossTeam<W>::TEAMS + team;
  if (row >= a.rows) return;
  const int V = a.V, y = a.targets[row];
  const char* z = (const char*)a.Z + row * a.ldz * ES;
  char* g = (char*)a.Gz + row * a.ldg * ES;
  if (y < 0 || y >= V) {
    if (lane == 0 && a.logp) a.logp[row] = 0.f;
    zero_row<DT>(g, V, lane, LANES);
    return;
  }
  const float w = a.w[row];
  // In LDS before the first exchange: where the gradient replaces the logits
  // (Gz = Z) another thread overwrites this one.
  if (lane == 0) zt_s[team] = logit_at<DT>(z, y);
  float top, sum = 0.f;
  Oct<DT> v[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (lane + j * LANES) * 8;
      v[j].load(z + (int64_t)col * ES, V - col, NEG_INF<DT>);
    }
    top = LOWEST;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, v[j].at(e));
    top = team_max<W>(top, red);
    float none = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += exp_from(v[j].at(e), top);
    team_sum2<W>(sum, none, red);
  } else {
    row_sum<DT, W, 4>(z, V, lane, top, sum);
    team_row<W>(top, sum, red);
  }
  if (lane == 0 && a.logp) a.logp[row] = (float)row_logp(zt_s[team], top, sum);
  if (w == 0.f || sum == 0.f) {
    zero_row<DT>(g, V, lane, LANES);
    return;
  }
  const float f = w / sum;
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (lane + j * LANES) * 8;
      grad_octet<DT>(v[j], top, f, w, y - col);
      v[j].store(g + (int64_t)col * ES, V - col);
    }
  } else {
    for (int col = lane * 8; col < V; col += LANES * 8) {
      Oct<DT> u;
      u.load(z + (int64_t)col * ES, V - col, NEG_INF<DT>);
      grad_octet<DT>(u, top, f, w, y - col);
      u.store(g + (int64_t)col * ES, V - col);
    }
  }
}

// The preference loss's gradient from the rows' statistics and the pairs'
// slopes: workgroup = (row, LG_OCTETS octets).
constexpr int LG_U = 4, LG_THREADS = 256, LG_OCTETS = LG_U * LG_THREADS;
template <int DT>
__global__ __launch_bounds__(LG_THREADS) void logit_grads_kernel(LossArgs a, uint32_t parts) {
  constexpr int ES = Oct<DT>::ES;
  const uint32_t r = blockIdx.x / parts;
  const int64_t row = a.row0 + r;
  const int V = a.V, y = a.targets[row], t = (int)(row % a.T);
  const int o0 = (int)(blockIdx.x - r * parts) * LG_OCTETS + (int)threadIdx.x;
  const char* z = (const char*)a.Z + row * a.ldz * ES;
  char* g = (char*)a.Gz + row * a.ldg * ES;
  const RowStat st = a.stat[row];
  float w = a.w[row / a.T];
  if (t >= a.split) w = -w;
  Oct<DT> v[LG_U];
  if (y < 0 || y >= V || w == 0.f || st.scale == 0.f) {
    const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    v[0].set(none);
#pragma unroll
    for (int u = 0; u < LG_U; ++u) {
      const int col = (o0 + u * LG_THREADS) * 8;
      v[0].store(g + (int64_t)col * ES, V - col);
    }
    return;
  }
  const float f = w * st.scale;
#pragma unroll
  for (int u = 0; u < LG_U; ++u) {
    const int col = (o0 + u * LG_THREADS) * 8;
    v[u].load(z + (int64_t)col * ES, V - col, NEG_INF<DT>);
  }
#pragma unroll
  for (int u = 0; u < LG_U; ++u) {
    const int col = (o0 + u * LG_THREADS) * 8;
    grad_octet<DT>(v[u], st.top, f, w, y - col);
    v[u].store(g + (int64_t)col * ES, V - col);
  }
}

// One workgroup per pair: the two sums of log-ratios, in double and in a fixed order.
constexpr int PF_THREADS = 256;
__global__ __launch_bounds__(PF_THREADS) void preference_kernel(PreferenceArgs a) {
  __shared__ double red[2][PF_THREADS / WAVE];
  const int64_t b = blockIdx.x;
  double c = 0.0, r = 0.0;
  for (int t = (int)threadIdx.x; t < a.T; t += PF_THREADS) {
    const int64_t row = b * a.T + t;
    const int y = a.targets[row];
    if (y < 0 || y >= a.V) continue;
    const double d = a.logp[row] - (a.ref ? (double)a.ref[row] : 0.0);
    if (t < a.split) c += d; else r += d;
  }
  c = wave_sum_d(c);
  r = wave_sum_d(r);
  if (threadIdx.x % WAVE == 0) {
    red[0][threadIdx.x / WAVE] = c;
    red[1][threadIdx.x / WAVE] = r;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  c = r = 0.0;
  for (int w = 0; w < PF_THREADS / WAVE; ++w) {
    c += red[0][w];
    r += red[1][w];
  }
  const double beta = a.beta, eps = a.smoothing;
  const double m = beta * c - beta * r;
  const double x = exp(-fabs(m)), small = x / (1.0 + x), large = 1.0 / (1.0 + x);
  const double up = m >= 0.0 ? large : small, down = m >= 0.0 ? small : large;  // sigma(m), sigma(-m)
  const double tail = log1p(x);   // -log sigma(m) = max(-m, 0) + tail
  // Without smoothing the second term is left out: 0 * inf is NaN at m = inf.
  double loss = (1.0 - eps) * (fmax(-m, 0.0) + tail);
  if (eps > 0.0) loss += eps * (fmax(m, 0.0) + tail);
  if (m != m) loss = m;
  a.loss[b] = (float)loss;
  if (a.rewards) {
    a.rewards[2 * b] = (float)(beta * c);
    a.rewards[2 * b + 1] = (float)(beta * r);
  }
  a.slope[b] = (float)(beta * ((1.0 - eps) * down - eps * up));
}

// Threads of a row: a wave up to 2048 logits, 4 waves up to 8192, 16 above.
hipError_t launch_token_logprobs(const LossArgs& a, int dt, hipStream_t s) {
  const bool bf = dt == DT_BF16;
  if (a.rows == 0) return hipSuccess;
  const unsigned n = (unsigned)a.rows;
  if (a.V <= 2048) {
    const dim3 grid((n + 3) / 4), block(LossTeam<1>::THREADS);
    if (bf) hipLaunchKernelGGL((token_logprobs_kernel<DT_BF16, 1>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((token_logprobs_kernel<DT_F32, 1>), grid, block, 0, s, a);
  } else if (a.V <= 8192) {
    const dim3 grid(n), block(LossTeam<4>::THREADS);
    if (bf) hipLaunchKernelGGL((token_logprobs_kernel<DT_BF16, 4>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((token_logprobs_kernel<DT_F32, 4>), grid, block, 0, s, a);
  } else {
    const dim3 grid(n), block(LossTeam<16>::THREADS);
    if (bf) hipLaunchKernelGGL((token_logprobs_kernel<DT_BF16, 16>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((token_logprobs_kernel<DT_F32, 16>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

template <int DT, int W, int NV>
static hipError_t ce(const LossArgs& a, hipStream_t s) {
  const unsigned teams = LossTeam<W>::TEAMS;
  hipLaunchKernelGGL((cross_entropy_kernel<DT, W, NV>),
                     dim3((unsigned)((a.rows + teams - 1) / teams)), dim3(LossTeam<W>::THREADS), 0, s, a);
  return hipGetLastError();
}

template <int DT>
static hipError_t ce_by_width(const LossArgs& a, hipStream_t s) {
  const int octs = (a.V + 7) / 8;
  if (octs <= 64) return ce<DT, 1, 1>(a, s);
  if (octs <= 256) return ce<DT, 1, 4>(a, s);
  if (octs <= 1024) return ce<DT, 4, 4>(a, s);
  if (octs <= 4096) return ce<DT, 16, 4>(a, s);
  if (octs <= 8192) return ce<DT, 16, 8>(a, s);
  return ce<DT, 16, 0>(a, s);
}

hipError_t launch_cross_entropy(const LossArgs& a, int dt, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return dt == DT_BF16 ? ce_by_width<DT_BF16>(a, s) : ce_by_width<DT_F32>(a, s);
}

hipError_t launch_logit_grads(const LossArgs& a, int dt, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const uint32_t parts = (uint32_t)((((int64_t)a.V + 7) / 8 + LG_OCTETS - 1) / LG_OCTETS);
  const dim3 grid((unsigned)(a.rows * parts)), block(LG_THREADS);
  if (dt == DT_BF16) hipLaunchKernelGGL((logit_grads_kernel<DT_BF16>), grid, block, 0, s, a, parts);
  else hipLaunchKernelGGL((logit_grads_kernel<DT_F32>), grid, block, 0, s, a, parts);
  return hipGetLastError();
}

hipError_t launch_preference(const PreferenceArgs& a, int B, hipStream_t s) {
  hipLaunchKernelGGL(preference_kernel, dim3((unsigned)B), dim3(PF_THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace dpg
