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
// All of it is bound by HBM: a logit costs one exponential for its row's sum and
// one for its gradient, and moves 2 to 12 bytes. Cross-entropy
// keeps its row in registers between the sum and the gradient, so the logits
// are read once (a row of 50257 is 98 KB in bf16: 7 units of 16 bytes a thread of
// 1024). A pair's weight needs the last row's log p before the first row's
// gradient, so there the logits are passed twice. (Fewer pairs at a time, so that the second
// read meets the memory-side cache, was no gain: 16 pairs of 1024 rows of 50257 in bf16 took 652 us in
// one pass, 688 two at a time, 832 one by one, for the launches' ends; nor were streaming loads in the
// first pass, 684, or the rows backwards in the second, 670.)
// Measured, rows of 50257 of which a third is not scored (and not read): bf16 log-probabilities of 24 x
// 128 42 us (4.8 TB/s: few rows a CU, and an exponential for every 2 bytes), cross-entropy of 32 x 128
// 123 us (5.6 TB/s; a copy runs at 4.9), in fp32 of 24 x 100 158 us (5.1); a preference loss of 16 x 1024
// tokens 657 us, 3.9 GB in two passes (5.9).
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

// exp(d) for d <= 0. log2 e as one fp32 number is LOST off (1.3e-8 of itself), so that
// every exp(d) is off by d LOST of itself, the same way in every row: 6e-8 of a sum of
// exponentials, which a sum of hundreds of log-probabilities shows. Such sums (EXACT) add
// up d exp(d) as well and put the first order back. (As a second term of the exponent it would be
// rounded away.)
constexpr double LOST = 1.4426950408889634 / (double)LOG2E - 1.0;
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * LOG2E); }

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

// A running sum of exponentials from `top`. EXACT: in double, with that of d exp(d): a
// factor from one maximum to the next that is rounded to fp32 is off the same way wherever
// the same two maxima meet, and bf16 logits have few of them.
template <bool EXACT>
struct RunningSum {
  float top = LOWEST, sum = 0.f;
  __device__ __forceinline__ void move(float m) {
    sum *= exp_of(top - m);
    top = m;
  }
  __device__ __forceinline__ void add(float s, float) { sum += s; }
  __device__ __forceinline__ double total() const { return (double)sum; }
  template <int W>
  __device__ __forceinline__ void meet(double* red) {   // of a team
    float none = 0.f;
    move(team_max<W>(top, (float*)red));
    team_sum2<W>(sum, none, (float*)red);
  }
};
template <>
struct RunningSum<true> {
  float top = LOWEST;
  double sum = 0.0, slope = 0.0;
  __device__ __forceinline__ void move(float m) {
    if (m != top) {
      const double x = exp((double)top - (double)m);
      sum *= x;
      slope *= x;   // d up to the maximum that its exponential was taken from: x is exact
      top = m;
    }
  }
  __device__ __forceinline__ void add(float s, float t) {
    sum += (double)s;
    slope += (double)t;
  }
  __device__ __forceinline__ double total() const { return fma(LOST, slope, sum); }
  template <int W>
  __device__ __forceinline__ void meet(double* red) {
    move(team_max<W>(top, (float*)red));
    sum = wave_sum_d(sum);
    slope = wave_sum_d(slope);
    if constexpr (W > 1) {
      const int w = (int)threadIdx.x / WAVE;
      __syncthreads();
      if (threadIdx.x % WAVE == 0) {
        red[2 * w] = sum;
        red[2 * w + 1] = slope;
      }
      __syncthreads();
      sum = slope = 0.0;
      for (int i = 0; i < W; ++i) {
        sum += red[2 * i];
        slope += red[2 * i + 1];
      }
    }
  }
};

// Elements by which a row starts behind a 16-byte boundary. Its units are counted from there,
// unit u the N elements from N u - phase on, so that every whole one is an aligned access
// wherever the row starts and neighbouring lanes never share a line (rows of 50257 in bf16,
// one behind the other, so counted and from the row's start: 24 x 128 log-probabilities 47 and 55 us, their
// cross-entropy 106 and 138, a preference loss of 8 x 512 tokens 172 and 212).
template <int DT>
__device__ __forceinline__ int row_phase(const char* z) {
  return (int)((uintptr_t)z & 15) / Unit<DT>::ES;
}

// That of the lane's logits: units `lane`, `lane` + LANES, ... of the row, U of them in
// flight. EXACT rows are read a second time soon, others take streaming loads.
template <int DT, int W, int U, bool EXACT>
__device__ __forceinline__ RunningSum<EXACT> row_sum(const char* z, int V, int lane) {
  constexpr int LANES = W * WAVE, N = Unit<DT>::N;
  const int phase = row_phase<DT>(z);
  RunningSum<EXACT> s;
  for (int o = lane; o * N - phase < V; o += U * LANES) {
    Unit<DT> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (o + u * LANES) * N - phase;
      v[u].template load<!EXACT>(z + (int64_t)col * Unit<DT>::ES, V - col, NEG_INF<DT>, u ? 0 : -col);
    }
    float m = s.top;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) m = fmaxf(m, v[u].at(e));
    s.move(m);
    float part = 0.f, slope = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = v[u].at(e) - m, x = exp_of(d);
        part += x;
        if constexpr (EXACT) slope = fmaf(fmaxf(d, -200.f), x, slope);   // x is 0 below
      }
    s.add(part, slope);
  }
  return s;
}

__device__ __forceinline__ double row_logp(float zt, float top, double sum) {
  return sum == 0.0 ? -__builtin_inf() : (double)zt - (double)top - log(sum);
}

template <int DT>
__device__ __forceinline__ float logit_at(const char* z, int col) {
  if constexpr (DT == DT_BF16) return bf16_to_f32(((const uint16_t*)z)[col]);
  else return ((const float*)z)[col];
}

template <int DT, int W, int U, bool EXACT>
__global__ __launch_bounds__(LossTeam<W>::THREADS) void token_logprobs_kernel(LossArgs a) {
  __shared__ double red[2 * W];
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
  const char* z = (const char*)a.Z + row * a.ldz * Unit<DT>::ES;
  const float zt = logit_at<DT>(z, y);
  RunningSum<EXACT> s = row_sum<DT, W, U, EXACT>(z, a.V, lane);
  s.template meet<W>(red);
  if (lane == 0) {
    const double total = s.total(), logp = row_logp(zt, s.top, total);
    if (a.logp) a.logp[row] = (float)logp;
    if (a.lse) a.lse[row] = total == 0.0 ? -__builtin_inff() : (float)((double)s.top + log(total));
    if (a.logp64) a.logp64[row] = logp;
    if (a.stat) a.stat[row] = RowStat{s.top, total == 0.0 ? 0.f : (float)(1.0 / total)};
  }
}

// The gradients w p of a unit, f = w / sum. The target's is put right afterwards, by
// the thread that stored it.
template <int DT>
__device__ __forceinline__ void grad_unit(Unit<DT>& v, float top, float f) {
  float o[Unit<DT>::N];
#pragma unroll
  for (int e = 0; e < Unit<DT>::N; ++e) o[e] = exp_of(v.at(e) - top) * f;
  v.set(o);
}
template <int DT>
__device__ __forceinline__ void grad_target(char* g, int y, float zt, float top, float f, float w) {
  const float v = fmaf(exp_of(zt - top), f, -w);
  if constexpr (DT == DT_BF16)
    ((uint16_t*)g)[y] = (uint16_t)__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v, v}, bf16x2));
  else
    ((float*)g)[y] = v;
}

// Rows that give no gradient: units from `lane` on, LANES apart.
template <int DT, bool NT>
__device__ __forceinline__ void zero_row(char* g, int V, int lane, int lanes) {
  Unit<DT> v;
  const float none[Unit<DT>::N] = {};
  v.set(none);
  for (int col = lane * Unit<DT>::N - row_phase<DT>(g); col < V; col += lanes * Unit<DT>::N)
    v.template store<NT>(g + (int64_t)col * Unit<DT>::ES, V - col, -col);
}

// NV > 0: the row stays in registers, NV units a lane. NV = 0: rows longer than
// that are read again for the gradient. Loads are streaming ones, and stores where their
// units are aligned too (NT) (32 x 128 bf16 rows of 50257: 140 us without the hints, 129 with).
// (Eight waves a SIMD: a CU then works on two rows of 16 waves, one loading while the other
// computes. Longer rows, up to 24 units a lane, have a CU to themselves, which still beats reading them
// twice: 1024 bf16 rows of 65000 54 us, read twice 75; of 131072 117 and 138; of 170000 173, 4.0 TB/s, where rows
// read twice reach 3.4.)
template <int DT, int W, int NV, bool NT>
__global__ __launch_bounds__(LossTeam<W>::THREADS, DT == DT_BF16 && NV <= 8 ? 8 : 4) void cross_entropy_kernel(LossArgs a) {
  __shared__ double red[2 * W];
  __shared__ float zt_s[LossTeam<W>::TEAMS];
  constexpr int LANES = W * WAVE, ES = Unit<DT>::ES, N = Unit<DT>::N;
  const int lane = (int)threadIdx.x % LANES, team = (int)threadIdx.x / LANES;
  const int64_t r = (int64_t)blockIdx.x * LossTeam<W>::TEAMS + team;
  if (r >= a.rows) return;
  const int64_t row = a.row0 + r;
  const int V = a.V, y = a.targets[row];
  const char* z = (const char*)a.Z + row * a.ldz * ES;
  char* g = (char*)a.Gz + row * a.ldg * ES;
  const int phase = row_phase<DT>(z);
  if (y < 0 || y >= V) {
    if (lane == 0 && a.logp) a.logp[row] = 0.f;
    zero_row<DT, NT>(g, V, lane, LANES);
    return;
  }
  const float w = a.w[row];
  // In LDS before the first exchange: where the gradient replaces the logits
  // (Gz = Z) this one is overwritten.
  if (lane == 0) zt_s[team] = logit_at<DT>(z, y);
  if constexpr (W == 1) __builtin_amdgcn_wave_barrier();
  float top, sum = 0.f;
  Unit<DT> v[NV > 0 ? NV : 1];
  // Makes the row opaque: unpacked values and exponentials that a later pass over it could
  // use again would be kept, in several times its registers.
  auto hide = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) asm volatile("" : "+v"(v[j].r[0]));
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (lane + j * LANES) * N - phase;
      v[j].template load<true>(z + (int64_t)col * ES, V - col, NEG_INF<DT>, j ? 0 : -col);
    }
    top = LOWEST;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) top = fmaxf(top, v[j].at(e));
    top = team_max<W>(top, (float*)red);
    hide();
    float none = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) sum += exp_of(v[j].at(e) - top);
    team_sum2<W>(sum, none, (float*)red);
  } else {
    RunningSum<false> all = row_sum<DT, W, 4, false>(z, V, lane);
    all.meet<W>(red);
    top = all.top;
    sum = all.sum;
  }
  if (lane == 0 && a.logp) a.logp[row] = (float)row_logp(zt_s[team], top, sum);
  if (w == 0.f || sum == 0.f) {
    zero_row<DT, NT>(g, V, lane, LANES);
    return;
  }
  const float f = w / sum;
  hide();
  if constexpr (NV > 0) {
    int first = lane * N - phase;
    asm volatile("" : "+v"(first));   // opaque too: the units' places are found again
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = first + j * LANES * N;
      grad_unit<DT>(v[j], top, f);
      v[j].template store<NT>(g + (int64_t)col * ES, V - col, j ? 0 : -col);
    }
  } else {
    for (int col = lane * N - phase; col < V; col += LANES * N) {
      Unit<DT> u;
      u.template load<true>(z + (int64_t)col * ES, V - col, NEG_INF<DT>, -col);
      grad_unit<DT>(u, top, f);
      u.template store<NT>(g + (int64_t)col * ES, V - col, -col);
    }
  }
  if (((y + phase) / N) % LANES == lane) grad_target<DT>(g, y, zt_s[team], top, f, w);
}

// The preference loss's gradient from the rows' statistics and the pairs'
// slopes: workgroup = (row, LG_UNITS units).
constexpr int LG_U = 4, LG_THREADS = 256, LG_UNITS = LG_U * LG_THREADS;
template <int DT, bool NT>
__global__ __launch_bounds__(LG_THREADS) void logit_grads_kernel(LossArgs a, uint32_t parts) {
  constexpr int ES = Unit<DT>::ES, N = Unit<DT>::N;
  const uint32_t r = blockIdx.x / parts;
  const int64_t row = a.row0 + r;
  const int V = a.V, y = a.targets[row], t = (int)(row % a.T);
  const int o0 = (int)(blockIdx.x - r * parts) * LG_UNITS + (int)threadIdx.x;
  const char* z = (const char*)a.Z + row * a.ldz * ES;
  char* g = (char*)a.Gz + row * a.ldg * ES;
  const int phase = row_phase<DT>(z);
  const RowStat st = a.stat[row];
  float w = a.w[row / a.T];
  if (t >= a.split) w = -w;
  Unit<DT> v[LG_U];
  if (y < 0 || y >= V || w == 0.f || st.scale == 0.f) {
    const float none[N] = {};
    v[0].set(none);
#pragma unroll
    for (int u = 0; u < LG_U; ++u) {
      const int col = (o0 + u * LG_THREADS) * N - phase;
      v[0].template store<NT>(g + (int64_t)col * ES, V - col, u ? 0 : -col);
    }
    return;
  }
  const float f = w * st.scale;
  // The target's logit, by the thread that replaces it.
  const int yo = (y + phase) / N;
  const bool mine = yo / LG_UNITS == (int)(blockIdx.x - r * parts) && yo % LG_THREADS == (int)threadIdx.x;
  const float zt = mine ? logit_at<DT>(z, y) : 0.f;
#pragma unroll
  for (int u = 0; u < LG_U; ++u) {
    const int col = (o0 + u * LG_THREADS) * N - phase;
    v[u].template load<true>(z + (int64_t)col * ES, V - col, NEG_INF<DT>, u ? 0 : -col);
  }
#pragma unroll
  for (int u = 0; u < LG_U; ++u) {
    const int col = (o0 + u * LG_THREADS) * N - phase;
    grad_unit<DT>(v[u], st.top, f);
    v[u].template store<NT>(g + (int64_t)col * ES, V - col, u ? 0 : -col);
  }
  if (mine) grad_target<DT>(g, y, zt, st.top, f, w);
}

// One workgroup per pair: the two sums of log-ratios, in double and in a fixed order.
constexpr int PF_THREADS = 256;
__global__ __launch_bounds__(PF_THREADS) void preference_kernel(PreferenceArgs a) {
  __shared__ double red[2][PF_THREADS / WAVE];
  const int64_t b = a.b0 + (int64_t)blockIdx.x;
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

// Calls launch(args, groups) for slabs of rows, each of `per` to a workgroup.
template <typename F>
static hipError_t by_rows(LossArgs a, int64_t per, F launch) {
  const int64_t all = a.rows, most = MAX_GROUPS * per;
  for (int64_t done = 0; done < all; done += most) {
    a.rows = all - done < most ? all - done : most;
    launch(a, dim3((unsigned)((a.rows + per - 1) / per)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.row0 += a.rows;
  }
  return hipSuccess;
}

template <int DT, int W, int U, bool EXACT>
static hipError_t tl(const LossArgs& a, hipStream_t s) {
  const dim3 block(LossTeam<W>::THREADS);
  return by_rows(a, LossTeam<W>::TEAMS, [&](const LossArgs& q, dim3 grid) {
    hipLaunchKernelGGL((token_logprobs_kernel<DT, W, U, EXACT>), grid, block, 0, s, q);
  });
}

// Threads of a row: a wave up to 2048 logits, 4 waves up to 8192. Above, 16 where few rows have to fill
// the chip; where there are rows for every CU's every wave 8, or 4 with EXACT sums, whose
// ends cost more (rows then start and end at different times; 24 x 128 rows of 50257 in bf16, 4
// units in flight: 8 waves 42 us, 4 waves 45; 8 units 46; the preference loss's pass with 8
// waves made it 707 us, with 4 657, with 8 units 665).
template <int DT, bool EXACT>
static hipError_t tl_by_width(const LossArgs& a, hipStream_t s) {
  if (a.V <= 2048) return tl<DT, 1, 4, EXACT>(a, s);
  if (a.V <= 8192) return tl<DT, 4, 4, EXACT>(a, s);
  if (a.rows < 2048) return tl<DT, 16, 8, EXACT>(a, s);
  return tl<DT, EXACT ? 4 : 8, 4, EXACT>(a, s);
}

hipError_t launch_token_logprobs(const LossArgs& a, int dt, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (a.logp64) return dt == DT_BF16 ? tl_by_width<DT_BF16, true>(a, s) : tl_by_width<DT_F32, true>(a, s);
  return dt == DT_BF16 ? tl_by_width<DT_BF16, false>(a, s) : tl_by_width<DT_F32, false>(a, s);
}

template <int DT, int W, int NV, bool NT>
static hipError_t ce(const LossArgs& a, hipStream_t s) {
  return by_rows(a, LossTeam<W>::TEAMS, [&](const LossArgs& q, dim3 grid) {
    hipLaunchKernelGGL((cross_entropy_kernel<DT, W, NV, NT>), grid, dim3(LossTeam<W>::THREADS), 0, s, q);
  });
}

// Units of a row, whatever its phase (see row_phase).
template <int DT>
static int64_t row_units(const LossArgs& a) {
  constexpr int N = Unit<DT>::N;
  const bool aligned = ((uintptr_t)a.Z & 15) == 0 && (a.ldz * Unit<DT>::ES) % 16 == 0;
  return ((int64_t)a.V + (aligned ? 0 : N - 1) + N - 1) / N;
}
// Whether every row's gradient has its logits' phase, so that its stores are aligned too.
template <int DT>
static bool same_phase(const LossArgs& a) {
  return (((uintptr_t)a.Gz - (uintptr_t)a.Z) & 15) == 0 && ((a.ldg - a.ldz) * Unit<DT>::ES) % 16 == 0;
}

template <int DT, bool NT>
static hipError_t ce_by_width(const LossArgs& a, hipStream_t s) {
  const int64_t units = row_units<DT>(a);
  constexpr int F = 8 / Unit<DT>::N;   // units per 8 elements
  if (units <= 64 * F) return ce<DT, 1, F, NT>(a, s);
  if (units <= 256 * F) return ce<DT, 1, 4 * F, NT>(a, s);
  if (units <= 1024 * F) return ce<DT, 4, 4 * F, NT>(a, s);
  if (units <= 4096 * F) return ce<DT, 16, 4 * F, NT>(a, s);
  if (units <= 7168 * F) return ce<DT, 16, 7 * F, NT>(a, s);
  if (DT == DT_BF16 && units <= 8192) return ce<DT, 16, 8, NT>(a, s);
  if (units <= 16384) return ce<DT, 16, 16, NT>(a, s);
  if (units <= 24576) return ce<DT, 16, 24, NT>(a, s);
  return ce<DT, 16, 0, NT>(a, s);
}

template <int DT>
static hipError_t ce_by_type(const LossArgs& a, hipStream_t s) {
  return same_phase<DT>(a) ? ce_by_width<DT, true>(a, s) : ce_by_width<DT, false>(a, s);
}
hipError_t launch_cross_entropy(const LossArgs& a, int dt, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return dt == DT_BF16 ? ce_by_type<DT_BF16>(a, s) : ce_by_type<DT_F32>(a, s);
}

template <int DT, bool NT>
static hipError_t lg(LossArgs a, hipStream_t s) {
  const uint32_t parts = (uint32_t)((row_units<DT>(a) + LG_UNITS - 1) / LG_UNITS);
  const int64_t all = a.rows, most = 4 * MAX_GROUPS / parts;   // V <= 2^30: at least 31
  for (int64_t done = 0; done < all; done += most) {
    a.rows = all - done < most ? all - done : most;
    const dim3 grid((unsigned)(a.rows * parts));
    hipLaunchKernelGGL((logit_grads_kernel<DT, NT>), grid, dim3(LG_THREADS), 0, s, a, parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.row0 += a.rows;
  }
  return hipSuccess;
}

hipError_t launch_logit_grads(const LossArgs& a, int dt, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (dt == DT_BF16) return same_phase<DT_BF16>(a) ? lg<DT_BF16, true>(a, s) : lg<DT_BF16, false>(a, s);
  return same_phase<DT_F32>(a) ? lg<DT_F32, true>(a, s) : lg<DT_F32, false>(a, s);
}

hipError_t launch_preference(PreferenceArgs a, int B, hipStream_t s) {
  for (int64_t b0 = 0; b0 < B; b0 += MAX_GROUPS) {
    a.b0 = (int32_t)b0;
    const int64_t n = B - b0 < MAX_GROUPS ? B - b0 : MAX_GROUPS;
    hipLaunchKernelGGL(preference_kernel, dim3((unsigned)n), dim3(PF_THREADS), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace dpg
