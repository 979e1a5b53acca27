// LayerNorm of every token and its backward pass with per-example gradients of
// gain and bias (part of vector.hip).
//
// Forward: xhat = (x - mean) rstd, y = gain xhat + bias, with the mean and the
// variance of the row's d features (the mean first, then the squares about it,
// both from registers) and rstd = 1 / sqrt(variance + eps).
// Backward, with g = gain gy: dx = rstd (g - mean(g) - xhat mean(g xhat)).
// Example i's gradients are sums over its tokens, as for every vector parameter
// here: dgain_i = sum_t gy xhat, dbias_i = sum_t gy (the chain rule of
// vec_reduce_kernel, which wants xhat in memory; here it is formed from x and
// the saved statistics), and the flat norm takes ||dgain_i||^2 + ||dbias_i||^2.
//
// Both passes are bound by HBM: 2 (forward) or 3 (backward) elements a feature, 16 bytes a lane and
// access (fp32 rows of 5000 by 32 bytes a lane, 4 x 1000 backward: 80 us, so 72). Measured: 32 x 128 x 768
// bf16 forward 6.3 us (2.0 TB/s, launch and one round of rows), backward 8.4 + 3.4 us; 16 x 1024 x 1600
// bf16 30 and 47 us (3.5 TB/s), 32 x 1024 x 768 backward 40 (3.8); 2 x 8191 x 1601 fp32 backward 67 + 10
// us (4.7 TB/s in the first launch, whose 252 registers leave one workgroup a CU).
// A row is read once into the registers of a team, one wave up to 2048
// features (its sums need no barrier), 4 waves up to 4096, 16 up to 32768, and
// both sums of a row meet in one exchange. A lane holds the same features of
// every row it meets, so the token sums of dgain and dbias stay in its
// registers; a workgroup covers a range of an example's rows, and ranges are
// added in order by a second launch (no atomics: results do not depend on
// timing). One range per example needs none.
#pragma once
#include "rows.hpp"

namespace dpg {

constexpr int LN_WAVES = 8;   // waves of a workgroup whose teams are single waves

template <int W>
struct LnTeam {
  static constexpr int THREADS = W == 1 ? LN_WAVES * WAVE : W * WAVE;
  static constexpr int TEAMS = W == 1 ? LN_WAVES : 1;
};

// N of a parameter's d elements of either type from col on; a null one is `none`.
template <int N>
__device__ __forceinline__ void ln_params(const void* p, int dt, int col, int d, float none, float (&v)[N]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = none;
  } else if (dt == DT_BF16) {
    if constexpr (N == 8) {
      Oct<DT_BF16> o;
      o.load((const char*)p + (int64_t)col * 2, d - col);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = o.at(e);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = col + e < d ? bf16_to_f32(((const uint16_t*)p)[col + e]) : 0.f;
    }
  } else {
    Oct<DT_F32, N> o;
    o.load((const char*)p + (int64_t)col * 4, d - col);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = o.at(e);
  }
}

// A lane's units of a row.
template <int DT, int W, int NV>
__device__ __forceinline__ void ln_load(const void* base, int64_t ld, int64_t row, int lane, int d, Unit<DT> (&v)[NV]) {
  const char* p = (const char*)base + row * ld * Unit<DT>::ES;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (lane + j * W * WAVE) * Unit<DT>::N;
    v[j].load(p + (int64_t)col * Unit<DT>::ES, d - col);
  }
}
// Whether the next row is fetched while this one is worked on: rows of up to 16 elements a lane.
template <int DT, int W, int NV>
constexpr bool LN_AHEAD = NV * Unit<DT>::N <= 16 && NV * Unit<DT>::N * W <= 128;

template <int DT, int W, int NV>
__global__ __launch_bounds__(LnTeam<W>::THREADS) void ln_forward_kernel(LnForwardArgs a) {
  __shared__ float red[2 * W];
  constexpr int LANES = W * WAVE, N = Unit<DT>::N;
  const int lane = (int)threadIdx.x % LANES, team = (int)threadIdx.x / LANES;
  const int d = a.d;
  const float inv_d = 1.f / (float)d;
  const int64_t step = (int64_t)gridDim.x * LnTeam<W>::TEAMS;
  int64_t row = (int64_t)blockIdx.x * LnTeam<W>::TEAMS + team;
  if (row >= a.rows) return;   // a whole team
  Unit<DT> v[NV], next[NV];
  ln_load<DT, W, NV>(a.x, a.ldx, row, lane, d, v);
  float gain[NV][N], bias[NV][N];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    ln_params(a.gain, a.param_dt, (lane + j * LANES) * N, d, 1.f, gain[j]);
    ln_params(a.bias, a.param_dt, (lane + j * LANES) * N, d, 0.f, bias[j]);
  }
  for (; row < a.rows; row += step) {
    // The next row is on its way while this one is worked on.
    const bool more = row + step < a.rows;
    constexpr bool AHEAD = LN_AHEAD<DT, W, NV>;
    if (AHEAD && more) ln_load<DT, W, NV>(a.x, a.ldx, row + step, lane, d, next);
    char* y = (char*)a.y + row * a.ldy * Unit<DT>::ES;
    float sum = 0.f, none = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) sum += v[j].at(e);
    team_sum2<W>(sum, none, red);
    const float about = sum * inv_d;
    float sq = 0.f, rest = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float c = v[j].at(e) - about;
        if ((lane + j * LANES) * N + e < d) {
          sq = fmaf(c, c, sq);
          rest += c;
        }
      }
    team_sum2<W>(sq, rest, red);
    // The first mean is off by its roundings; the differences tell by how much.
    rest *= inv_d;
    const float mean = about + rest;
    const float var = fmaxf(fmaf(-rest, rest, sq * inv_d), 0.f);
    const float rstd = 1.f / sqrtf((sq != sq ? sq : var) + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (lane + j * LANES) * N;
      float o[N];
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = fmaf((v[j].at(e) - mean) * rstd, gain[j][e], bias[j][e]);
      v[j].set(o);
      v[j].store(y + (int64_t)col * Unit<DT>::ES, d - col);
    }
    if (lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    if (more) {
      if constexpr (AHEAD) {
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = next[j];
      } else {
        ln_load<DT, W, NV>(a.x, a.ldx, row + step, lane, d, v);
      }
    }
  }
}

// Rows of 513 to 1024 features: values that the second pass over a row could use again, and second
// copies of the running sums, are not kept in registers, so that two workgroups fit a CU instead of one
// (fp32 then without the next row; 32 x 1024 x 768 bf16 42.5 us, so 39.9; 32 x 512 x 768 fp32 39.0,
// 36.8); nor are those of more than 4096, whose 16 waves leave each lane 128 registers (8 x 512 x 12288 bf16 117,
// 103). Elsewhere it only costs (16 x 1024 x 1600 bf16 47.3 and 48.4).
template <int DT, int W, int NV>
constexpr bool LN_LEAN = W == 1 ? NV * Unit<DT>::N == 16 : W == 16;
// Rows of more than 16384 features: the gain waits in LDS (8 x 512 x 20480 bf16 233 us, 780 with all of it in
// registers, most of them spilled; 2 x 1024 x 20480 fp32 233 and 319).
template <int DT, int W, int NV>
constexpr bool LN_GAIN_LDS = W == 16 && NV * Unit<DT>::N == 32;

// Item: (example b, range s of a.span rows). DX: dx is wanted; WG: the gradients are.
template <int DT, int W, int NV, bool DX, bool WG>
__global__ __launch_bounds__(LnTeam<W>::THREADS) void ln_backward_kernel(LnBackwardArgs a) {
  constexpr int LANES = W * WAVE, TEAMS = LnTeam<W>::TEAMS, N = Unit<DT>::N;
  __shared__ float red[2 * W];
  __shared__ float meet[WG && TEAMS > 1 ? TEAMS : 1][WG && TEAMS > 1 ? 2 * N * WAVE : 1];
  __shared__ float sq_red[LnTeam<W>::THREADS / WAVE];
  const int lane = (int)threadIdx.x % LANES, team = (int)threadIdx.x / LANES;
  const uint32_t item = xcd_remap(blockIdx.x, gridDim.x);
  const int bl = (int)(item / (uint32_t)a.ranges), s = (int)(item - (uint32_t)bl * a.ranges);
  const int b = a.b0 + bl;
  const int d = a.d;
  const float inv_d = 1.f / (float)d;
  const int t0 = s * a.span, t1 = t0 + min(a.span, a.T - t0);
  const int64_t row0 = (int64_t)b * a.T;
  Unit<DT> x[NV], g[NV];
  float mean = 0.f, rstd = 0.f;
  auto fetch = [&](int t, Unit<DT> (&px)[NV], Unit<DT> (&pg)[NV], float& m, float& r) __attribute__((always_inline)) {
    ln_load<DT, W, NV>(a.x, a.ldx, row0 + t, lane, d, px);
    ln_load<DT, W, NV>(a.gy, a.ldgy, row0 + t, lane, d, pg);
    m = a.mean[row0 + t];
    r = a.rstd[row0 + t];
  };
  if (t0 + team < t1) fetch(t0 + team, x, g, mean, rstd);
  constexpr bool GL = LN_GAIN_LDS<DT, W, NV> && DX;
  __shared__ float gain_s[GL ? NV * N * LANES : 1];   // a lane reads what it wrote
  float gain[GL ? 1 : NV][N];
  auto gain_of = [&](int j, int e) __attribute__((always_inline)) {
    if constexpr (GL) return gain_s[(j * N + e) * LANES + lane];
    else return gain[j][e];
  };
  float dg[NV][N], db[NV][N];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (DX) ln_params(a.gain, a.param_dt, (lane + j * LANES) * N, d, 1.f, gain[GL ? 0 : j]);
    if constexpr (GL) {
#pragma unroll
      for (int e = 0; e < N; ++e) gain_s[(j * N + e) * LANES + lane] = gain[0][e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) dg[j][e] = db[j][e] = 0.f;
  }
  for (int t = t0 + team; t < t1; t += TEAMS) {
    const int64_t row = row0 + t;
    // The next row is on its way while this one is worked on, where registers allow.
    constexpr bool LEAN = LN_LEAN<DT, W, NV>, AHEAD = LN_AHEAD<DT, W, NV> && !(LEAN && WG && DT == DT_F32);
    Unit<DT> nx[NV], ng[NV];
    float nm = 0.f, nr = 0.f;
    const bool more = t + TEAMS < t1;
    if (AHEAD && more) fetch(t + TEAMS, nx, ng, nm, nr);
    float s1 = 0.f, s2 = 0.f;
    // Features past d have gy = 0 here, so their xhat drops out of every sum.
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float gy = g[j].at(e), xh = (x[j].at(e) - mean) * rstd;
        if constexpr (WG) {
          dg[j][e] = fmaf(gy, xh, dg[j][e]);
          db[j][e] += gy;
          if constexpr (LEAN) asm volatile("" : "+v"(dg[j][e]), "+v"(db[j][e]));
        }
        if constexpr (DX) {
          const float w = gy * gain_of(j, e);
          s1 += w;
          s2 = fmaf(w, xh, s2);
        }
      }
    if constexpr (DX) {
      team_sum2<W>(s1, s2, red);
      if constexpr (LEAN) {   // without the gradients too, so that dx has the same bits
#pragma unroll
        for (int j = 0; j < NV; ++j) asm volatile("" : "+v"(x[j].r[0]), "+v"(g[j].r[0]));
      }
      const float c1 = s1 * inv_d, c2 = s2 * inv_d;
      char* pd = (char*)a.dx + row * a.lddx * Unit<DT>::ES;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int col = (lane + j * LANES) * N;
        float o[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float xh = (x[j].at(e) - mean) * rstd;
          o[e] = rstd * (g[j].at(e) * gain_of(j, e) - c1 - xh * c2);
        }
        if (a.accumulate_dx) {
          Unit<DT> p;
          p.load(pd + (int64_t)col * Unit<DT>::ES, d - col);
#pragma unroll
          for (int e = 0; e < N; ++e) o[e] += p.at(e);
        }
        x[j].set(o);
        x[j].store(pd + (int64_t)col * Unit<DT>::ES, d - col);
      }
    }
    if (more) {
      if constexpr (AHEAD) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          x[j] = nx[j];
          g[j] = ng[j];
        }
        mean = nm;
        rstd = nr;
      } else {
        fetch(t + TEAMS, x, g, mean, rstd);
      }
    }
  }
  if constexpr (WG) {
    // The teams' sums meet in LDS, one unit of every lane at a time.
    float* part = a.ranges > 1 ? a.ws + ((int64_t)b * a.ranges + s) * 2 * d : nullptr;
    float* out_g = part ? part : a.dgain ? a.dgain + (int64_t)b * d : nullptr;
    float* out_b = part ? part + d : a.dbias ? a.dbias + (int64_t)b * d : nullptr;
    float sq = 0.f;
    auto put = [&](int col, bool bias, float v) {
      float* out = bias ? out_b : out_g;
      if (col >= d) return;
      if (out) out[col] = v;
      if (bias ? a.dbias : a.dgain) sq = fmaf(v, v, sq);
    };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (TEAMS > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < N; ++e) {
          meet[team][e * WAVE + lane] = dg[j][e];
          meet[team][(N + e) * WAVE + lane] = db[j][e];
        }
        __syncthreads();
#pragma unroll
        for (int q0 = 0; q0 < 2 * N; q0 += TEAMS) {   // a team takes every eighth of a unit's 2 N sums
          const int q = q0 + team;
          float v = 0.f;
#pragma unroll
          for (int w = 0; w < TEAMS; ++w) v += meet[w][q * WAVE + lane];
          put((lane + j * LANES) * N + q % N, q >= N, v);
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          put((lane + j * LANES) * N + e, false, dg[j][e]);
          put((lane + j * LANES) * N + e, true, db[j][e]);
        }
      }
    }
    if (a.ranges == 1 && a.norm2) {
      sq = wave_sum(sq);
      if (threadIdx.x % WAVE == 0) sq_red[threadIdx.x / WAVE] = sq;
      __syncthreads();
      if (threadIdx.x == 0) {
        float v = 0.f;
        for (int w = 0; w < LnTeam<W>::THREADS / WAVE; ++w) v += sq_red[w];
        a.norm2[b] = (a.accumulate ? a.norm2[b] : 0.f) + v;
      }
    }
  }
}
static_assert(LN_WAVES == 8, "2 N sums of a unit in whole turns");

// The ranges' partial sums of example blockIdx.y. FEW (at most LN_FEW ranges): a thread adds
// a feature's, in order, one workgroup per example, which writes the norm too. Otherwise
// LN_FIN_COLS features a workgroup, by 16 groups of threads that each add every
// sixteenth range (then the groups, in order); each leaves a partial of the norm, or, where there
// is one, the norm. (8192 tokens of 64 features 13 us in all; by one workgroup's threads, a chain
// of 512 loads and additions each, 28.)
constexpr int LN_FIN_COLS = 64, LN_FIN_GROUPS = 16, LN_FIN_THREADS = LN_FIN_COLS * LN_FIN_GROUPS;
template <bool FEW>
__global__ __launch_bounds__(LN_FIN_THREADS) void ln_finish_kernel(LnBackwardArgs a) {
  const int b = (int)blockIdx.y, d = a.d;
  const float* ws = a.ws + (int64_t)b * a.ranges * 2 * d;
  float sq = 0.f;
  auto put = [&](int col, float vg, float vb) {
    if (a.dgain) { a.dgain[(int64_t)b * d + col] = vg; sq = fmaf(vg, vg, sq); }
    if (a.dbias) { a.dbias[(int64_t)b * d + col] = vb; sq = fmaf(vb, vb, sq); }
  };
  if constexpr (FEW) {
    __shared__ float red[LN_FIN_THREADS / WAVE];
    for (int col = (int)threadIdx.x; col < d; col += LN_FIN_THREADS) {
      float vg = 0.f, vb = 0.f;
#pragma unroll 8
      for (int s = 0; s < a.ranges; ++s) {
        vg += ws[(int64_t)s * 2 * d + col];
        vb += ws[(int64_t)s * 2 * d + d + col];
      }
      put(col, vg, vb);
    }
    if (!a.norm2) return;
    sq = wave_sum(sq);
    if (threadIdx.x % WAVE == 0) red[threadIdx.x / WAVE] = sq;
    __syncthreads();
    if (threadIdx.x != 0) return;
    sq = 0.f;
    for (int w = 0; w < LN_FIN_THREADS / WAVE; ++w) sq += red[w];
    a.norm2[b] = (a.accumulate ? a.norm2[b] : 0.f) + sq;
  } else {
    __shared__ float meet[LN_FIN_GROUPS][2][LN_FIN_COLS];
    const int c = (int)threadIdx.x % LN_FIN_COLS, grp = (int)threadIdx.x / LN_FIN_COLS;
    const int col = (int)blockIdx.x * LN_FIN_COLS + c;
    float vg = 0.f, vb = 0.f;
    if (col < d) {
#pragma unroll 8
      for (int s = grp; s < a.ranges; s += LN_FIN_GROUPS) {
        vg += ws[(int64_t)s * 2 * d + col];
        vb += ws[(int64_t)s * 2 * d + d + col];
      }
    }
    meet[grp][0][c] = vg;
    meet[grp][1][c] = vb;
    __syncthreads();
    if (grp != 0) return;
    if (col < d) {
      vg = vb = 0.f;
#pragma unroll
      for (int q = 0; q < LN_FIN_GROUPS; ++q) {
        vg += meet[q][0][c];
        vb += meet[q][1][c];
      }
      put(col, vg, vb);
    }
    if (!a.norm2) return;
    sq = wave_sum(sq);
    if (threadIdx.x != 0) return;
    if (gridDim.x == 1) a.norm2[b] = (a.accumulate ? a.norm2[b] : 0.f) + sq;
    else a.sq[(int64_t)b * gridDim.x + blockIdx.x] = sq;
  }
}

template <int DT, int W, int NV>
static hipError_t ln_forward(const LnForwardArgs& a, hipStream_t s) {
  const int64_t need = (a.rows + LnTeam<W>::TEAMS - 1) / LnTeam<W>::TEAMS;
  // As many workgroups as the registers let the GPU hold: rows beyond are prefetched.
  constexpr int64_t MOST = 256 * (W == 1 ? (NV * Unit<DT>::N == 8 ? 4 : NV * Unit<DT>::N == 16 ? 3 : 2) : W == 4 ? 4 : 2);
  const unsigned grid = (unsigned)(need < MOST ? need : MOST);
  hipLaunchKernelGGL((ln_forward_kernel<DT, W, NV>), dim3(grid), dim3(LnTeam<W>::THREADS), 0, s, a);
  return hipGetLastError();
}

template <int DT, int W, int NV>
static hipError_t ln_backward(LnBackwardArgs a, hipStream_t s) {
  const dim3 block(LnTeam<W>::THREADS);
  const bool wg = a.dgain || a.dbias;
  hipError_t e = hipSuccess;
  const int most = (int)(MAX_GROUPS / a.ranges);   // examples of a launch
  for (int64_t b0 = 0; b0 < a.B && e == hipSuccess; b0 += most) {
    a.b0 = (int)b0;
    const dim3 grid((unsigned)((a.B - b0 < most ? a.B - b0 : most) * a.ranges));
    if (a.dx && wg)
      hipLaunchKernelGGL((ln_backward_kernel<DT, W, NV, true, true>), grid, block, 0, s, a);
    else if (a.dx)
      hipLaunchKernelGGL((ln_backward_kernel<DT, W, NV, true, false>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((ln_backward_kernel<DT, W, NV, false, true>), grid, block, 0, s, a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || a.ranges == 1 || !wg) return e;
  const dim3 fin(LN_FIN_THREADS);
  if (a.ranges <= LN_FEW) {
    hipLaunchKernelGGL((ln_finish_kernel<true>), dim3(1, (unsigned)a.B), fin, 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((ln_finish_kernel<false>), dim3((unsigned)a.chunks, (unsigned)a.B), fin, 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess || !a.norm2 || a.chunks == 1) return e;
  return launch_finish_rows(a.sq, a.B, a.chunks, a.norm2, a.accumulate, 1.f, s);
}

// Calls f<W, NV> for the team that holds rows of d features (F units are 8 of them).
#define DPG_LN_TEAMS(FN, DT)                           \
  do {                                                 \
    constexpr int F = 8 / Unit<DT>::N;                 \
    const int octs = (a.d + 7) / 8;                    \
    if (octs <= 64) return FN<DT, 1, F>(a, s);         \
    if (octs <= 128) return FN<DT, 1, 2 * F>(a, s);    \
    if (octs <= 256) return FN<DT, 1, 4 * F>(a, s);    \
    if (octs <= 512) return FN<DT, 4, 2 * F>(a, s);    \
    if (octs <= 1024) return FN<DT, 16, F>(a, s);      \
    if (octs <= 2048) return FN<DT, 16, 2 * F>(a, s);  \
    return FN<DT, 16, 4 * F>(a, s);                    \
  } while (0)

hipError_t launch_ln_forward(const LnForwardArgs& a, int dt, hipStream_t s) {
  if (dt == DT_BF16) DPG_LN_TEAMS(ln_forward, DT_BF16);
  DPG_LN_TEAMS(ln_forward, DT_F32);
}

hipError_t launch_ln_backward(const LnBackwardArgs& a, int dt, hipStream_t s) {
  if (dt == DT_BF16) DPG_LN_TEAMS(ln_backward, DT_BF16);
  DPG_LN_TEAMS(ln_backward, DT_F32);
}
#undef DPG_LN_TEAMS

}  // namespace dpg
