// Orthogonalised updates: Newton-Schulz products that drive a matrix's singular
// values towards 1, as the Muon optimiser applies to a momentum (part of misc.hip).
//
// X_0 = G / (||G||_F + eps), taken along the shorter side (m <= n), then
//   A = X X^T,  P = a I + b A + c A^2,  X <- P X        (once per step)
// and out = (prior) + scale X. A and A^2 are symmetric: only tiles on and above
// the diagonal are computed, and stored twice. So a step costs
// m(m+1)n + m^2(m+1) + 2 m^2 n operations in three launches for the whole group.
//
// The products run on the fp16 matrix cores. Singular values are at most about
// 1.2 on the way, so that X, held as 2^12 X, and A and P, held as 2^10 A and
// 2^10 P, lie well inside fp16's range: its 11 bits round 8 times finer than
// bf16's at the same rate.
//   PL = 1 (bf16 results): one fp16 plane per operand. Five steps on noisy sums
//     come to 1.1e-3 to 1.5e-3 of the result against fp64, and rounding the
//     result to bf16 is 1.7e-3 by itself. (It grows with ||G||_F over the
//     size of what lies beside G's leading directions: 3e-3 at 10, 7e-3 at 30.)
//   PL = 2 (fp32 results): two planes, x = x0 + x1 with x1 what is left (22 bits
//     together), and the three products x0 y0 + x0 y1 + x1 y0; x1 y1 is below
//     2^-22. About 3e-7 in all.
// Sums are fp32 in the matrix cores, the Frobenius norm is in fp64.
//
// Layout: m and n are padded with zeros to multiples of a tile, so that the
// products have no edges. All three are C[i,j] = sum_k P[i,k] Q[j,k] with both
// operands contiguous along k: X X^T, A A^T, and P (X^T)^T, for which X is kept
// in both orientations (X^T twice, as the update reads one while it writes the other).
#pragma once
#include "rows.hpp"

namespace dpg {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char ns_lds_t;

constexpr float NS_SX = 4096.f, NS_SA = 1024.f;   // what X, and A and P, are held times

// Byte offsets of a matrix's buffers (see NsMat) from its workspace.
__device__ __forceinline__ uint16_t* ns_plane(const NsMat& M, int which, int plane, int pl) {
  return (uint16_t*)(M.ws + ns_offset(M.mp, M.np, which, plane, pl));
}

// Partial sums of squares of G, in double: item = (matrix, part).
template <int DT>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsArgs args) {
  const NsArgs& a = *(const NsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  (void)args;
  __shared__ double red[4];
  const int ln = (int)(threadIdx.x & (WAVE - 1));
  const int l = wave_find(blockIdx.x, ln < a.n ? a.M[ln].item_begin : 0u, a.n);
  const NsMat& M = a.M[l];
  const uint32_t part = blockIdx.x - M.item_begin, parts = (uint32_t)ns_parts(M.rows, M.cols);
  const uint32_t per_row = ((uint32_t)M.cols + 7) / 8, total = per_row * (uint32_t)M.rows;
  double sum = 0.0;
  for (uint32_t o = part * 256 + threadIdx.x; o < total; o += parts * 256) {
    const uint32_t r = o / per_row, c = (o - r * per_row) * 8;
    Oct<DT> v;
    v.load((const char*)M.G + ((int64_t)r * M.ldg + c) * Oct<DT>::ES, M.cols - (int)c);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)v.at(e), (double)v.at(e), sum);
  }
  sum = wave_sum_d(sum);
  if (ln == 0) red[threadIdx.x / WAVE] = sum;
  __syncthreads();
  if (threadIdx.x == 0) ((double*)M.ws)[part] = red[0] + red[1] + red[2] + red[3];
}

__device__ __forceinline__ uint16_t f16_bits(float v) {
  return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// X_0 and its transpose from G: workgroup = 64 x 64 of the padded X.
template <int DT, int PL>
__global__ __launch_bounds__(256) void ns_convert_kernel(NsArgs args) {
  const NsArgs& a = *(const NsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  (void)args;
  __shared__ float tile[64][65];
  __shared__ double red[4];
  const int ln = (int)(threadIdx.x & (WAVE - 1)), w = (int)threadIdx.x / WAVE;
  const int l = wave_find(blockIdx.x, ln < a.n ? a.M[ln].item_begin : 0u, a.n);
  const NsMat& M = a.M[l];
  const uint32_t item = blockIdx.x - M.item_begin;
  const int tn = M.np / 64;
  const int i0 = (int)(item / (uint32_t)tn) * 64, j0 = (int)(item % (uint32_t)tn) * 64;
  const bool flip = M.rows > M.cols;
  double sq = 0.0;
  for (int p = (int)threadIdx.x; p < ns_parts(M.rows, M.cols); p += 256) sq += ((const double*)M.ws)[p];
  sq = wave_sum_d(sq);
  if (ln == 0) red[w] = sq;
  __syncthreads();
  const double norm = sqrt(red[0] + red[1] + red[2] + red[3]) + (double)a.eps;
  // The scaled element is rounded once: 1/norm in double, times an exact value.
  const double f = (double)NS_SX / norm;
  const int r0 = flip ? j0 : i0, c0 = flip ? i0 : j0;
  for (int r = w; r < 64; r += 4) {
    float v = 0.f;
    if (r0 + r < M.rows && c0 + ln < M.cols) {
      const int64_t at = (int64_t)(r0 + r) * M.ldg + c0 + ln;
      const float g = DT == DT_BF16 ? bf16_to_f32(((const uint16_t*)M.G)[at]) : ((const float*)M.G)[at];
      v = (float)((double)g * f);
    }
    if (flip) tile[ln][r] = v; else tile[r][ln] = v;
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < PL; ++p) {
    uint16_t* x = ns_plane(M, NS_X, p, PL);
    uint16_t* xt = ns_plane(M, NS_XT0, p, PL);
    for (int r = w; r < 64; r += 4) {
      float u = tile[r][ln], v = tile[ln][r];
      if (p == 1) {
        u -= (float)(_Float16)u;
        v -= (float)(_Float16)v;
      }
      x[(int64_t)(i0 + r) * M.np + j0 + ln] = f16_bits(u);
      xt[(int64_t)(j0 + r) * M.mp + i0 + ln] = f16_bits(v);
    }
  }
}

// The products. Tile 128 x 128 of C, 4 waves of 64 x 64; stages of 32 k in a ring
// of NS_RING, loaded straight into LDS (16 bytes a lane; LDS rows are 64 bytes, and
// chunk c of row r lies at c ^ (r / 2 % 4), which spreads 8 rows' reads of one chunk over all
// banks). A stage's loads are issued NS_RING - 1 stages ahead; every wave waits for
// its own and a barrier tells that everyone's have landed, and that the slot
// read before is free. Stages past the end read zeros through the range check, so
// that the wait counts are constants.
constexpr int NS_BK = 32, NS_RING = 4;
constexpr int NS_EP_LD = 36;   // floats per row of a wave's 32 x 32 epilogue slice

template <int N>
__device__ __forceinline__ void ns_wait() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

__device__ __forceinline__ f32x16 mfma32_f16(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <int PL, int KIND>
__global__ __launch_bounds__(256) void ns_gemm_kernel(NsArgs args) {
  const NsArgs& a = *(const NsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  (void)args;
  constexpr int ROWB = NS_BK * 2, PLANE = NS_TILE * ROWB, OP = PL * PLANE, STAGE = 2 * OP;
  constexpr int RING = PL == 1 ? NS_RING : 2;
  constexpr int LOADS = STAGE / 1024 / 4;   // KB loads per wave and stage
  __shared__ __align__(1024) char ring[RING * STAGE];
  static_assert(4 * 32 * NS_EP_LD * 4 <= RING * STAGE, "epilogue slices fit the ring");

  const int lane = (int)(threadIdx.x & (WAVE - 1));
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
  const uint32_t item = xcd_remap(blockIdx.x, gridDim.x);
  const int l = wave_find(item, lane < a.n ? a.M[lane].item_begin : 0u, a.n);
  const NsMat& M = a.M[l];
  uint32_t rel = item - M.item_begin;
  const int mt = M.mp / NS_TILE, nt = M.np / NS_TILE;
  int ti, tj;
  if constexpr (KIND == NS_UPDATE) {
    tj = (int)(rel / (uint32_t)mt);
    ti = (int)(rel - (uint32_t)tj * mt);
  } else {   // tiles on and above the diagonal, column by column: column j has j + 1
    tj = (int)((sqrtf(8.f * (float)rel + 1.f) - 1.f) * 0.5f);
    while ((uint32_t)(tj + 1) * (uint32_t)(tj + 2) / 2 <= rel) ++tj;
    while ((uint32_t)tj * (uint32_t)(tj + 1) / 2 > rel) --tj;
    ti = (int)(rel - (uint32_t)tj * (uint32_t)(tj + 1) / 2);
  }
  (void)nt;
  const int K = KIND == NS_GRAM ? M.np : M.mp;
  const int src_p = KIND == NS_GRAM ? NS_X : KIND == NS_POLY ? NS_A : NS_P;
  const int src_q = KIND == NS_GRAM ? NS_X : KIND == NS_POLY ? NS_A : (a.step & 1 ? NS_XT1 : NS_XT0);
  const int i0 = ti * NS_TILE, j0 = tj * NS_TILE;

  // Waves 0, 1 load P's rows, waves 2, 3 Q's: 64 rows each, 16 rows a load.
  const bool is_p = w < 2;
  const uint32_t ldb = (uint32_t)K * 2;
  const int row_base = (is_p ? i0 : j0) + (w & 1) * 64;
  u32x4 desc[PL];
#pragma unroll
  for (int p = 0; p < PL; ++p) {
    const uint64_t base = (uint64_t)ns_plane(M, is_p ? src_p : src_q, p, PL) + (uint64_t)row_base * ldb;
    desc[p] = u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)base),
                    (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32)),
                    (uint32_t)__builtin_amdgcn_readfirstlane((int)(64 * ldb)), (uint32_t)RSRC_WORD3};
  }
  const int lr = lane >> 2;   // row of a load
  const uint32_t lvo = (uint32_t)lr * ldb + (uint32_t)(((lane & 3) ^ ((lr >> 1) & 3)) * 16);
  const uint32_t ring_base = (uint32_t)(uintptr_t)(ns_lds_t*)ring + (uint32_t)((is_p ? 0 : OP) + (w & 1) * 64 * ROWB);
  const int nS = K / NS_BK;
  auto issue = [&](int s) __attribute__((always_inline)) {
    const uint32_t k0 = s < nS ? (uint32_t)s * ROWB : 64u * ldb;
#pragma unroll
    for (int t = 0; t < LOADS; ++t) {
      const int p = t / 4, q = t % 4;
      const uint32_t m0v = (uint32_t)__builtin_amdgcn_readfirstlane(
          (int)(ring_base + (uint32_t)(s % RING) * STAGE + p * PLANE + q * 1024));
      const uint32_t so = (uint32_t)__builtin_amdgcn_readfirstlane((int)(k0 + (uint32_t)q * 16 * ldb));
      asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                   :: "s"(m0v), "v"(lvo), "s"(desc[p]), "s"(so));
    }
  };
  static_assert(LOADS == 4 * PL, "four loads per plane");

  const int wm = (w >> 1) * 64, wn = (w & 1) * 64;
  const int fr = lane & 31, fx = (fr >> 1) & 3;
  uint32_t fo[2];   // byte offset of the lane's chunk in k half h of row fr
#pragma unroll
  for (int h = 0; h < 2; ++h) fo[h] = (uint32_t)(fr * ROWB + (((2 * h + (lane >> 5)) ^ fx) << 4));

  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x16{};

#pragma unroll
  for (int s = 0; s < RING - 1; ++s) issue(s);
  for (int s = 0; s < nS; ++s) {
    ns_wait<(RING - 2) * LOADS>();
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    issue(s + RING - 1);
    const char* st = ring + (s % RING) * STAGE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 fp[PL][2], fq[PL][2];
#pragma unroll
      for (int p = 0; p < PL; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          fp[p][i] = *(const u32x4*)(st + p * PLANE + (wm + i * 32) * ROWB + fo[h]);
          fq[p][i] = *(const u32x4*)(st + OP + p * PLANE + (wn + i * 32) * ROWB + fo[h]);
        }
      // Q first: a lane then holds row i = lane % 32 of a block and groups of 4 consecutive j.
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if constexpr (PL == 2) {
            acc[i][j] = mfma32_f16(fq[1][j], fp[0][i], acc[i][j]);
            acc[i][j] = mfma32_f16(fq[0][j], fp[1][i], acc[i][j]);
          }
          acc[i][j] = mfma32_f16(fq[0][j], fp[0][i], acc[i][j]);
        }
    }
  }
  ns_wait<0>();   // loads past the end still write the ring
  __syncthreads();

  // Epilogue, one 32 x 32 block at a time through the wave's own slice, in one
  // orientation and then the other: lanes take 8 consecutive elements of a row.
  float* slice = (float*)ring + w * 32 * NS_EP_LD;
  constexpr bool SYM = KIND != NS_UPDATE;
  const float ca = a.coef[0], cb = a.coef[1], cc = a.coef[2];
  const bool last = KIND == NS_UPDATE && a.last;
  const bool flip = M.rows > M.cols;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int o = 0; o < 2; ++o) {   // o = 1: transposed
        if (SYM && o == 1 && ti == tj) continue;
        if (last && (o == 1) != flip) continue;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int jj = 8 * g + 4 * (lane >> 5);
          if (o == 0) {
            *(f32x4*)(slice + fr * NS_EP_LD + jj) = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1],
                                                          acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) slice[(jj + r) * NS_EP_LD + fr] = acc[i][j][4 * g + r];
          }
        }
        const int bi = i0 + wm + i * 32, bj = j0 + wn + j * 32;
        const int rb = o == 0 ? bi : bj, cb0 = o == 0 ? bj : bi;
#pragma unroll
        for (int it = 0; it < 2; ++it) {
          const int lr2 = (lane >> 2) + 16 * it;
          const int row = rb + lr2, col = cb0 + (lane & 3) * 8;
          float v[8];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const f32x4 x = *(const f32x4*)(slice + lr2 * NS_EP_LD + (lane & 3) * 8 + 4 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = x[e];
          }
          if (last) {
            const int n_rows = flip ? M.np : M.mp;
            (void)n_rows;
            if (row < M.rows && col < M.cols) {
              const float f = M.scale * (1.f / (NS_SX * NS_SA));
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] *= f;
              auto put = [&](auto oct) {
                char* p = (char*)M.out + ((int64_t)row * M.ldo + col) * decltype(oct)::ES;
                if (a.accumulate) {
                  oct.load(p, M.cols - col);
#pragma unroll
                  for (int e = 0; e < 8; ++e) v[e] += oct.at(e);
                }
                oct.set(v);
                oct.store(p, M.cols - col);
              };
              if (a.out_dt == DT_BF16) put(Oct<DT_BF16>()); else put(Oct<DT_F32>());
            }
            continue;
          }
          const int64_t at = (int64_t)row * (KIND == NS_UPDATE && o == 0 ? M.np : M.mp) + col;
          if constexpr (KIND == NS_GRAM) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= NS_SA / (NS_SX * NS_SX);
          } else if constexpr (KIND == NS_POLY) {
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = PL - 1; p >= 0; --p) {
              const f16x8 y = *(const f16x8*)(ns_plane(M, NS_A, p, PL) + at);
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] += (float)y[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[e] = fmaf(v[e], cc / NS_SA, cb * x[e]);
              if (row == col + e) v[e] = fmaf(ca, NS_SA, v[e]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= 1.f / NS_SA;
          }
          const int dst = KIND == NS_GRAM ? NS_A : KIND == NS_POLY ? NS_P
                          : o == 0 ? NS_X : (a.step & 1 ? NS_XT0 : NS_XT1);
#pragma unroll
          for (int p = 0; p < PL; ++p) {
            f16x8 h;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              h[e] = (_Float16)v[e];
              v[e] -= (float)h[e];
            }
            *(f16x8*)(ns_plane(M, dst, p, PL) + at) = h;
          }
        }
      }
}

template <int PL>
static hipError_t ns_product(NsArgs& a, int kind, hipStream_t s) {
  uint32_t items = 0;
  for (int l = 0; l < a.n; ++l) {
    const uint32_t mt = (uint32_t)(a.M[l].mp / NS_TILE), nt = (uint32_t)(a.M[l].np / NS_TILE);
    a.M[l].item_begin = items;
    items += kind == NS_UPDATE ? mt * nt : mt * (mt + 1) / 2;
  }
  const dim3 grid(items), block(256);
  if (kind == NS_GRAM) hipLaunchKernelGGL((ns_gemm_kernel<PL, NS_GRAM>), grid, block, 0, s, a);
  else if (kind == NS_POLY) hipLaunchKernelGGL((ns_gemm_kernel<PL, NS_POLY>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((ns_gemm_kernel<PL, NS_UPDATE>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <int DT, int PL>
static hipError_t ns_run(NsArgs a, const float* coef, int steps, hipStream_t s) {
  uint32_t items = 0;
  for (int l = 0; l < a.n; ++l) {
    a.M[l].item_begin = items;
    items += (uint32_t)ns_parts(a.M[l].rows, a.M[l].cols);
  }
  hipLaunchKernelGGL((ns_norm_kernel<DT>), dim3(items), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  items = 0;
  for (int l = 0; l < a.n; ++l) {
    a.M[l].item_begin = items;
    items += (uint32_t)(a.M[l].mp / 64) * (uint32_t)(a.M[l].np / 64);
  }
  hipLaunchKernelGGL((ns_convert_kernel<DT, PL>), dim3(items), dim3(256), 0, s, a);
  e = hipGetLastError();
  for (int k = 0; k < steps && e == hipSuccess; ++k) {
    for (int q = 0; q < 3; ++q) a.coef[q] = coef[3 * k + q];
    a.step = k;
    a.last = k == steps - 1 ? 1 : 0;
    for (int kind : {NS_GRAM, NS_POLY, NS_UPDATE}) {
      e = ns_product<PL>(a, kind, s);
      if (e != hipSuccess) break;
    }
  }
  return e;
}

hipError_t launch_orthogonalize(const NsArgs& a, int dt, int planes, const float* coef, int steps,
                                hipStream_t s) {
  if (dt == DT_BF16)
    return planes == 1 ? ns_run<DT_BF16, 1>(a, coef, steps, s) : ns_run<DT_BF16, 2>(a, coef, steps, s);
  return planes == 1 ? ns_run<DT_F32, 1>(a, coef, steps, s) : ns_run<DT_F32, 2>(a, coef, steps, s);
}

}  // namespace dpg
