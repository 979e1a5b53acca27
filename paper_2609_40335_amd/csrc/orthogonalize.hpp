// Orthogonalised updates: Newton-Schulz products that drive a matrix's singular
// values towards 1, as the Muon optimiser applies to a momentum (part of misc.hip).
//
// X_0 = G / (||G||_F + eps), taken along the shorter side (m <= n), then
//   A = X X^T,  P = a I + b A + c A^2,  X <- P X        (once per step)
// and out = (prior) + scale X. A and A^2 are symmetric: only tiles on and above
// the diagonal are computed, and stored twice. So a step costs
// m(m+1)n + m^2(m+1) + 2 m^2 n operations in three launches for the whole group. Bound by the
// matrix cores, where launches have whole rounds of long tiles: GPT-2's 48 block matrices 98 us for A,
// 43 for A^2 and 168 for the update (780 TFLOP/s), 195 to 235 where it carries X by itself (510 MB
// more to move), 1.87 ms in five steps; 1601 x 6397 with two planes 108 us an update (920 TFLOP/s of
// fp16 products), 1.03 ms in five steps.
//
// The products run on the fp16 matrix cores. Singular values are at most about
// 1.2 on the way, so that X, held as 2^12 X, and A and P, held as 2^10 A and
// 2^10 P, lie well inside fp16's range: its 11 bits round 8 times finer than
// bf16's at the same rate.
// What is rounded off X, or off a in P = aI + b A + c A^2, falls on all directions of X, and those
// beside a few leading ones grow a-fold a step (485-fold in five). So X is held in two planes, and
// goes into the update by itself, X <- a X + (b A + c A^2) X, in 32 bits (see a.own).
//   PL = 1 (bf16 results): one fp16 plane per operand of a product, whose error is 2e-4 of
//     X (with nothing else, a matrix of rank 8 came out 4.8e-2 off). The last two states of X
//     make do with it, and with P = aI + ...: there b A + c A^2 is as large as a, and
//     a X without the product of x1 would be further off than neither. Five steps on noisy
//     sums come to 0.9e-3 to 1.4e-3 of the result against fp64, at rank 8 to 2.7e-3, and
//     rounding the result to bf16 is 1.7e-3 by itself.
//   PL = 2 (fp32 results): two planes, x = x0 + x1 with x1 what is left (22 bits
//     together), and the three products x0 y0 + x0 y1 + x1 y0; x1 y1 is below
//     2^-22. Never further off than 32-bit products: 1e-6 for sums under noise (theirs 1.3e-6 to
//     4.4e-6), growing as theirs do beside a few leading directions (512 x 1024 of rank 8 1.7e-5, theirs
//     2.0e-5; of rank 32 1.0e-5 and 1.1e-5, with P = aI + ... in every step 2.0e-5). The last step,
//     whose roundings grow no more, has its a in P.
// Sums are fp32 in the matrix cores, the Frobenius norm is in fp64.
//
// Layout: m and n are padded with zeros to multiples of a tile, so that the
// products have no edges. X is kept as Y = X^T [n, m], twice, as the update reads
// one while it writes the other. A buffer's blocks of 16 rows and 32 columns are
// 1 KB each and lie one behind the other along its columns, so that a wave loads and
// stores whole KBs (a load of 64 bytes from each of 16 rows took a third longer); a
// block's 16-byte chunks stand as LDS wants them, chunk c of row r at
// c ^ (r / 2 % 4), which spreads the reads of a fragment over all banks. A A and P Y^T
// are sums over columns of both operands, so that a fragment is 16 bytes of a row;
// Y^T Y is one over rows, whose fragments the transposing LDS reads collect.
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

// Partial sums of squares of G, in double: item = (matrix, part). Units of 16 bytes, eight in
// flight. NT: streaming loads, here and in the next kernel, for a group that the
// memory-side cache does not hold anyway (GPT-2's 340 MB: 57 + 97 us with them, 86 + 82 without).
template <int DT, bool NT>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsArgs args) {
  const NsArgs& a = *(const NsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  (void)args;
  __shared__ double red[4];
  const int ln = (int)(threadIdx.x & (WAVE - 1));
  const int l = wave_find(blockIdx.x, ln < a.n ? a.M[ln].item_begin : 0u, a.n);
  const NsMat& M = a.M[l];
  constexpr uint32_t N = Unit<DT>::N;
  const uint32_t part = blockIdx.x - M.item_begin, parts = (uint32_t)ns_parts(M.rows, M.cols);
  // A matrix without gaps is one long row.
  const bool flat = M.ldg == M.cols;
  const int cols = flat ? M.rows * M.cols : M.cols;
  const uint32_t per_row = ((uint32_t)cols + N - 1) / N, total = flat ? per_row : per_row * (uint32_t)M.rows;
  const uint32_t stride = parts * 256;
  constexpr int U = 8;   // units in flight
  double sum = 0.0;
  for (uint32_t o = part * 256 + threadIdx.x; o < total; o += U * stride) {
    Unit<DT> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t at = o + u * stride, r = flat ? 0u : at / per_row, c = (at - r * per_row) * N;
      v[u].template load<NT>((const char*)M.G + ((int64_t)r * M.ldg + c) * Unit<DT>::ES, at < total ? cols - (int)c : 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < (int)N; ++e) sum = fma((double)v[u].at(e), (double)v[u].at(e), sum);
  }
  sum = wave_sum_d(sum);
  if (ln == 0) red[threadIdx.x / WAVE] = sum;
  __syncthreads();
  if (threadIdx.x == 0) ((double*)M.ws)[part] = red[0] + red[1] + red[2] + red[3];
}

// Byte offset of the 16-byte chunk at position q of row r's 4 in block (r / 16, k32) of
// a buffer with K columns, and the chunk (of 8 k) that stands there.
__device__ __forceinline__ int64_t ns_at(int r, int k32, int q, int K) {
  return ((int64_t)(r >> 4) * (K / 32) + k32) * 1024 + (r & 15) * 64 + q * 16;
}
__device__ __forceinline__ int ns_chunk(int r, int q) { return q ^ ((r >> 1) & 3); }

// The 16-byte chunks of eight values' planes.
template <int PL>
__device__ __forceinline__ void ns_cut(float (&v)[8], f16x8 (&h)[PL]) {
#pragma unroll
  for (int p = 0; p < PL; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[p][e] = (_Float16)v[e];
      v[e] -= (float)h[p][e];
    }
}

// Y_0 from G: workgroup = 64 x 64 of the padded Y. Both planes, or (PL = 1, not a.fine_next) one.
template <int DT, int PL, bool NT>
__global__ __launch_bounds__(256) void ns_convert_kernel(NsArgs args) {
  const NsArgs& a = *(const NsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  (void)args;
  __shared__ float tile[64][65];
  __shared__ double red[4];
  const int tid = (int)threadIdx.x, ln = tid & (WAVE - 1);
  const int l = wave_find(blockIdx.x, ln < a.n ? a.M[ln].item_begin : 0u, a.n);
  const NsMat& M = a.M[l];
  const uint32_t item = blockIdx.x - M.item_begin;
  const int tn = M.mp / 64;
  const int i0 = (int)(item / (uint32_t)tn) * 64, j0 = (int)(item % (uint32_t)tn) * 64;
  const bool flip = M.rows <= M.cols;   // Y's rows run along the longer side
  const int r0 = flip ? j0 : i0, c0 = flip ? i0 : j0;
  // Two octets of G a thread, requested before the norm is read.
  Oct<DT> g[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int r = r0 + (tid >> 3) + 32 * u, c = c0 + (tid & 7) * 8;
    g[u].template load<NT>((const char*)M.G + ((int64_t)r * M.ldg + c) * Oct<DT>::ES, r < M.rows ? M.cols - c : 0);
  }
  double sq = 0.0;
  for (int p = tid; p < ns_parts(M.rows, M.cols); p += 256) sq += ((const double*)M.ws)[p];
  sq = wave_sum_d(sq);
  if (ln == 0) red[tid / WAVE] = sq;
  __syncthreads();
  const double norm = sqrt(red[0] + red[1] + red[2] + red[3]) + (double)a.eps;
  // The scaled element is rounded once: 1/norm in double, times an exact value.
  const double f = (double)NS_SX / norm;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int r = (tid >> 3) + 32 * u, c = (tid & 7) * 8;
    const int have = r0 + r < M.rows ? M.cols - (c0 + c) : 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // Padding stays zero where the factor is not finite.
      const float v = e < have ? (float)((double)g[u].at(e) * f) : 0.f;
      if (flip) tile[c + e][r] = v; else tile[r][c + e] = v;
    }
  }
  __syncthreads();
  // 8 blocks of 16 rows and 32 columns, a wave two of them.
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int blk = (tid >> 6) + 4 * u, rb = (blk >> 1) * 16, kb = (blk & 1) * 32;
    const int r = rb + (ln >> 2), q = ln & 3, k = kb + ns_chunk(r, q) * 8;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = tile[r][k + e];
    f16x8 h[2];
    ns_cut<2>(x, h);
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (p < PL || a.fine_next)
        *(f16x8*)((char*)ns_plane(M, NS_Y0, p, PL) + ns_at(i0 + r, (j0 + kb) / 32, q, M.mp)) = h[p];
  }
}

// The products. A workgroup of 4 waves (2 x 2) makes a tile of 64 FM x 64 FN of C,
// a wave 32 FM x 32 FN of it. Stages of 32 k lie in a ring of RING in LDS, loaded straight
// into it (16 bytes a lane). The
// fragments of the next 16 k are read while the present ones are multiplied, one
// read behind every few matrix instructions. In the middle of stage s a wave waits
// for its own loads of stage s + 1, and the barrier behind that tells that everyone's have
// landed and that nobody reads stage s - 1 any more, whose slot the loads of stage
// s + RING - 1 then fill. Stages past the end read zeros through the range check,
// so that the wait counts are constants.
constexpr int NS_BK = 32;
constexpr int NS_EP_LD = 36;   // floats per row of a wave's 32 x 32 epilogue slice

typedef __bf16 ns_b16x4 __attribute__((ext_vector_type(4)));   // any 16-bit type
typedef __attribute__((address_space(3))) ns_b16x4 ns_lds_b16x4;
__device__ __forceinline__ u32x2 ns_read_tr(const ns_lds_t* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((ns_lds_b16x4*)p));
}

template <int N>
__device__ __forceinline__ void ns_wait() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

__device__ __forceinline__ f32x16 mfma32_f16(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The last update's 32 x 32 block at (bi, bj) of X, whose columns are the rows of `slice`,
// to out (X or its transpose): octets of any alignment.
__device__ __forceinline__ void ns_give(const NsArgs& a, const NsMat& M, const float* slice, int lane,
                                        int bi, int bj) {
  const float scale = M.scale * (1.f / (NS_SX * NS_SA));
  const bool flip = M.rows <= M.cols;
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const int r = (lane >> 2) + 16 * it, c = (lane & 3) * 8;
    const int row = (flip ? bi : bj) + r, col = (flip ? bj : bi) + c;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = scale * (flip ? slice[(c + e) * NS_EP_LD + r] : slice[r * NS_EP_LD + c + e]);
    if (row >= M.rows || col >= M.cols) continue;
    auto put = [&](auto oct) __attribute__((always_inline)) {
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
}

// A block's rows to the slice of a wave: slice row j holds column j of the block, or (T) slice row i its row i.
template <bool T>
__device__ __forceinline__ void ns_fill(float* slice, const f32x16& c, int lane) {
  const int fr = lane & 31;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int jj = 8 * g + 4 * (lane >> 5);
    if constexpr (!T) {
      *(f32x4*)(slice + fr * NS_EP_LD + jj) = f32x4{c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) slice[(jj + r) * NS_EP_LD + fr] = c[4 * g + r];
    }
  }
}

// Eight consecutive floats of a slice row.
__device__ __forceinline__ void ns_take(const float* slice, int r, int c, float (&v)[8]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x4 x = *(const f32x4*)(slice + r * NS_EP_LD + c + 4 * q);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * q + e] = x[e];
  }
}

// a I + b A + c A^2 of eight elements of A^2 (v, times NS_SA^2) and of A (x, times
// NS_SA) at row and columns col .., times NS_SA.
__device__ __forceinline__ void ns_poly(float (&v)[8], const float (&x)[8], const float* coef, int row, int col) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = fmaf(v[e], coef[2] / NS_SA, coef[1] * x[e]);
    if (row == col + e) v[e] = fmaf(coef[0], NS_SA, v[e]);
  }
}

// A 32 x 32 block of the slice to rows row0 .. and columns col0 .. of a buffer: two KBs,
// one per 16 rows. POLY and UPDATE add other terms from `have`, the chunks of A or X of the same places.
template <int P>
struct NsHave {
  f16x8 y[2][P];
  __device__ __forceinline__ void load(const NsMat& M, int which, int pl, int row0, int col0, int lane) {
#pragma unroll
    for (int it = 0; it < 2; ++it)
#pragma unroll
      for (int p = 0; p < P; ++p)
        y[it][p] = *(const f16x8*)((const char*)ns_plane(M, which, p, pl) +
                                   ns_at(row0 + (lane >> 2) + 16 * it, col0 / 32, lane & 3, M.mp));
  }
  __device__ __forceinline__ void sum(int it, float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)y[it][P - 1][e];
#pragma unroll
    for (int p = P - 2; p >= 0; --p)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += (float)y[it][p][e];
  }
};
template <int PL, int KIND, int P>
__device__ __forceinline__ void ns_keep(const NsArgs& a, const NsMat& M, const float* slice, int lane, int row0,
                                        int col0, int dst, const NsHave<P>& have) {
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const int r = (lane >> 2) + 16 * it, q = lane & 3, c = ns_chunk(r, q) * 8;
    float v[8];
    ns_take(slice, r, c, v);
    const int64_t at = ns_at(row0 + r, col0 / 32, q, M.mp);
    if constexpr (KIND == NS_POLY) {
      float x[8];
      have.sum(it, x);
      ns_poly(v, x, a.coef, row0 + r, col0 + c);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= KIND == NS_GRAM ? NS_SA / (NS_SX * NS_SX) : 1.f / NS_SA;
    }
    constexpr bool FINE = KIND == NS_UPDATE;
    if constexpr (FINE)
      if (a.own != 0.f) {
        float x[8];
        have.sum(it, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(a.own, x[e], v[e]);
      }
    constexpr int TO = KIND == NS_UPDATE ? 2 : PL;
    f16x8 h[TO];
    ns_cut<TO>(v, h);
#pragma unroll
    for (int p = 0; p < TO; ++p) {
      if (p >= PL && !a.fine_next) continue;
      f16x8* to = (f16x8*)((char*)ns_plane(M, dst, p, PL) + at);
      // Y is read by other XCDs next, and is larger than the L2s.
      if constexpr (KIND == NS_UPDATE) __builtin_nontemporal_store(h[p], to); else *to = h[p];
    }
  }
}

// The tile of item rel of a symmetric product: tiles on and above the diagonal, column
// by column (column j has j + 1 of them).
__device__ __forceinline__ void ns_triangle(uint32_t rel, int& ti, int& tj) {
  tj = (int)((sqrtf(8.f * (float)rel + 1.f) - 1.f) * 0.5f);
  while ((uint32_t)(tj + 1) * (uint32_t)(tj + 2) / 2 <= rel) ++tj;
  while ((uint32_t)tj * (uint32_t)(tj + 1) / 2 > rel) --tj;
  ti = (int)(rel - (uint32_t)tj * (uint32_t)(tj + 1) / 2);
}

// Ring depth and workgroups per CU (160 KB of LDS; at least 3 stages).
template <int PL, int FM, int FN>
struct NsShape {
  static constexpr int STAGE = PL * 64 * (FM + FN) * NS_BK * 2;
  static constexpr int GROUPS = 3 * STAGE * 2 <= 160 * 1024 && FM * FN <= 8 ? 2 : 1;
  static constexpr int FIT = 160 * 1024 / GROUPS / STAGE;
  static constexpr int DEEP = FM * FN == 1 ? 8 : 4;   // small tiles: latency is all there is
  static constexpr int RING = FIT > DEEP ? DEEP : FIT;
  static_assert(RING >= 3, "a stage is loaded two ahead");
};

// Where a part's sums lie: wave w's block (of 4) of item `slot`, floats 4 q .. of every lane.
__device__ __forceinline__ f32x4* ns_partial(float* part, uint32_t slot, int w, int block, int q, int lane) {
  return (f32x4*)(part + (((size_t)slot * 4 + w) * 4 + block) * 1024 + q * 256 + lane * 4);
}

// KIND: NS_GRAM, NS_POLY, NS_UPDATE, or NS_LAST, the last step's update, which goes to out.
// PART: for a launch of few tiles with long sums; an item is one of a.ks ranges of a
// tile's k and leaves its sums in a.part, for ns_join_kernel.
template <int PL, int KIND, int FM, int FN, bool PART>
__global__ __launch_bounds__(256, (NsShape<PL, FM, FN>::GROUPS)) void ns_gemm_kernel(NsArgs args) {
  const NsArgs& a = *(const NsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  (void)args;
  using S = NsShape<PL, FM, FN>;
  constexpr int ROWB = NS_BK * 2, BM = 64 * FM, BN = 64 * FN;
  constexpr int PLP = BM * ROWB, PLQ = BN * ROWB, OPQ = PL * PLP, STAGE = S::STAGE, RING = S::RING;
  constexpr int LOADS = PL * (FM + FN);   // KB loads per wave and stage
  __shared__ __align__(1024) char ring[RING * STAGE];
  static_assert(4 * 32 * NS_EP_LD * 4 <= RING * STAGE, "epilogue slices fit the ring");
  static_assert(STAGE == 4 * LOADS * 1024, "one KB per load");

  const int lane = (int)(threadIdx.x & (WAVE - 1));
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
  const uint32_t xcd = blockIdx.x % N_XCD, item = a.xcd_begin[xcd] + blockIdx.x / N_XCD;
  if (item >= a.xcd_begin[xcd + 1]) return;
  const int l = wave_find(item, lane < a.n ? a.M[lane].item_begin : 0u, a.n);
  const NsMat& M = a.M[l];
  uint32_t rel = item - M.item_begin;
  uint32_t range = 0;
  if constexpr (PART) {
    range = rel % (uint32_t)a.ks;
    rel /= (uint32_t)a.ks;
  }
  int ti, tj;
  constexpr bool SYM = KIND == NS_GRAM || KIND == NS_POLY;
  if constexpr (!SYM) {
    const int mt = (M.mp + BM - 1) / BM;
    tj = (int)(rel / (uint32_t)mt);
    ti = (int)(rel - (uint32_t)tj * mt);
  } else {
    static_assert(!SYM || FM == FN, "mirrored tiles are square");
    ns_triangle(rel, ti, tj);
  }
  const int K = KIND == NS_GRAM ? M.np : M.mp;
  const int y_now = a.step & 1 ? NS_Y1 : NS_Y0, y_next = a.step & 1 ? NS_Y0 : NS_Y1;
  const int src_p = KIND == NS_GRAM ? y_now : KIND == NS_POLY ? NS_A : NS_P;
  const int src_q = KIND == NS_POLY ? NS_A : y_now;
  const int i0 = ti * BM, j0 = tj * BN;

  // Wave w loads KBs FM w .. of P's stage and FN w .. of Q's: 16 rows each, or (GRAM) 16
  // rows of k by 32 columns, KB 2 c + h the columns 32 c .. and the k half h. Of a
  // tile that reaches past the matrix it loads the last rows instead: they
  // only meet elements of C past it too.
  constexpr bool KROWS = KIND == NS_GRAM;
  const uint32_t row_kb = (uint32_t)(M.mp / 32) * 1024;   // 16 rows of any buffer
  auto records = [&](int src, int plane, uint32_t rows16) __attribute__((always_inline)) {
    const uint64_t base = (uint64_t)ns_plane(M, src, plane, PL);
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)base),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32)),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)(rows16 * row_kb)), (uint32_t)RSRC_WORD3};
  };
  u32x4 dp[PL], dq[PL];
#pragma unroll
  for (int p = 0; p < PL; ++p) {
    dp[p] = records(src_p, p, (uint32_t)(KROWS ? M.np : M.mp) / 16);
    dq[p] = records(src_q, p, (uint32_t)(KIND == NS_POLY ? M.mp : M.np) / 16);
  }
  auto first = [&](int t0, int q, int F, int have) __attribute__((always_inline)) {
    const int kb = w * F + q;
    if constexpr (KROWS) return (uint32_t)(kb & 1) * row_kb + (uint32_t)min(t0 / 32 + (kb >> 1), have / 32 - 1) * 1024;
    else return (uint32_t)min(t0 / 16 + kb, have / 16 - 1) * row_kb;
  };
  uint32_t op[FM], oq[FN];   // offsets of the wave's KBs of stage 0
#pragma unroll
  for (int q = 0; q < FM; ++q) op[q] = first(i0, q, FM, M.mp);
#pragma unroll
  for (int q = 0; q < FN; ++q) oq[q] = first(j0, q, FN, SYM ? M.mp : M.np);
  const uint32_t stage_step = KROWS ? 2 * row_kb : 1024u;
  const uint32_t lvo = (uint32_t)lane * 16;
  const uint32_t ring_base = (uint32_t)(uintptr_t)(ns_lds_t*)ring;
  const int all_s = K / NS_BK;   // stages of the tile, of which this item takes nS from s0 on
  const int s0 = PART ? (int)((int64_t)all_s * range / a.ks) : 0;
  const int nS = PART ? (int)((int64_t)all_s * (range + 1) / a.ks) - s0 : all_s;
  // Load t of stage s.
  auto issue = [&](int s, int t) __attribute__((always_inline)) {
    const bool is_p = t < PL * FM;
    const int u = is_p ? t : t - PL * FM, F = is_p ? FM : FN;
    const int p = u / F, q = u % F;
    const uint32_t k0 = s < nS ? (uint32_t)(s0 + s) * stage_step : 0u;
    const uint32_t vo = s < nS ? lvo : 0x80000000u;   // past the end: outside the records (< 2 GiB)
    const uint32_t dst = ring_base + (uint32_t)(s % RING) * STAGE + (is_p ? p * PLP : OPQ + p * PLQ) +
                         (uint32_t)(w * F + q) * 1024;
    const uint32_t m0v = (uint32_t)__builtin_amdgcn_readfirstlane((int)dst);
    const uint32_t so = (uint32_t)__builtin_amdgcn_readfirstlane((int)(k0 + (is_p ? op[q] : oq[q])));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(m0v), "v"(vo), "s"(is_p ? dp[p] : dq[p]), "s"(so));
  };

  const int wm = (w >> 1) * 32 * FM, wn = (w & 1) * 32 * FN;
  const int fr = lane & 31, fx = (fr >> 1) & 3;
  // Byte offsets of a lane in a fragment: its 16-byte chunk in k half h of row fr; or
  // (GRAM) of the two transposing reads, in whose 16-lane groups lane j addresses row j / 4
  // and columns 4 (j % 4) .. of the group's 16, and gets column j of the 4 rows.
  uint32_t fo[2];
  if constexpr (KROWS) {
    const int g = lane >> 4, jl = lane & 15;
    const int row = 8 * (g >> 1) + (jl >> 2), col = 16 * (g & 1) + 4 * (jl & 3);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = row + 4 * u;
      fo[u] = (uint32_t)(r * 64 + (ns_chunk(r, col >> 3) << 4) + (col & 7) * 2);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) fo[h] = (uint32_t)(fr * ROWB + (((2 * h + (lane >> 5)) ^ fx) << 4));
  }

  // With two planes the small products have a sum of their own: the matrix core cuts what
  // lies below a fixed distance from a sum's largest term, towards zero, so that every product on
  // the running sum costs a long one some of its last bits.
  f32x16 acc[FM][FN], little[PL == 2 ? FM : 1][PL == 2 ? FN : 1];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      acc[i][j] = f32x16{};
      if constexpr (PL == 2) little[i][j] = f32x16{};
    }

  struct Frags {
    u32x4 p[PL][FM], q[PL][FN];
  };
  constexpr int READS = PL * (FM + FN);
  auto frag = [&](const char* at, int h) __attribute__((always_inline)) {
    if constexpr (KROWS) {
      const ns_lds_t* p = (const ns_lds_t*)at + h * 1024;
      const u32x2 lo = ns_read_tr(p + fo[0]), hi = ns_read_tr(p + fo[1]);
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      return *(const u32x4*)(at + fo[h]);
    }
  };
  // 32 rows of a stage are 2 KB either way.
  auto read = [&](Frags& f, const char* st, int h, int r) __attribute__((always_inline)) {
    if (r < PL * FM)
      f.p[r / FM][r % FM] = frag(st + (r / FM) * PLP + (wm + (r % FM) * 32) * ROWB, h);
    else
      f.q[(r - PL * FM) / FN][(r - PL * FM) % FN] =
          frag(st + OPQ + ((r - PL * FM) / FN) * PLQ + (wn + ((r - PL * FM) % FN) * 32) * ROWB, h);
  };
  // The products of 16 k, with the reads of the next 16 and (LD) the loads of stage sl
  // spread among them. A lane then holds column j = lane % 32 of a block and
  // groups of 4 consecutive rows i.
  constexpr int TERMS = PL == 2 ? 3 : 1, MF = TERMS * FM * FN;
  auto half = [&](const Frags& f, Frags& nx, const char* st, int h, int sl, bool ld) __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < MF; ++k) {
      const int t = k / (FM * FN), i = (k / FN) % FM, j = k % FN;
      // small products first: x1 y0, x0 y1, then x0 y0
      const int pq = TERMS == 3 && t == 0 ? 1 : 0, pp = TERMS == 3 && t == 1 ? 1 : 0;
      f32x16& to = t < TERMS - 1 ? little[PL == 2 ? i : 0][PL == 2 ? j : 0] : acc[i][j];
      to = mfma32_f16(f.p[pp][i], f.q[pq][j], to);
#pragma unroll
      for (int r = 0; r < READS; ++r)
        if (r * MF / READS == k) read(nx, st, h, r);
      if (ld) {
#pragma unroll
        for (int t2 = 0; t2 < LOADS; ++t2)
          if (t2 * MF / LOADS == k) issue(sl, t2);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

#pragma unroll
  for (int s = 0; s < RING - 1; ++s)
#pragma unroll
    for (int t = 0; t < LOADS; ++t) issue(s, t);
  ns_wait<(RING - 2) * LOADS>();
  __syncthreads();
  Frags f0, f1;
#pragma unroll
  for (int r = 0; r < READS; ++r) read(f0, ring, 0, r);
  int slot = 0;
  for (int s = 0; s < nS; ++s) {
    __builtin_amdgcn_sched_barrier(0);
    const int next = slot + 1 == RING ? 0 : slot + 1;
    half(f0, f1, ring + slot * STAGE, 1, 0, false);
    ns_wait<(RING - 3) * LOADS>();
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    half(f1, f0, ring + next * STAGE, 0, s + RING - 1, true);
    slot = next;
  }
  if constexpr (PL == 2) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] += little[i][j];
  }
  if constexpr (PART) {   // the raw sums, four floats of every lane at a time
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *ns_partial(a.part, item, w, i * FN + j, q, lane) =
              f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    ns_wait<0>();   // loads past the end still write the ring
    return;
  }
  // POLY's other operand, all of it requested at once.
  constexpr bool POLY = KIND == NS_POLY && !PART;
  NsHave<PL> have[POLY ? FM : 1][POLY ? FN : 1][2];
  if constexpr (POLY) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int bi = i0 + wm + i * 32, bj = j0 + wn + j * 32;
        have[i][j][0].load(M, NS_A, PL, bj, bi, lane);
        have[i][j][1].load(M, NS_A, PL, bi, bj, lane);
      }
  }
  // X by itself (see a.own), DEEP blocks ahead of where it is added.
  constexpr bool FINE = KIND == NS_UPDATE;
  constexpr int DEEP = FINE ? (FM * FN < 4 ? FM * FN : 4) : 1;
  NsHave<2> mine[DEEP];
  const int jn = SYM ? M.mp : M.np;
  auto want = [&](int blk) __attribute__((always_inline)) {
    const int bi = i0 + wm + blk / FN * 32, bj = j0 + wn + blk % FN * 32;
    if (a.own != 0.f && bi < M.mp && bj < jn) mine[blk % DEEP].load(M, y_now, PL, bj, bi, lane);
  };
  if constexpr (FINE) {
#pragma unroll
    for (int blk = 0; blk < DEEP; ++blk) want(blk);
  }
  ns_wait<0>();   // loads past the end still write the ring
  __syncthreads();

  // Epilogue, one 32 x 32 block at a time through the wave's own slice.
  float* slice = (float*)ring + w * 32 * NS_EP_LD;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int bi = i0 + wm + i * 32, bj = j0 + wn + j * 32;
      const bool in = bi < M.mp && bj < jn;   // a block past the matrix is left out
      if constexpr (KIND == NS_LAST) {
        if (in) {
          ns_fill<false>(slice, acc[i][j], lane);
          ns_give(a, M, slice, lane, bi, bj);
        }
      } else {
        constexpr int dst = KIND == NS_GRAM ? NS_A : NS_P;
        const int hi = POLY ? i : 0, hj = POLY ? j : 0;
        if (in) {
          ns_fill<false>(slice, acc[i][j], lane);
          if constexpr (FINE)
            ns_keep<PL, KIND>(a, M, slice, lane, bj, bi, y_next, mine[(i * FN + j) % DEEP]);
          else
            ns_keep<PL, KIND>(a, M, slice, lane, bj, bi, SYM ? dst : y_next, have[hi][hj][0]);
          if (SYM && ti != tj) {
            ns_fill<true>(slice, acc[i][j], lane);
            ns_keep<PL, KIND>(a, M, slice, lane, bi, bj, dst, have[hi][hj][1]);
          }
        }
        if constexpr (FINE)
          if (i * FN + j + DEEP < FM * FN) want(i * FN + j + DEEP);
      }
    }
  }
}

// The parts of a split symmetric product, added in order: a workgroup takes a quarter
// (64 x 64) of a tile, a wave a 32 x 32 block of it.
template <int PL, int KIND>
__global__ __launch_bounds__(256) void ns_join_kernel(NsArgs args) {
  const NsArgs& a = *(const NsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  (void)args;
  __shared__ float slices[4][32 * NS_EP_LD];
  const int lane = (int)(threadIdx.x & (WAVE - 1));
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
  const uint32_t tile = blockIdx.x / 4, quarter = blockIdx.x % 4;
  const int l = wave_find(tile, lane < a.n ? a.M[lane].item_begin : 0u, a.n);
  const NsMat& M = a.M[l];
  int ti, tj;
  ns_triangle(tile - M.item_begin, ti, tj);
  const int bi = ti * NS_TILE + (int)(quarter >> 1) * 64 + (w >> 1) * 32;
  const int bj = tj * NS_TILE + (int)(quarter & 1) * 64 + (w & 1) * 32;
  NsHave<PL> have[2];
  if constexpr (KIND == NS_POLY) {
    have[0].load(M, NS_A, PL, bj, bi, lane);
    have[1].load(M, NS_A, PL, bi, bj, lane);
  }
  f32x16 c = {};
#pragma unroll 4
  for (int r = 0; r < a.ks; ++r)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 v = *ns_partial(a.part, tile * (uint32_t)a.ks + r, (int)quarter, w, q, lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) c[4 * q + e] += v[e];
    }
  constexpr int dst = KIND == NS_GRAM ? NS_A : NS_P;
  ns_fill<false>(slices[w], c, lane);
  ns_keep<PL, KIND>(a, M, slices[w], lane, bj, bi, dst, have[0]);
  if (ti != tj) {
    ns_fill<true>(slices[w], c, lane);
    ns_keep<PL, KIND>(a, M, slices[w], lane, bi, bj, dst, have[1]);
  }
}

// All steps of a matrix in one workgroup, its Y, A and P in LDS as the buffers' blocks (see
// above; sides padded to 32, blocks along mp). A wave takes every eighth 32 x 32 block
// of a product. An update's blocks stay in registers until every wave has read Y. With one plane X's
// blocks also stay there, in fp32, for as long as X goes into the update by itself (ns_fine).
// Bound by latency: fifteen products in a row, each a barrier, a chain of LDS reads and the turn
// through the slice. (Four matrices of a block of width 64, five steps, fp32 results: 43 us; in 17
// launches of 5 to 9 us each 143.)
template <int DT, int PL>
__global__ __launch_bounds__(NS_SMALL_WAVES * WAVE) void ns_small_kernel(NsArgs args, NsCoefs coefs) {
  const NsArgs& a = *(const NsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  (void)args;
  constexpr int W = NS_SMALL_WAVES;
  __shared__ __align__(1024) char buf[NS_SMALL_LDS];
  __shared__ float slices[W][32 * NS_EP_LD];
  __shared__ double red[W];
  const int tid = (int)threadIdx.x, lane = tid & (WAVE - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const NsMat& M = a.M[blockIdx.x];
  const int mp = M.mp, np = M.np, mb = mp / 32, nb = np / 32;
  const int planeY = np * mp * 2, planeA = mp * mp * 2;
  char *Y = buf, *A = buf + PL * planeY, *P = A + PL * planeA;
  float* slice = slices[w];

  // ||G||_F as everywhere: squares and sums in double.
  const uint32_t per_row = ((uint32_t)M.cols + 7) / 8, total = per_row * (uint32_t)M.rows;
  double sq = 0.0;
  for (uint32_t o = (uint32_t)tid; o < total; o += W * WAVE) {
    const uint32_t r = o / per_row, c = (o - r * per_row) * 8;
    Oct<DT> v;
    v.load((const char*)M.G + ((int64_t)r * M.ldg + c) * Oct<DT>::ES, M.cols - (int)c);
#pragma unroll
    for (int e = 0; e < 8; ++e) sq = fma((double)v.at(e), (double)v.at(e), sq);
  }
  sq = wave_sum_d(sq);
  if (lane == 0) red[w] = sq;
  __syncthreads();
  sq = 0.0;
  for (int i = 0; i < W; ++i) sq += red[i];
  const double f = (double)NS_SX / (sqrt(sq) + (double)a.eps);
  // Y: chunk id -> block, row of the block, position.
  const bool flip = M.rows <= M.cols;   // Y = G^T
  for (int id = tid; id < np * mp / 8; id += W * WAVE) {
    const int blk = id >> 6, r = (id >> 2) & 15, q = id & 3;
    const int j = (blk / mb) * 16 + r, i = (blk % mb) * 32 + ns_chunk(r, q) * 8;
    Oct<DT> g;
    float v[8];
    if (!flip) g.load((const char*)M.G + ((int64_t)j * M.ldg + i) * Oct<DT>::ES, j < M.rows ? M.cols - i : 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = flip ? i + e < M.rows && j < M.cols : j < M.rows && i + e < M.cols;
      float x = flip ? 0.f : g.at(e);
      if (flip && in) {
        const int64_t at = (int64_t)(i + e) * M.ldg + j;
        x = DT == DT_BF16 ? bf16_to_f32(((const uint16_t*)M.G)[at]) : ((const float*)M.G)[at];
      }
      v[e] = in ? (float)((double)x * f) : 0.f;
    }
    f16x8 h[PL];
    ns_cut<PL>(v, h);
#pragma unroll
    for (int p = 0; p < PL; ++p) *(f16x8*)(Y + p * planeY + id * 16) = h[p];
  }

  // Fragments of 32 rows (or, TR, 32 columns) of a buffer at 16 k.
  const int fr = lane & 31;
  const int tr_row = 8 * (lane >> 5) + ((lane & 15) >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  auto rows = [&](const char* b, int row32, int k) __attribute__((always_inline)) {   // rows 32 row32 .., k 16 k ..
    const int q = ns_chunk(fr, 2 * (k & 1) + (lane >> 5));
    return *(const u32x4*)(b + ((2 * row32 + (fr >> 4)) * mb + (k >> 1)) * 1024 + (fr & 15) * 64 + q * 16);
  };
  auto cols = [&](const char* b, int col32, int k) __attribute__((always_inline)) {   // columns 32 col32 .., k 16 k ..
    const ns_lds_t* p = (const ns_lds_t*)(b + (k * mb + col32) * 1024);
    u32x2 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = tr_row + 4 * u;
      x[u] = ns_read_tr(p + r * 64 + (ns_chunk(r, tr_col >> 3) << 4) + (tr_col & 7) * 2);
    }
    return u32x4{x[0][0], x[0][1], x[1][0], x[1][1]};
  };
  // A block's sum over ks steps of 16 k; fp(p, k), fq(p, k): the operands' planes.
  auto product = [&](int ks, auto fp, auto fq) __attribute__((always_inline)) {
    f32x16 big = {}, little = {};
    for (int k = 0; k < ks; k += 2) {   // ks is even: the reads of two steps are in flight together
      u32x4 x[2][PL], y[2][PL];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int p = 0; p < PL; ++p) {
          x[u][p] = fp(p, k + u);
          y[u][p] = fq(p, k + u);
        }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if constexpr (PL == 2) {
          little = mfma32_f16(x[u][1], y[u][0], little);
          little = mfma32_f16(x[u][0], y[u][1], little);
        }
        big = mfma32_f16(x[u][0], y[u][0], big);
      }
    }
    if constexpr (PL == 2) big += little;
    return big;
  };
  // The slice as rows row0 .. and columns col0 .. of a buffer, both multiples of 32.
  auto keep = [&](char* b, int plane, int row0, int col0, auto change) __attribute__((always_inline)) {
#pragma unroll
    for (int it = 0; it < 2; ++it) {
      const int r = (lane >> 2) + 16 * it, q = lane & 3, c = ns_chunk(r, q) * 8;
      float v[8];
      ns_take(slice, r, c, v);
      const int at = ((row0 / 16 + it) * mb + col0 / 32) * 1024 + lane * 16;
      change(v, at, row0 + r, col0 + c);
      f16x8 h[PL];
      ns_cut<PL>(v, h);
#pragma unroll
      for (int p = 0; p < PL; ++p) *(f16x8*)(b + p * plane + at) = h[p];
    }
  };
  auto times = [](float s) {
    return [s](float (&v)[8], int, int, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= s;
    };
  };

  // X, as Y is held (times NS_SX), where the matrix instructions leave its blocks.
  f32x16 X[PL == 1 ? NS_SMALL_BLOCKS : 1];
  if (PL == 1 && ns_fine(0, a.steps, PL)) {
#pragma unroll
    for (int u = 0; u < NS_SMALL_BLOCKS; ++u) {
      const int t = w + u * W;
      if (t < mb * nb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int i = 32 * (t % mb) + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3), j = 32 * (t / mb) + fr;
          const int r = flip ? i : j, c = flip ? j : i;
          float g = 0.f;
          if (r < M.rows && c < M.cols) {
            const int64_t at = (int64_t)r * M.ldg + c;
            g = DT == DT_BF16 ? bf16_to_f32(((const uint16_t*)M.G)[at]) : ((const float*)M.G)[at];
            g = (float)((double)g * f);
          }
          X[PL == 1 ? u : 0][e] = g;
        }
    }
  }

  for (int step = 0; step < a.steps; ++step) {
    const float* coef = coefs.c + 3 * step;
    const bool fine = ns_fine(step, a.steps, PL);
    const float cf[3] = {fine ? 0.f : coef[0], coef[1], coef[2]};
    auto poly = [&](float (&v)[8], int at, int row, int col) __attribute__((always_inline)) {
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = PL - 1; p >= 0; --p) {
        const f16x8 y = *(const f16x8*)(A + p * planeA + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += (float)y[e];
      }
      ns_poly(v, x, cf, row, col);
    };
#pragma unroll
    for (int kind = NS_GRAM; kind <= NS_POLY; ++kind) {
      __syncthreads();
      // All blocks: the mirrored ones cost a wave without work of its own nothing, where
      // storing a block twice would be another turn through the slice.
      for (int t = w; t < mb * mb; t += W) {
        const int ti = t / mb, tj = t % mb;
        const f32x16 c =
            kind == NS_GRAM
                ? product(np / 16, [&](int p, int k) { return cols(Y + p * planeY, ti, k); },
                          [&](int p, int k) { return cols(Y + p * planeY, tj, k); })
                : product(mp / 16, [&](int p, int k) { return rows(A + p * planeA, ti, k); },
                          [&](int p, int k) { return rows(A + p * planeA, tj, k); });
        ns_fill<false>(slice, c, lane);
        if (kind == NS_GRAM) keep(A, planeA, 32 * tj, 32 * ti, times(NS_SA / (NS_SX * NS_SX)));
        else keep(P, planeA, 32 * tj, 32 * ti, poly);
      }
    }
    __syncthreads();
    f32x16 c[NS_SMALL_BLOCKS];
#pragma unroll
    for (int u = 0; u < NS_SMALL_BLOCKS; ++u) {
      const int t = w + u * W;   // block (t % mb) of X's rows, t / mb of its columns
      if (t < mb * nb)
        c[u] = product(mp / 16, [&](int p, int k) { return rows(P + p * planeA, t % mb, k); },
                       [&](int p, int k) { return rows(Y + p * planeY, t / mb, k); });
      if (PL == 1 && fine) {
        c[u] += coef[0] * NS_SA * X[PL == 1 ? u : 0];
        X[PL == 1 ? u : 0] = c[u] * (1.f / NS_SA);
      }
    }
    const bool last = step == a.steps - 1;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < NS_SMALL_BLOCKS; ++u) {
      const int t = w + u * W;
      if (t < mb * nb) {
        ns_fill<false>(slice, c[u], lane);
        if (last) ns_give(a, M, slice, lane, 32 * (t % mb), 32 * (t / mb));
        else keep(Y, planeY, 32 * (t / mb), 32 * (t % mb), [&](float (&v)[8], int at, int, int) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= 1.f / NS_SA;
          if constexpr (PL == 2) {   // the X that this one takes the place of
            const f16x8 y0 = *(const f16x8*)(Y + at), y1 = *(const f16x8*)(Y + planeY + at);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(coef[0], (float)y1[e] + (float)y0[e], v[e]);
          }
        });
      }
    }
  }
}

// Work items of matrix l in a product.
template <int KIND, int FM, int FN>
static uint32_t ns_tiles(const NsMat& M) {
  const uint32_t mt = (uint32_t)((M.mp + 64 * FM - 1) / (64 * FM));
  const uint32_t nt = (uint32_t)((M.np + 64 * FN - 1) / (64 * FN));
  return KIND == NS_GRAM || KIND == NS_POLY ? mt * (mt + 1) / 2 : mt * nt;
}

// Items of one launch and how they are dealt to the XCDs: each gets a contiguous range
// of the list (neighbouring tiles share operand panels through its L2), whole
// matrices where ns_order's bins are even for this product, equal work otherwise. (In the
// caller's order, with equal counts, the Gram of GPT-2's blocks took 128 us: the XCDs
// of the longest sums were last. So dealt it takes 98 to 105.)
template <int PL, int KIND, int FM, int FN, bool PART>
static hipError_t ns_launch(NsArgs& a, const NsBins& bins, hipStream_t s) {
  uint32_t items = 0;
  double work[NS_MAX_MATS], all = 0.0;
  for (int l = 0; l < a.n; ++l) {
    const uint32_t n = ns_tiles<KIND, FM, FN>(a.M[l]) * (PART ? (uint32_t)a.ks : 1u);
    a.M[l].item_begin = items;
    items += n;
    // An item costs its k and, for its ends, about 256 k more.
    work[l] = (double)n * ((KIND == NS_GRAM ? a.M[l].np : a.M[l].mp) / (PART ? a.ks : 1) + 256);
    all += work[l];
  }
  double most = 0.0;
  for (int x = 0; x < N_XCD; ++x) {
    double sum = 0.0;
    for (int l = bins.begin[x]; l < bins.begin[x + 1]; ++l) sum += work[l];
    most = sum > most ? sum : most;
  }
  a.xcd_begin[0] = 0;
  a.xcd_begin[N_XCD] = items;
  if (most * N_XCD <= 1.15 * all) {
    for (int x = 1; x < N_XCD; ++x)
      a.xcd_begin[x] = bins.begin[x] < a.n ? a.M[bins.begin[x]].item_begin : items;
  } else {
    double before = 0.0;
    int l = 0;
    for (int x = 1; x < N_XCD; ++x) {
      const double cut = all * x / N_XCD;
      while (l < a.n - 1 && before + work[l] <= cut) before += work[l++];
      const uint32_t end = l + 1 < a.n ? a.M[l + 1].item_begin : items, n = end - a.M[l].item_begin;
      const double part = (cut - before) / work[l] * n + 0.5;
      a.xcd_begin[x] = a.M[l].item_begin + (part >= n ? n : (uint32_t)part);
    }
  }
  uint32_t longest = 0;
  for (int x = 0; x < N_XCD; ++x) {
    const uint32_t n = a.xcd_begin[x + 1] - a.xcd_begin[x];
    longest = n > longest ? n : longest;
  }
  hipLaunchKernelGGL((ns_gemm_kernel<PL, KIND, FM, FN, PART>), dim3(longest * N_XCD), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int PL, int KIND>
static hipError_t ns_symmetric(NsArgs& a, const NsBins& bins, hipStream_t s) {
  const NsPlan plan = ns_plan(a, KIND, PL);
  a.ks = plan.ks;
  if (plan.small) return ns_launch<PL, KIND, 1, 1, false>(a, bins, s);
  if constexpr (PL == 1 && KIND == NS_GRAM)
    if (plan.wide) return ns_launch<PL, KIND, 4, 4, false>(a, bins, s);
  if (a.ks == 1) return ns_launch<PL, KIND, 2, 2, false>(a, bins, s);
  const hipError_t e = ns_launch<PL, KIND, 2, 2, true>(a, bins, s);
  if (e != hipSuccess) return e;
  uint32_t tiles = 0;
  for (int l = 0; l < a.n; ++l) {
    a.M[l].item_begin = tiles;
    tiles += ns_tiles<KIND, 2, 2>(a.M[l]);
  }
  hipLaunchKernelGGL((ns_join_kernel<PL, KIND>), dim3(4 * tiles), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Large tiles: 128 x 128 for the symmetric products, whose launches have few; for updates
// 128 x 256 with one plane (fewer LDS reads per product: 171 us for GPT-2's blocks, 197 with 128 x
// 128), the last 190 us (200 with 256 x 256, which waits for its stores), 128 x 128 with two (105 us
// for 1601 x 6397, three rounds, and 331 for 4096 x 4096; with 256 x 128, whose ring has three stages
// instead of four, 116, two rounds of twice the length, and 367; either way a CU holds one workgroup).
template <int PL>
static hipError_t ns_step(NsArgs& a, const NsBins& bins, hipStream_t s) {
  constexpr int FN = PL == 1 ? 4 : 2;
  hipError_t e = ns_symmetric<PL, NS_GRAM>(a, bins, s);
  if (e == hipSuccess) e = ns_symmetric<PL, NS_POLY>(a, bins, s);
  if (e != hipSuccess) return e;
  const NsPlan plan = ns_plan(a, a.last ? NS_LAST : NS_UPDATE, PL);
  if (a.last)
    return plan.small ? ns_launch<PL, NS_LAST, 1, 1, false>(a, bins, s) : ns_launch<PL, NS_LAST, 2, FN, false>(a, bins, s);
  if (plan.small) return ns_launch<PL, NS_UPDATE, 1, 1, false>(a, bins, s);
  // With X by itself a tile's end moves three times as much, beside which a second workgroup works
  // (128 x 256 and 256 x 256, all five steps, us: GPT-2's blocks 1845, 1917; 24 x (1024 x 1024, 1024 x
  // 4096) 1745, 1808; 4096 x 4096 1668, 1664; 4096 x 16384 5063, 5038).
  if constexpr (PL == 1)
    if (plan.wide && a.own == 0.f) return ns_launch<PL, NS_UPDATE, 4, 4, false>(a, bins, s);
  return ns_launch<PL, NS_UPDATE, 2, FN, false>(a, bins, s);
}

template <int DT, int PL, bool NT>
static hipError_t ns_begin(NsArgs& a, hipStream_t s) {
  uint32_t items = 0;
  for (int l = 0; l < a.n; ++l) {
    a.M[l].item_begin = items;
    items += (uint32_t)ns_parts(a.M[l].rows, a.M[l].cols);
  }
  hipLaunchKernelGGL((ns_norm_kernel<DT, NT>), dim3(items), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  items = 0;
  for (int l = 0; l < a.n; ++l) {
    a.M[l].item_begin = items;
    items += (uint32_t)(a.M[l].mp / 64) * (uint32_t)(a.M[l].np / 64);
  }
  hipLaunchKernelGGL((ns_convert_kernel<DT, PL, NT>), dim3(items), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int DT, int PL>
static hipError_t ns_run(NsArgs a, const float* coef, int steps, hipStream_t s) {
  const NsBins bins = ns_order(a);
  int64_t bytes = 0;
  for (int l = 0; l < a.n; ++l) bytes += (int64_t)a.M[l].rows * a.M[l].cols * Oct<DT>::ES;
  a.fine_next = ns_fine(0, steps, PL) ? 1 : 0;
  hipError_t e = bytes > ((int64_t)256 << 20) ? ns_begin<DT, PL, true>(a, s) : ns_begin<DT, PL, false>(a, s);
  for (int k = 0; k < steps && e == hipSuccess; ++k) {
    for (int q = 0; q < 3; ++q) a.coef[q] = coef[3 * k + q];
    a.own = 0.f;
    if (ns_fine(k, steps, PL)) {
      a.own = a.coef[0];
      a.coef[0] = 0.f;
    }
    a.fine_next = ns_fine(k + 1, steps, PL) ? 1 : 0;
    a.step = k;
    a.last = k == steps - 1 ? 1 : 0;
    e = ns_step<PL>(a, bins, s);
  }
  return e;
}

hipError_t launch_orthogonalize_small(const NsArgs& args, int dt, int planes, const float* coef, int steps,
                                      hipStream_t s) {
  NsArgs a = args;
  NsCoefs c{};
  a.steps = steps;
  for (int k = 0; k < 3 * steps; ++k) c.c[k] = coef[k];
  const dim3 grid((unsigned)a.n), block(NS_SMALL_WAVES * WAVE);
  if (dt == DT_BF16) {
    if (planes == 1) hipLaunchKernelGGL((ns_small_kernel<DT_BF16, 1>), grid, block, 0, s, a, c);
    else hipLaunchKernelGGL((ns_small_kernel<DT_BF16, 2>), grid, block, 0, s, a, c);
  } else {
    if (planes == 1) hipLaunchKernelGGL((ns_small_kernel<DT_F32, 1>), grid, block, 0, s, a, c);
    else hipLaunchKernelGGL((ns_small_kernel<DT_F32, 2>), grid, block, 0, s, a, c);
  }
  return hipGetLastError();
}

hipError_t launch_orthogonalize(const NsArgs& a, int dt, int planes, const float* coef, int steps,
                                hipStream_t s) {
  if (dt == DT_BF16)
    return planes == 1 ? ns_run<DT_BF16, 1>(a, coef, steps, s) : ns_run<DT_BF16, 2>(a, coef, steps, s);
  return planes == 1 ? ns_run<DT_F32, 1>(a, coef, steps, s) : ns_run<DT_F32, 2>(a, coef, steps, s);
}

}  // namespace dpg
