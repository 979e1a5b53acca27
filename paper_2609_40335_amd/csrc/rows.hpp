// Octets (8 consecutive elements) and 16-byte units of rows of any alignment, and sums over
// the threads that share a row. A part of the sources that include it.
#pragma once
#include "common.hpp"

namespace dpg {

constexpr float LOG2E = 1.4426950408889634f;

typedef __attribute__((address_space(1))) u32x4_any global_u32x4_any_w;
// NT: a hint that the line is not used again soon.
template <bool NT>
__device__ __forceinline__ void store16_any(char* p, const u32x4& v) {
  if constexpr (NT) __builtin_nontemporal_store(v, (global_u32x4_any_w*)(uintptr_t)p);
  else *(global_u32x4_any_w*)(uintptr_t)p = v;
}
template <bool NT>
__device__ __forceinline__ u32x4 load16_hint(const char* p) {
  if constexpr (NT) return __builtin_nontemporal_load((global_u32x4_any*)(uintptr_t)p);
  else return load16_any(p);
}

// N consecutive elements' bits as loaded: an octet is 16 bytes of bf16, 32 of fp32.
template <int DT, int N_ = 8>
struct Oct {
  static constexpr int ES = DT == DT_BF16 ? 2 : 4, N = N_, R = N * ES / 16;
  u32x4 r[R];

  // Elements [lo, n) at p (n may be past N, or not above lo: nothing is read; lo may be below 0);
  // the others are `fill`, as bits of the type twice in a dword (bf16) or once (fp32).
  template <bool NT = false>
  __device__ __forceinline__ void load(const char* p, int64_t n, uint32_t fill = 0u, int lo = 0) {
    if (n >= N && lo <= 0) {
#pragma unroll
      for (int q = 0; q < R; ++q) r[q] = load16_hint<NT>(p + 16 * q);
      return;
    }
    if constexpr (DT == DT_BF16) {
      r[0] = u32x4{fill, fill, fill, fill};
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < n && e >= lo) {
          const uint32_t v = ((global_u16*)(uintptr_t)p)[e];
          r[0][e >> 1] = (e & 1) ? (r[0][e >> 1] & 0xFFFFu) | (v << 16) : (r[0][e >> 1] & 0xFFFF0000u) | v;
        }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) r[e >> 2][e & 3] = e < n && e >= lo ? ((const uint32_t*)p)[e] : fill;
    }
  }

  __device__ __forceinline__ float at(int e) const {
    if constexpr (DT == DT_BF16)
      return __uint_as_float((e & 1) ? r[0][e >> 1] & 0xFFFF0000u : r[0][e >> 1] << 16);
    else
      return __uint_as_float(r[e >> 2][e & 3]);
  }

  // Rounds N values to the type (to nearest even; NaN stays NaN).
  __device__ __forceinline__ void set(const float (&v)[N]) {
    if constexpr (DT == DT_BF16) {
#pragma unroll
      for (int q = 0; q < N / 2; ++q)
        r[0][q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * q], v[2 * q + 1]}, bf16x2));
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) r[e >> 2][e & 3] = __float_as_uint(v[e]);
    }
  }

  template <bool NT = false>
  __device__ __forceinline__ void store(char* p, int64_t n, int lo = 0) const {
    if (n >= N && lo <= 0) {
#pragma unroll
      for (int q = 0; q < R; ++q) store16_any<NT>(p + 16 * q, r[q]);
      return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n && e >= lo) {
        if constexpr (DT == DT_BF16)
          ((uint16_t*)p)[e] = (uint16_t)(r[0][e >> 1] >> ((e & 1) * 16));
        else
          ((uint32_t*)p)[e] = r[e >> 2][e & 3];
      }
  }
};

// A unit: 16 bytes, one access of a lane.
template <int DT>
using Unit = Oct<DT, DT == DT_BF16 ? 8 : 4>;

// The sum over a row of 16 lanes, in each of them, by rotating adds (VALU, no LDS
// permutes): lanes whose values meet add the same two in either order, so all hold the same bits.
template <int N>
__device__ __forceinline__ float row_rotate(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), 0x120 + N, 0xF, 0xF, true));
}
__device__ __forceinline__ float row16_sum(float x) {
  x += row_rotate<8>(x);
  x += row_rotate<4>(x);
  x += row_rotate<2>(x);
  return x + row_rotate<1>(x);
}

// Sums of two values over a team of W waves, in every thread: W = 1 a wave of
// its own, otherwise the whole workgroup through `red` (2 W floats), in a fixed order.
template <int W>
__device__ __forceinline__ void team_sum2(float& a, float& b, float* red) {
  a = xor32_sum(xor16_sum(row16_sum(a)));
  b = xor32_sum(xor16_sum(row16_sum(b)));
  if constexpr (W > 1) {
    const int w = (int)threadIdx.x / WAVE;
    __syncthreads();   // the previous sums have been read
    if (threadIdx.x % WAVE == 0) {
      red[2 * w] = a;
      red[2 * w + 1] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      a += red[2 * i];
      b += red[2 * i + 1];
    }
  }
}

}  // namespace dpg
