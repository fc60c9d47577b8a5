// Reductions over a wave, 64-bit exponentials and loads at any element, for the operators on
// rows of logits.
#pragma once
#include <type_traits>

#include "common.h"

namespace atspeed {

typedef unsigned long long u64;
typedef u32x4_t u32x4_any_t __attribute__((aligned(2)));   // 16 bytes at any element

// Where differences are held at it, nothing is left of the exponential.
constexpr float kLeast = -740.f;
// e^d for N numbers d from -1e9 to 0, to 2.4e-10 of themselves and 1 at 0, side by side: 2^n by
// the exponent, 2^r for r on [-1/2, 1/2] by the polynomial of degree 7 that is 1 at 0 and has
// the least largest relative error (found by exchanging its extrema).
template <int N>
__device__ __forceinline__ void exp_64(double (&d)[N]) {
  constexpr double log2e = 0x1.71547652b82fep0;
  constexpr double c[8] = {1.0, 0x1.62e4300b9dab4p-1, 0x1.ebfbe045705a1p-3, 0x1.c6b0551d56c6dp-5,
                           0x1.3b2a1bf5b7f04p-7, 0x1.5dc05149ba9cap-10, 0x1.443f95e689c5dp-13, 0x1.c04815415f25ep-17};
  double shifted[N], r[N];
#pragma unroll
  for (int i = 0; i < N; ++i) shifted[i] = __builtin_fma(d[i], log2e, 0x1.8p52);   // its low bits: the nearest whole number
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = __builtin_fma(d[i], log2e, 0x1.8p52 - shifted[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) d[i] = c[7];
#pragma unroll
  for (int s = 6; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = __builtin_fma(d[i], r[i], c[s]);
#pragma unroll
  for (int i = 0; i < N; ++i) d[i] = __builtin_ldexp(d[i], (int)(unsigned)__double_as_longlong(shifted[i]));
}
// e^(x - top), x <= top
__device__ __forceinline__ double exp_below(double x, double top) {
  double d[1] = {fmax(x - top, (double)kLeast)};
  exp_64(d);
  return d[0];
}

// Largest of two, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A word of the lane that step s of a reduction over the wave pairs this one with: lanes 1,
// 2, then mirrored within 8 and 16 (whose parts are alike by then), 16 and 32 apart.
template <int S>
__device__ __forceinline__ uint32_t partner(uint32_t x) {
  if (S == 0) return __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true);         // quad_perm 1 0 3 2
  if (S == 1) return __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true);         // quad_perm 2 3 0 1
  if (S == 2) return __builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true);        // row_half_mirror
  if (S == 3) return __builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true);        // row_mirror
  return __shfl_xor(x, S == 4 ? 16 : 32);
}
template <int S>
__device__ __forceinline__ double partner(double x) {
  const u64 u = (u64)__double_as_longlong(x);
  return __longlong_as_double((long long)((u64)partner<S>((uint32_t)(u >> 32)) << 32 | partner<S>((uint32_t)u)));
}
__device__ __forceinline__ float wave_max_nan(float x) {
  static_for<6>([&](auto s) { x = max_nan(x, __uint_as_float(partner<s>(__float_as_uint(x)))); });
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
template <int S>
__device__ __forceinline__ float partner(float x) { return __uint_as_float(partner<S>(__float_as_uint(x))); }
template <class F>
__device__ __forceinline__ F wave_sum(F x) {
  static_for<6>([&](auto s) { x += partner<s>(x); });
  return x;
}

// Lane i: the sum of lanes 0 .. i.
template <class N>
__device__ __forceinline__ N wave_scan(N x) {
  const auto from = [&](auto ctrl, auto rows) {
    return __builtin_bit_cast(N, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl.value, rows.value, 0xf, false));
  };
  typedef std::integral_constant<int, 0xf> All;
  x += from(std::integral_constant<int, 0x111>{}, All{});   // row_shr: 1, 2, 4, 8 lanes of a row of 16
  x += from(std::integral_constant<int, 0x112>{}, All{});
  x += from(std::integral_constant<int, 0x114>{}, All{});
  x += from(std::integral_constant<int, 0x118>{}, All{});
  x += from(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast: 15 to the next row
  x += from(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // 31 to the rows behind
  return x;
}

}  // namespace atspeed
