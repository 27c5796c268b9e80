// Row layout of the gate kernels (a feature row in the registers of 4 to 64
// lanes), its sums and extremes, and the 8-bit checkpoint of a row.
#pragma once
#include <hip/hip_runtime.h>

namespace chg {

constexpr float kLnEps = 1e-5f;

// logistic sigmoid; the hardware reciprocal (about 1 ulp) instead of an IEEE division
__device__ __forceinline__ float sigm(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, false));
}

// sums of two values over pairs of lanes 32 (16) apart: the lane-half swaps of gfx950
__device__ __forceinline__ float pl_sum32(float a, float b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float pl_sum16(float a, float b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// sum over the LPR lanes of a row, in every lane
template <int LPR>
__device__ __forceinline__ float rowsum(float v) {
  static_assert(LPR == 4 || LPR == 8 || LPR == 16 || LPR == 32 || LPR == 64, "row of 4 to 64 lanes");
  v += dpp<0xB1>(v);  // quad_perm [1,0,3,2]
  v += dpp<0x4E>(v);  // quad_perm [2,3,0,1]
  if (LPR >= 8) v += dpp<0x141>(v);   // row_half_mirror: pairs the two quads of 8 lanes
  if (LPR >= 16) v += dpp<0x140>(v);  // row_mirror: pairs the two halves of 16 lanes
  if (LPR >= 32) v = pl_sum16(v, v);
  if (LPR == 64) v = pl_sum32(v, v);
  return v;
}

// largest and least value over the lanes of a row; a NaN anywhere gives NaN
template <int LPR>
__device__ __forceinline__ float rowmax(float v) {
  v = __builtin_elementwise_maximum(v, dpp<0xB1>(v));
  v = __builtin_elementwise_maximum(v, dpp<0x4E>(v));
  if (LPR >= 8) v = __builtin_elementwise_maximum(v, dpp<0x141>(v));
  if (LPR >= 16) v = __builtin_elementwise_maximum(v, dpp<0x140>(v));
  if (LPR >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if (LPR == 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
template <int LPR>
__device__ __forceinline__ float rowmin(float v) {
  return -rowmax<LPR>(-v);
}

// ---------------------------------------------------------------------------
// 8-bit checkpoint of a half row x (chgnet_ops.h): codes 0 .. 255 in steps of
// (max - min) / 255 above the least value. Steps from the range of each half
// row and not from a wider block or a power of two: the error is at most half
// a step, 1/510 of the range (for normal values of d = 128 about 0.6 % of
// their deviation, rms; e4m3 in blocks of 32 would be off by 2.6 %). Every
// operation is one IEEE rounding, so that the codes are the same bits wherever
// they are formed.
// ---------------------------------------------------------------------------
constexpr float kCodeStep = 1.0f / 255.0f, kLeastStep = 0x1p-100f;

// step and its reciprocal from the extremes. A row of equal values takes the
// least step, whose reciprocal is finite; NaN and infinities stay in `step`.
__device__ __forceinline__ void code_step(float lo, float hi, float& step, float& inv) {
  step = (hi - lo) * kCodeStep;
  step = step < kLeastStep ? kLeastStep : step;
  inv = 1.0f / step;
}
// the code in the low byte: 2^23 has the last place 1, so the sum rounds the
// exact product to even
__device__ __forceinline__ unsigned code_of(float x, float lo, float inv) {
  return __float_as_uint(fmaf(x - lo, inv, 0x1p23f));
}
// the low bytes of four values, the first lowest
__device__ __forceinline__ unsigned pack_codes(unsigned a, unsigned b, unsigned c, unsigned d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u),
                               0x05040100u);
}
// the code in byte k of a word, as a number of steps
template <int K>
__device__ __forceinline__ float code_value(unsigned w) {
  return (float)((w >> (8 * K)) & 0xffu);
}

}  // namespace chg
