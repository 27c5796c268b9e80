// Dropout as an operator (chgnet_ops.h): out = x / (1 - p) where the generator
// keeps a value, else 0. No mask is stored: the same call on the upstream
// gradient is the backward pass.
//
// A thread has the eight columns of one generator's result, in 16-byte accesses at
// any value's address. Bound by memory: 16,384 x 8,192 in bf16 105 us (5.1 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.hpp"
#include "elem.hpp"
#include "philox.hpp"

namespace chg {
namespace {

template <class T>
__global__ void __launch_bounds__(256) k_dropout(int64_t rows, int d, const T* __restrict__ x, int64_t ldx, Drop drop,
                                                 T* __restrict__ out, int64_t ldout) {
  constexpr int W = 16 / sizeof(T);
  const int groups = (d + 7) / 8;
  const Philox rng(drop);
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, stride = (int64_t)gridDim.x * 256;
  int64_t row = first / groups;
  int g = (int)(first % groups);
  const int64_t step_rows = stride / groups;
  const int step_g = (int)(stride % groups);
  while (row < rows) {
    const uint32_t m = rng.mask8((uint32_t)row, (uint32_t)g, drop.cut);
    const T* p = x + row * ldx + 8 * (int64_t)g;
    T* o = out + row * ldout + 8 * (int64_t)g;
    const int n = d - 8 * g;
    if (n >= 8) {
      typedef T vec __attribute__((ext_vector_type(W)));
      typedef vec any __attribute__((aligned(sizeof(T))));
#pragma unroll
      for (int q = 0; q < 8 / W; ++q) {
        vec t = *reinterpret_cast<const any*>(p + q * W);
#pragma unroll
        for (int k = 0; k < W; ++k) t[k] = m >> (q * W + k) & 1 ? (T)((float)t[k] * drop.scale) : (T)0.f;
        *reinterpret_cast<any*>(o + q * W) = t;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (k < n) o[k] = m >> k & 1 ? (T)((float)p[k] * drop.scale) : (T)0.f;
    }
    row += step_rows;
    g += step_g;
    if (g >= groups) {
      g -= groups;
      ++row;
    }
  }
}

}  // namespace

int dropout_entry(int64_t rows, int32_t d, int32_t dtype, const void* x, int64_t ldx, float p, uint64_t seed,
                  uint64_t call, const int64_t* step, void* out, int64_t ldout, hipStream_t st) {
  if (rows < 0 || rows >= (int64_t(1) << 32)) return fail(CHGNET_EINVAL, "dropout: rows must be in 0 .. 2^32 - 1");
  if (d < 1 || d > (1 << 30)) return fail(CHGNET_EINVAL, "dropout: d must be in 1 .. 2^30");
  if (!elem_size(dtype)) return fail(CHGNET_EINVAL, "dropout: unknown dtype");
  if (!(p >= 0.0f && p <= 1.0f)) return fail(CHGNET_EINVAL, "dropout: p must be in 0 .. 1");
  if (ldx < d || ldout < d) return fail(CHGNET_EINVAL, "dropout: a row stride is below the row's width");
  if (!aligned_to(step, 8)) return fail(CHGNET_EINVAL, "dropout: step is not aligned");
  if (rows == 0) return CHGNET_OK;
  if (!x || !out) return fail(CHGNET_EINVAL, "dropout: null argument");
  const size_t es = elem_size(dtype);
  if (!aligned_to(x, es) || !aligned_to(out, es)) return fail(CHGNET_EINVAL, "dropout: an array is not aligned to its values");
  const Drop drop = make_drop(p, seed, call, step);
  const unsigned blocks = (unsigned)std::min<int64_t>(2048, cdiv(rows * cdiv(d, 8), 256));
  return with_type(dtype, [&](auto t) -> int {
    using T = decltype(t);
    KLAUNCH(st, "k_dropout", k_dropout<T><<<blocks, 256, 0, st>>>(rows, d, static_cast<const T*>(x), ldx, drop,
                                                                  static_cast<T*>(out), ldout));
    return CHGNET_OK;
  });
}

}  // namespace chg
