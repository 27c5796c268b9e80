// The gate of the gated MLP as an operator (chgnet_ops.h): forward with an
// 8-bit checkpoint of its input, and the backward pass from that checkpoint.
//
//   y_c = g_c xhat_c + b_c, y_g = g_g xhat_g + b_g, xhat = (x - mean) r,
//   r = 1 / sqrt(var + eps);  phi = y_c s(y_c) s(y_g),  s the logistic sigmoid
//   gy_c = dphi s(y_g) s(y_c) (1 + y_c (1 - s(y_c)))
//   gy_g = dphi y_c s(y_c) s(y_g) (1 - s(y_g))
//   dx = r (dy - mean(dy) - xhat mean(dy xhat)),  dy = gy g
//   dg = sum over rows of gy xhat,  db = sum over rows of gy
//
// Both passes read and write each value once: a row of width d costs 14 d + 8
// bytes in each in fp32. A row sits in the registers of LPR lanes, so that its
// mean, variance and range are sums and extremes over lanes (DPP, no LDS); the
// LayerNorm parameters stay in registers while a wavefront walks its rows, and
// the next rows are loaded before the present ones are worked on.
//
// Measured (kernel time, bytes that the pass cannot do without over it): 397,934
// rows of 128 in fp32 forward 103 to 116 us (6.2 to 7.0 TB/s), without the
// checkpoint 104 (5.9), backward 117 to 142 (5.0 to 6.1), where a copy of as much
// reaches 4.7 TB/s; 85,274 rows of 64 14.4 and 17.7 us (5.3 and 4.3). Both are
// bound by memory there, with the vector units busy 56 to 68 % of the time. Rows
// of 16-bit values are as busy on half the bytes, and bound by that, the more so
// without vector loads (20,011 rows of 333 in bf16 20 and 25 us, 2.7 and 2.1 TB/s)
// and where columns of the layout are empty: 8e6 values in bf16 take, forward and
// backward in us a call, 15 and 23 as rows of 256, 20 and 29 of 333, 24 and 44 of
// 130, 31 and 44 of 34, 49 and 63 of 20.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.hpp"
#include "elem.hpp"
#include "rowops.hpp"

namespace chg {
namespace {

// Powers of two that keep the sums over a row of d values in fp32's range wherever
// its mean and variance are: values are summed as x 2^-l and squares as ((x - mean)
// 2^-h)^2, with the least l and h of 2^l >= d and 4^h >= d. (Without them the sum of
// squares passes the range at a variance d times smaller, where the backward pass,
// which sums squares of codes, does not. They take up to 4 % of the forward pass
// in bf16 rows of 128 columns and fewer, whose vector units are the busiest (8e6
// values as rows of 64 15.8 -> 16.4 us, of 20 48.4 -> 49.2), and 0.2 us at most in
// wider ones. A path of its own for such rows took up to 5 of 22 us of all, for
// its registers.) The squares of fp16 values, 65,504 at most, need none.
struct Scale {
  float sum, mean, dev, var, up;  // 2^-l, 2^(l - h) / d, 2^-h, 4^h / d, 2^h
  __device__ __forceinline__ Scale(int d, float inv_d, bool any) {
    const int l = any ? 31 - __builtin_clz(2 * d - 1) : 0, h = (l + 1) / 2;
    auto pow2 = [](int e) { return __int_as_float((127 + e) << 23); };
    sum = pow2(-l);
    mean = inv_d * pow2(l - h);
    dev = pow2(-h);
    var = inv_d * pow2(2 * h);
    up = pow2(h);
  }
};

// Row of d values in LPR lanes: lane j holds the NQ groups of VEC values at
// columns (q LPR + j) VEC. MIN: d is greater, so that only the groups past it
// are looked at for their end; FULL: d is exactly the LPR VEC NQ columns.
// Results are stored past the caches (nontemporal), and with FAR the inputs are
// loaded so: both are of use to others than this kernel only. Measured in fp32
// on both passes of 85,274 rows of 64 and of 397,934 rows of 128: 38.7 and 287 us
// with plain accesses, 32.7 and 274 with such stores, 40.2 and 240 with such
// loads too, which pay where the inputs do not fit the last cache (kFarBytes);
// a kernel that reads the results next takes no longer at any size. FAR is for
// FULL rows: others gain by it only far past that size (forward and backward of
// 320 columns in us, without and with: 55 and 66, 59 and 73 for 25e6 values in
// fp32, 131 and 136, 113 and 136 for 50e6, 97 and 120, 96 and 136 for 50e6 in bf16).
template <int VEC, int LPR, int NQ, int MIN, bool FULL, bool FAR>
struct Cols {
  static constexpr int CPL = VEC * NQ, RPW = 64 / LPR;
  int j, d;
  float inv_d;
  __device__ __forceinline__ int col(int q) const { return (q * LPR + j) * VEC; }
  __device__ __forceinline__ bool has(int q) const { return FULL || (q + 1) * LPR * VEC <= MIN || col(q) < d; }
  template <class T>
  __device__ __forceinline__ void load(const T* p, float (&v)[CPL]) const {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      float t[VEC] = {};
      if (has(q)) {
        if constexpr (FAR) load_nt<VEC>(p + col(q), t);
        else load_v<VEC>(p + col(q), t);
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[q * VEC + k] = t[k];
    }
  }
  template <class T>
  __device__ __forceinline__ void store(T* p, const float (&v)[CPL]) const {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      float t[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) t[k] = v[q * VEC + k];
      if (has(q)) store_nt<VEC>(p + col(q), t);
    }
  }
  // the LayerNorm parameters, which may sit at any float of the parameter vector
  __device__ __forceinline__ void load_any(const float* p, float (&v)[CPL]) const {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[q * VEC + k] = has(q) ? p[col(q) + k] : 0.f;
  }
  // (x - mean) 2^-h in place (0 in columns past d), and 2^h / deviation of x
  __device__ __forceinline__ float center(float (&x)[CPL], const Scale& sc) const {
    float s = x[0] * sc.sum;
#pragma unroll
    for (int k = 1; k < CPL; ++k) s = fmaf(x[k], sc.sum, s);
    const float m = rowsum<LPR>(s) * sc.mean;
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        float& y = x[q * VEC + k];
        y = has(q) ? fmaf(y, sc.dev, -m) : 0.f;
        v += y * y;
      }
    // at least the LayerNorm epsilon: no denormal argument
    return __builtin_amdgcn_rsqf(rowsum<LPR>(v) * sc.var + kLnEps) * sc.up;
  }
  // x - mean in place (0 in columns past d), and 1 / deviation of x * unit, for
  // codes x: what passes fp32's range is the variance alone, in unit^2
  __device__ __forceinline__ float center_codes(float (&x)[CPL], float unit) const {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < CPL; ++k) s += x[k];
    const float m = rowsum<LPR>(s) * inv_d;
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        float& y = x[q * VEC + k];
        y = has(q) ? y - m : 0.f;
        v += y * y;
      }
    return __builtin_amdgcn_rsqf(rowsum<LPR>(v) * inv_d * (unit * unit) + kLnEps);
  }
};

template <class T, int VEC, int LPR, int NQ, int MIN, bool FULL, bool FAR>
__global__ void __launch_bounds__(256) k_gate_act_fwd(int64_t rows, int d, const T* __restrict__ z, int64_t ldz,
                                                      const float* __restrict__ ln, T* __restrict__ phi, int64_t ldphi,
                                                      uint8_t* __restrict__ codes, float2* __restrict__ step) {
  using C = Cols<VEC, LPR, NQ, MIN, FULL, FAR>;
  constexpr int CPL = C::CPL;
  const int lane = threadIdx.x & 63;
  const int width = FULL ? VEC * LPR * NQ : d;
  const C cols{lane % LPR, width, 1.0f / (float)width};
  d = cols.d;
  float gc[CPL], bc[CPL], gg[CPL], bg[CPL];
  cols.load_any(ln, gc);
  cols.load_any(ln + d, bc);
  cols.load_any(ln + 2 * d, gg);
  cols.load_any(ln + 3 * d, bg);
  const Scale sc(d, cols.inv_d, !std::is_same<T, f16_t>::value);
  const int64_t stride = (int64_t)gridDim.x * 4 * C::RPW;
  int64_t row = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * C::RPW + lane / LPR;
  float nc[CPL], ng[CPL];
  if (row < rows) {
    cols.load(z + row * ldz, nc);
    cols.load(z + row * ldz + d, ng);
  }
  for (; row < rows; row += stride) {
    float xc[CPL], xg[CPL];
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
      xc[k] = nc[k];
      xg[k] = ng[k];
    }
    if (row + stride < rows) {
      cols.load(z + (row + stride) * ldz, nc);
      cols.load(z + (row + stride) * ldz + d, ng);
    }
    if (codes) {
      float2 st;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float(&x)[CPL] = h ? xg : xc;
        float lo = HUGE_VALF, hi = -HUGE_VALF, inv;
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float v = x[q * VEC + k];
            lo = __builtin_elementwise_minimum(lo, cols.has(q) ? v : HUGE_VALF);
            hi = __builtin_elementwise_maximum(hi, cols.has(q) ? v : -HUGE_VALF);
          }
        lo = rowmin<LPR>(lo);
        hi = rowmax<LPR>(hi);
        code_step(lo, hi, h ? st.y : st.x, inv);
        uint8_t* c = codes + row * 2 * d + h * d;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          unsigned u[VEC];
#pragma unroll
          for (int k = 0; k < VEC; ++k) u[k] = code_of(x[q * VEC + k], lo, inv);
          if (!cols.has(q)) continue;
          if constexpr (VEC == 4) *reinterpret_cast<unsigned*>(c + cols.col(q)) = pack_codes(u[0], u[1], u[2], u[3]);
          else c[cols.col(q)] = (uint8_t)u[0];
        }
      }
      if (cols.j == 0) step[row] = st;
    }
    const float rc = cols.center(xc, sc), rg = cols.center(xg, sc);
    float o[CPL];
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
      const float yc = gc[k] * (xc[k] * rc) + bc[k], yg = gg[k] * (xg[k] * rg) + bg[k];
      o[k] = yc * sigm(yc) * sigm(yg);
    }
    cols.store(phi + row * ldphi, o);
  }
}

// Threads of a backward block, and the blocks of a launch, which walk the rows:
// each ends in one partial row of the LayerNorm gradients. Two blocks a compute
// unit at 4 columns a lane; wider rows have registers for one (512 against 256
// blocks, forward and backward in us: 85,274 rows of 64 32.1 and 32.5, 397,934 of
// 128 238 and 234, 20,011 of 333 in 16 bits 49 and 45). Blocks of 256 threads,
// twice as many, take 251 us in place of 238.
constexpr int kBwdThreads = 512, kBwdBlocks = 512;

// part: [gridDim.x][4 d] partial sums of the LayerNorm gradients, or with one
// block their destination (`add`: to what it holds).
template <class T, int VEC, int LPR, int NQ, int MIN, bool FULL, bool FAR>
__global__ void __launch_bounds__(kBwdThreads) k_gate_act_bwd(int64_t rows, int d, const uint8_t* __restrict__ codes,
                                                              const float2* __restrict__ step,
                                                              const float* __restrict__ ln, const T* __restrict__ dphi,
                                                              int64_t lddphi, T* __restrict__ dz, int64_t lddz,
                                                              float* __restrict__ part, int add) {
  using C = Cols<VEC, LPR, NQ, MIN, FULL, FAR>;
  constexpr int CPL = C::CPL, W = kBwdThreads / 64;
  __shared__ float red[W][VEC * LPR * NQ];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int width = FULL ? VEC * LPR * NQ : d;
  const C cols{lane % LPR, width, 1.0f / (float)width};
  d = cols.d;
  const float inv_d = cols.inv_d;
  // LayerNorm parameters in registers; at 16 columns a lane with an end to look
  // for, where there is no room for them, in LDS (else 70 registers spill; single
  // values a lane still spill 6 of them)
  constexpr bool kLnInLds = CPL == 16 && !FULL;
  __shared__ float lnS[kLnInLds ? 4 * VEC * LPR * NQ : 1];
  float gc[CPL], bc[CPL], gg[CPL], bg[CPL];
  if constexpr (kLnInLds) {
    for (int t = threadIdx.x; t < 4 * VEC * LPR * NQ; t += kBwdThreads) {
      const int a = t / (VEC * LPR * NQ), c = t % (VEC * LPR * NQ);
      lnS[t] = c < d ? ln[a * d + c] : 0.f;
    }
    __syncthreads();
  } else {
    cols.load_any(ln, gc);
    cols.load_any(ln + d, bc);
    cols.load_any(ln + 2 * d, gg);
    cols.load_any(ln + 3 * d, bg);
  }
  float acc[4][CPL];
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int k = 0; k < CPL; ++k) acc[a][k] = 0.f;
  struct In {
    unsigned wc[NQ], wg[NQ];  // the codes of VEC columns each
    float2 st;
    float up[CPL];
  };
  auto load = [&](int64_t row, In& in) {
    const uint8_t* c = codes + row * 2 * d;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      in.wc[q] = in.wg[q] = 0;
      if (!cols.has(q)) continue;
      if constexpr (VEC == 4) {
        in.wc[q] = *reinterpret_cast<const unsigned*>(c + cols.col(q));
        in.wg[q] = *reinterpret_cast<const unsigned*>(c + d + cols.col(q));
      } else {
        in.wc[q] = c[cols.col(q)];
        in.wg[q] = c[d + cols.col(q)];
      }
    }
    in.st = step[row];
    cols.load(dphi + row * lddphi, in.up);
  };
  const int64_t stride = (int64_t)gridDim.x * W * C::RPW;
  int64_t row = ((int64_t)blockIdx.x * W + wave) * C::RPW + lane / LPR;
  In in;
  if (row < rows) load(row, in);
  for (; row < rows; row += stride) {
    float xc[CPL], xg[CPL], up[CPL];
    const float uc = in.st.x, ug = in.st.y;
    // xhat from the codes themselves: the least value that they count from
    // drops out with the mean, and their sum is exact
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      xc[q * VEC] = code_value<0>(in.wc[q]);
      xg[q * VEC] = code_value<0>(in.wg[q]);
      if constexpr (VEC == 4) {
        xc[4 * q + 1] = code_value<1>(in.wc[q]);
        xc[4 * q + 2] = code_value<2>(in.wc[q]);
        xc[4 * q + 3] = code_value<3>(in.wc[q]);
        xg[4 * q + 1] = code_value<1>(in.wg[q]);
        xg[4 * q + 2] = code_value<2>(in.wg[q]);
        xg[4 * q + 3] = code_value<3>(in.wg[q]);
      }
    }
#pragma unroll
    for (int k = 0; k < CPL; ++k) up[k] = in.up[k];
    if (row + stride < rows) load(row + stride, in);
    if constexpr (kLnInLds) {
      int at = 0;
      asm volatile("" : "+v"(at));  // read for each row: kept from moving out of the loop into registers
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float* p = lnS + at + cols.col(q) + k;
          gc[q * VEC + k] = p[0];
          bc[q * VEC + k] = p[VEC * LPR * NQ];
          gg[q * VEC + k] = p[2 * VEC * LPR * NQ];
          bg[q * VEC + k] = p[3 * VEC * LPR * NQ];
        }
    }
    const float rc = cols.center_codes(xc, uc), rg = cols.center_codes(xg, ug);
    const float fc = uc * rc, fg = ug * rg;
    float s1c = 0.f, s2c = 0.f, s1g = 0.f, s2g = 0.f;
    float dyc[CPL], dyg[CPL];
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
      xc[k] *= fc;
      xg[k] *= fg;
      const float yc = gc[k] * xc[k] + bc[k], yg = gg[k] * xg[k] + bg[k];
      const float sc = sigm(yc), sg = sigm(yg);
      const float silu = yc * sc;
      const float gyc = up[k] * sg * sc * (1.0f + yc * (1.0f - sc)), gyg = up[k] * silu * sg * (1.0f - sg);
      acc[0][k] += gyc * xc[k];
      acc[1][k] += gyc;
      acc[2][k] += gyg * xg[k];
      acc[3][k] += gyg;
      dyc[k] = gyc * gc[k];
      dyg[k] = gyg * gg[k];
      s1c += dyc[k];
      s2c += dyc[k] * xc[k];
      s1g += dyg[k];
      s2g += dyg[k] * xg[k];
    }
    s1c = rowsum<LPR>(s1c) * inv_d;
    s2c = rowsum<LPR>(s2c) * inv_d;
    s1g = rowsum<LPR>(s1g) * inv_d;
    s2g = rowsum<LPR>(s2g) * inv_d;
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
      dyc[k] = rc * (dyc[k] - s1c - xc[k] * s2c);
      dyg[k] = rg * (dyg[k] - s1g - xg[k] * s2g);
    }
    cols.store(dz + row * lddz, dyc);
    cols.store(dz + row * lddz + d, dyg);
  }
  // the block's partial sums: over a wavefront's row slots by lane swaps, then
  // over the wavefronts in order
#pragma unroll
  for (int a = 0; a < 4; ++a) {
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
      float v = acc[a][k];
      if (LPR <= 16) v = pl_sum16(v, v);
      if (LPR <= 32) v = pl_sum32(v, v);
      if (lane < LPR) red[wave][cols.col(k / VEC) + k % VEC] = v;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += kBwdThreads) {
      float s = red[0][c];
#pragma unroll
      for (int w = 1; w < W; ++w) s += red[w][c];
      float* o = part + (int64_t)blockIdx.x * 4 * d + a * d + c;
      *o = add ? *o + s : s;
    }
    __syncthreads();
  }
}

// out[c] (+)= sum over the n partial rows, in 64 bits: 32 columns a block, 32
// groups of threads each sum every 32nd row, and the groups are added in order.
__global__ void __launch_bounds__(1024) k_gate_ln_reduce(const float* __restrict__ part, int n, int count,
                                                         float* __restrict__ out, int add) {
  __shared__ double red[32][33];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
  double s = 0.0;
  if (col < count) {
#pragma unroll 4
    for (int r = g; r < n; r += 32) s += (double)part[(int64_t)r * count + col];
  }
  red[g][c] = s;
  __syncthreads();
  if (g != 0 || col >= count) return;
  for (int k = 1; k < 32; ++k) s += red[k][c];
  out[col] = add ? out[col] + (float)s : (float)s;
}

__global__ void __launch_bounds__(256) k_gate_ln_zero(int n, float* __restrict__ p) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

// Calls f with the narrowest layout that holds rows of width d: four values a lane
// where alignment allows 16-byte (8-byte) accesses, else one. (Groups of four at
// any address, with the row's last one short, took as long as these single values
// or longer: 8e6 values in bf16 forward and backward, groups against singles in us,
// of width 34 36 and 46, 31 and 44; 45 26 and 36, 26 and 36; 130 24 and 44, 24 and
// 44; 333 20 and 29, 20 and 29; 601 20 and 33, 20 and 33; 1,001 22 and 31, 22 and 31.)
template <class F>
int with_layout(int d, bool vec, bool far, F&& f) {
  using std::integral_constant;
#define CHG_ROW(VEC, LPR, NQ, MIN)                                                                 \
  if (d <= VEC * LPR * NQ) {                                                                      \
    const integral_constant<int, VEC> v;                                                          \
    const integral_constant<int, LPR> l;                                                          \
    const integral_constant<int, NQ> n;                                                           \
    const integral_constant<int, MIN> m;                                                          \
    if constexpr (VEC == 4) {                                                                     \
      if (d == VEC * LPR * NQ && far) return f(v, l, n, m, std::true_type{}, std::true_type{});   \
      if (d == VEC * LPR * NQ) return f(v, l, n, m, std::true_type{}, std::false_type{});         \
    }                                                                                             \
    return f(v, l, n, m, std::false_type{}, std::false_type{});                                   \
  }
  if (vec) {
    CHG_ROW(4, 16, 1, 0)
    CHG_ROW(4, 16, 2, 64)
    CHG_ROW(4, 16, 3, 128)
    CHG_ROW(4, 32, 2, 192)
    CHG_ROW(4, 32, 3, 256)
    CHG_ROW(4, 64, 2, 384)
    CHG_ROW(4, 64, 3, 512)
    CHG_ROW(4, 64, 4, 768)
  } else {
    CHG_ROW(1, 16, 1, 0)
    CHG_ROW(1, 16, 4, 16)
    CHG_ROW(1, 32, 4, 64)
    CHG_ROW(1, 32, 8, 128)
    CHG_ROW(1, 32, 12, 256)
    CHG_ROW(1, 64, 8, 384)
    CHG_ROW(1, 64, 12, 512)
    CHG_ROW(1, 64, 16, 768)
  }
#undef CHG_ROW
  return fail(CHGNET_EINVAL, "gate: d must be in 1..1024");
}

int check_gate(const char* who, int64_t rows, int32_t d, int32_t dtype) {
  if (rows < 0) return fail(CHGNET_EINVAL, std::string(who) + ": rows is negative");
  if (d < 1 || d > 1024) return fail(CHGNET_EINVAL, std::string(who) + ": d must be in 1..1024");
  if (!elem_size(dtype)) return fail(CHGNET_EINVAL, std::string(who) + ": unknown dtype");
  return CHGNET_OK;
}

// Blocks of a backward launch over `rows` rows, rpw a wavefront, cpl columns a
// lane. What one block does in two turns needs no second launch to add partial
// rows: 8.0 us a call against 10.7 (64 rows of 64 or 128); in four turns, 7.9 and
// 10.8 us a call, it has the GPU as long as both launches.
int bwd_blocks(int64_t rows, int rpw, int cpl) {
  const int64_t turns = cdiv(rows, rpw * (kBwdThreads / 64));
  return turns <= 2 ? 1 : (int)std::min<int64_t>(cpl <= 4 ? kBwdBlocks : kBwdBlocks / 2, turns);
}

}  // namespace

int gate_forward_entry(int64_t rows, int32_t d, int32_t dtype, const void* z, int64_t ldz, const float* ln, void* phi,
                       int64_t ldphi, uint8_t* codes, float* step, hipStream_t st) {
  CHG_TRY(check_gate("gate_forward", rows, d, dtype));
  if (ldz < 2 * (int64_t)d || ldphi < d) return fail(CHGNET_EINVAL, "gate_forward: a row stride is below the row's width");
  if ((codes == nullptr) != (step == nullptr))
    return fail(CHGNET_EINVAL, "gate_forward: the checkpoint needs both codes and step");
  if (rows == 0) return CHGNET_OK;
  if (!z || !ln || !phi) return fail(CHGNET_EINVAL, "gate_forward: null argument");
  const size_t es = elem_size(dtype);
  if (!aligned_to(z, es) || !aligned_to(phi, es) || !aligned_to(ln, 4) || !aligned_to(step, 8))
    return fail(CHGNET_EINVAL, "gate_forward: an array is not aligned to its values (step: 8 bytes)");
  const bool vec = d % 4 == 0 && ldz % 4 == 0 && ldphi % 4 == 0 && aligned_to(z, 4 * es) && aligned_to(phi, 4 * es) &&
                   aligned_to(codes, 4);
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_layout(d, vec, rows * 2 * d * (int64_t)es >= kFarBytes, [&](auto V, auto L, auto N, auto M, auto full, auto far) -> int {
      constexpr int rpw = 64 / L.value;
      // 8 blocks of 256 threads a compute unit walk the rows
      const unsigned blocks = (unsigned)std::min<int64_t>(2048, cdiv(rows, 4 * rpw));
      KLAUNCH(st, "k_gate_act_fwd",
              k_gate_act_fwd<T, V.value, L.value, N.value, M.value, full.value, far.value><<<blocks, 256, 0, st>>>(
                  rows, d, static_cast<const T*>(z), ldz, ln, static_cast<T*>(phi), ldphi, codes,
                  reinterpret_cast<float2*>(step)));
      return CHGNET_OK;
    });
  });
}

int gate_backward_workspace_entry(int64_t rows, int32_t d, size_t* bytes) {
  CHG_TRY(check_gate("gate_backward_workspace", rows, d, CHGNET_F32));
  if (!bytes) return fail(CHGNET_EINVAL, "gate_backward_workspace: bytes is NULL");
  // whichever layout the call takes: a block has at least 8 rows
  *bytes = sizeof(float) * 4 * (size_t)d * (size_t)std::min<int64_t>(kBwdBlocks, std::max<int64_t>(1, cdiv(rows, 8)));
  return CHGNET_OK;
}

int gate_backward_entry(int64_t rows, int32_t d, int32_t dtype, const uint8_t* codes, const float* step,
                        const float* ln, const void* dphi, int64_t lddphi, void* dz, int64_t lddz, float* dln,
                        int accumulate, void* ws, size_t ws_bytes, hipStream_t st) {
  CHG_TRY(check_gate("gate_backward", rows, d, dtype));
  if (lddz < 2 * (int64_t)d || lddphi < d)
    return fail(CHGNET_EINVAL, "gate_backward: a row stride is below the row's width");
  if (!dln || !aligned_to(dln, 4)) return fail(CHGNET_EINVAL, "gate_backward: dln is NULL or not aligned");
  if (rows == 0) {
    if (!accumulate)
      KLAUNCH(st, "k_gate_ln_zero", k_gate_ln_zero<<<(unsigned)cdiv(4 * d, 256), 256, 0, st>>>(4 * d, dln));
    return CHGNET_OK;
  }
  if (!codes || !step || !ln || !dphi || !dz) return fail(CHGNET_EINVAL, "gate_backward: null argument");
  const size_t es = elem_size(dtype);
  if (!aligned_to(dphi, es) || !aligned_to(dz, es) || !aligned_to(ln, 4) || !aligned_to(step, 8))
    return fail(CHGNET_EINVAL, "gate_backward: an array is not aligned to its values (step: 8 bytes)");
  size_t need = 0;
  CHG_TRY(gate_backward_workspace_entry(rows, d, &need));
  if (!ws || ws_bytes < need) return fail(CHGNET_EWORKSPACE, "gate_backward: workspace too small (query chgnet_gate_backward_workspace)");
  if (!aligned_to(ws, 16)) return fail(CHGNET_EINVAL, "gate_backward: ws is not 16-byte aligned");
  const bool vec = d % 4 == 0 && lddz % 4 == 0 && lddphi % 4 == 0 && aligned_to(dz, 4 * es) &&
                   aligned_to(dphi, 4 * es) && aligned_to(codes, 4);
  float* part = static_cast<float*>(ws);
  int blocks = 1;
  CHG_TRY(with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_layout(d, vec, rows * d * (int64_t)(es + 2) >= kFarBytes, [&](auto V, auto L, auto N, auto M, auto full, auto far) -> int {
      constexpr int rpw = 64 / L.value;
      blocks = bwd_blocks(rows, rpw, V.value * N.value);
      KLAUNCH(st, "k_gate_act_bwd",
              k_gate_act_bwd<T, V.value, L.value, N.value, M.value, full.value, far.value><<<blocks, kBwdThreads, 0, st>>>(
                  rows, d, codes, reinterpret_cast<const float2*>(step), ln, static_cast<const T*>(dphi), lddphi,
                  static_cast<T*>(dz), lddz, blocks == 1 ? dln : part, blocks == 1 && accumulate));
      return CHGNET_OK;
    });
  }));
  if (blocks > 1)
    KLAUNCH(st, "k_gate_ln_reduce",
            k_gate_ln_reduce<<<(unsigned)cdiv(4 * d, 32), 1024, 0, st>>>(part, blocks, 4 * d, dln, accumulate != 0));
  return CHGNET_OK;
}

}  // namespace chg
