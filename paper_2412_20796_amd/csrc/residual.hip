// The norms before and after a block with its gate, dropout and residual scale
// (chgnet_ops.h), forward and backward, and a norm alone.
//
//   t = w_p n(f) + b_p,  v = Drop(s(g) t),  y = alpha x + beta v,  h = w n(y) + b
//   n(x) = x r (RMS) or (x - mean) r (LayerNorm), r = 1 / sqrt(mean of squares + eps)
//   D  = dy + r (dn - [mean dn] - n mean(dn n)),  dn = w dh      (n, r of y)
//   dx = alpha D,  du = beta mask D,  dg = du t s(1 - s),  dt = du s
//   df = r_p (dm - [mean dm] - n_p mean(dm n_p)),  dm = w_p dt   (n_p, r_p of f)
//   dw = sum of dh n, db = sum of dh, dw_p = sum of dt n_p, db_p = sum of dt
//
// Nothing but y is kept for the backward pass: it has to read y and f anyway, and
// forms their sums again in registers. A row sits in the registers of 8 to 1,024
// threads; sums go over lanes by DPP and over wavefronts through LDS, and what
// must be summed before the same barrier goes over it together (two barriers a
// row for RMS norms on both sides, three for LayerNorms).
//
// Bound by memory. Measured (kernel time, bytes that a pass cannot do without over
// it; a copy reaches 4.7 TB/s): 16,384 rows of 8,192 in bf16 with RMS norms, gate and
// dropout forward 275 us (4.9 TB/s), backward 446 (4.8); 397,934 rows of 128 in fp32
// 201 and 327 us (5.1, 5.0), a LayerNorm alone 66 and 125; 65,536 rows of 512 in bf16 66
// and 140 us (5.1, 3.8), where the backward pass has two wavefronts a SIMD for its
// 170 registers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "elem.hpp"
#include "philox.hpp"
#include "rowops.hpp"

namespace chg {
namespace {

constexpr int kNoNorm = CHGNET_NORM_NONE, kRms = CHGNET_NORM_RMS, kLayer = CHGNET_NORM_LAYER;

// Powers of two that keep the sums over a row of d values in fp32's range
// wherever its mean and mean square are: values are summed as x 2^-l, squares
// as (x 2^-h)^2, with the least l and h of 2^l >= d and 4^h >= d.
struct Scale {
  float sum, mean, dev, var, up;  // 2^-l, 2^l / d, 2^-h, 4^h / d, 2^h
  __device__ __forceinline__ explicit Scale(int d) {
    const int l = d > 1 ? 32 - __builtin_clz(d - 1) : 0, h = (l + 1) / 2;
    auto pow2 = [](int e) { return __int_as_float((127 + e) << 23); };
    const float inv = 1.0f / (float)d;
    sum = pow2(-l);
    mean = inv * pow2(l);
    dev = pow2(-h);
    var = inv * pow2(2 * h);
    up = pow2(h);
  }
};

// Row of d values in TPR threads: thread j holds the NQ groups of VEC values (16
// bytes) at columns (q TPR + j) VEC. ANY: rows at any value's address, and a last
// group that is short; the hardware takes 16 bytes at any address. A short group is
// loaded whole where the array goes on behind it (the next row's values), and what
// is past the row is cleared; it is stored in 8, 4 and 2 bytes. (40,000 rows of 1,001 in
// bf16 with all parts take 96 and 268 us forward and backward; in single values 265 and
// 475, with short groups value by value 131 and 310.)
template <int VEC, int TPR, int NQ, bool ANY>
struct Row {
  static constexpr int CPL = VEC * NQ, WAVES = TPR > 64 ? TPR / 64 : 1;
  static constexpr int WHOLE = NQ / 2;  // groups that are never short: the next narrower layout holds them
  int j, d;
  uint32_t mask[ANY ? NQ - WHOLE : 1][4];
  __device__ __forceinline__ Row(int thread, int width) : j(thread), d(width) {
    if constexpr (ANY) {
#pragma unroll
      for (int q = WHOLE; q < NQ; ++q)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if constexpr (VEC == 8) mask[q - WHOLE][k] = (has(q, 2 * k) ? 0xffffu : 0u) | (has(q, 2 * k + 1) ? 0xffff0000u : 0u);
          else mask[q - WHOLE][k] = has(q, k) ? ~0u : 0u;
        }
    }
  }
  __device__ __forceinline__ int col(int q) const { return (q * TPR + j) * VEC; }
  __device__ __forceinline__ bool has(int q, int k) const { return col(q) + (ANY ? k : 0) < d; }
  // rows as they are stored, which may be loaded ahead
  typedef uint32_t words __attribute__((ext_vector_type(4)));
  template <class T>
  struct Raw {
    words q[NQ];
  };
  // `behind`: rows of the array after this one
  template <class T>
  __device__ __forceinline__ void load(const T* p, int64_t behind, int64_t ld, Raw<T>& r) const {
    typedef words any __attribute__((aligned(2)));
    typedef typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type bits;
    const bool goes_on = behind * ld >= VEC - 1;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int c = col(q);
      r.q[q] = words{};
      if constexpr (ANY) {
        if (c + VEC <= d || (goes_on && c < d)) {
          r.q[q] = *reinterpret_cast<const any*>(p + c);
        } else {
#pragma unroll
          for (int k = 0; k < VEC - 1; ++k)
            if (c + k < d)
              r.q[q][k * 4 / VEC] |= (uint32_t)reinterpret_cast<const bits*>(p)[c + k] << (VEC == 8 && k % 2 ? 16 : 0);
        }
        if (q >= WHOLE) {
#pragma unroll
          for (int k = 0; k < 4; ++k) r.q[q][k] &= mask[q - WHOLE < 0 ? 0 : q - WHOLE][k];
        }
      } else if (c < d) {
        r.q[q] = *reinterpret_cast<const words*>(p + c);
      }
    }
  }
  template <class T>
  __device__ __forceinline__ void values(const Raw<T>& r, float (&v)[CPL]) const {
    typedef T vec __attribute__((ext_vector_type(VEC)));
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const vec t = __builtin_bit_cast(vec, r.q[q]);
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[q * VEC + k] = (float)t[k];
    }
  }
  template <class T>
  __device__ __forceinline__ void load(const T* p, int64_t behind, int64_t ld, float (&v)[CPL]) const {
    Raw<T> r;
    load(p, behind, ld, r);
    values(r, v);
  }
  template <class T>
  __device__ __forceinline__ void store(T* p, const float (&v)[CPL]) const {
    typedef T vec __attribute__((ext_vector_type(VEC)));
    typedef words any __attribute__((aligned(2)));
    typedef uint32_t two __attribute__((ext_vector_type(2)));
    typedef two any2 __attribute__((aligned(2)));
    typedef uint32_t any1 __attribute__((aligned(2)));
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int c = col(q);
      vec t;
#pragma unroll
      for (int k = 0; k < VEC; ++k) t[k] = (T)v[q * VEC + k];
      const words w = __builtin_bit_cast(words, t);
      if constexpr (ANY) {
        if (c + VEC <= d) {
          *reinterpret_cast<any*>(p + c) = w;
        } else if (c < d) {
          const int n = d % VEC;  // values of the short group; `at`: words that are stored
          const int half = VEC / 2;
          int at = 0;
          if (n >= half) {
            *reinterpret_cast<any2*>(p + c) = two{w[0], w[1]};
            at = 2;
          }
          if constexpr (VEC == 8) {
            if (n & 2) {
              *reinterpret_cast<any1*>(p + c + 2 * at) = at ? w[2] : w[0];
              ++at;
            }
            if (n & 1) {
              const uint32_t last = at == 0 ? w[0] : at == 1 ? w[1] : at == 2 ? w[2] : w[3];
              *reinterpret_cast<uint16_t*>(p + c + 2 * at) = (uint16_t)last;
            }
          } else if (n & 1) {
            *reinterpret_cast<uint32_t*>(p + c + at) = at ? w[2] : w[0];
          }
        }
      } else if (c < d) {
        *reinterpret_cast<words*>(p + c) = w;
      }
    }
  }
  // parameters, which may sit at any float; `other` where there are none
  __device__ __forceinline__ void load_any(const float* p, float (&v)[CPL], float other) const {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[q * VEC + k] = !has(q, k) ? 0.f : p ? p[col(q) + k] : other;
  }
  // sums over the row of N values a thread, in every thread. The two buffers of
  // wide rows take turns: whoever writes to one has passed the barrier of the
  // other, which all reach after they have read this one.
  template <int N>
  __device__ __forceinline__ void sums(float (&v)[N], float (*red)[4][16], int& turn) const {
    if constexpr (WAVES == 1) {
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = rowsum<(TPR > 64 ? 64 : TPR)>(v[n]);
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        v[n] = rowsum<64>(v[n]);
        if ((threadIdx.x & 63) == 0) red[turn][n][(threadIdx.x >> 6) % WAVES] = v[n];
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < N; ++n) {
        v[n] = red[turn][n][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v[n] += red[turn][n][w];
      }
      turn ^= 1;
    }
  }
  __device__ __forceinline__ float part_sum(const float (&x)[CPL], const Scale& sc) const {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < CPL; ++k) s = fmaf(x[k], sc.sum, s);
    return s;
  }
  // x 2^-h, less the mean for a LayerNorm (0 in columns past d)
  __device__ __forceinline__ void center(float (&x)[CPL], bool layer, float mean, const Scale& sc) const {
    if (!layer) {
#pragma unroll
      for (int k = 0; k < CPL; ++k) x[k] *= sc.dev;
      return;
    }
    const float m = mean * sc.dev;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        float& y = x[q * VEC + k];
        y = has(q, k) ? fmaf(y, sc.dev, -m) : 0.f;
      }
  }
  __device__ __forceinline__ float part_dot(const float (&a)[CPL], const float (&b)[CPL]) const {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < CPL; ++k) s = fmaf(a[k], b[k], s);
    return s;
  }
  // Which of the thread's values a dropout keeps: the generator's words of groups of
  // 8 columns (of 4: the half of them), compared where they are used.
  struct Keep {
    uint32_t w[CPL / 2], cut;
    __device__ __forceinline__ bool operator()(int k) const {
      return k & 1 ? Philox::upper(w[k / 2], cut) : Philox::lower(w[k / 2], cut);
    }
  };
  __device__ __forceinline__ void kept(const Philox& rng, int64_t row, uint32_t cut, Keep& keep) const {
    keep.cut = cut;
    if (!cut) {
#pragma unroll
      for (int k = 0; k < CPL / 2; ++k) keep.w[k] = 0;
      return;
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      uint32_t w[4];
      rng.words((uint32_t)row, (uint32_t)col(q) >> 3, w);
      if constexpr (VEC == 8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) keep.w[4 * q + k] = w[k];
      } else {
        const bool second = col(q) & 4;
        keep.w[2 * q] = second ? w[2] : w[0];
        keep.w[2 * q + 1] = second ? w[3] : w[1];
      }
    }
  }
};

// 2^h / deviation of a row whose (x 2^-h)^2 sum to v; 0 where its variance
// passes fp32's range
__device__ __forceinline__ float deviation(float v, float eps, const Scale& sc) {
  return __builtin_amdgcn_rsqf(fmaf(v, sc.var, eps)) * sc.up;
}

struct ResArgs {
  int64_t rows;
  int d;
  const void *x, *f, *g, *dy, *dh;  // backward: x is y
  int64_t ldx, ldf, ldg, lddy, lddh;
  int gate;  // 0 none, 1 one value a row, 2 one a column
  const float *post, *pre;
  int post_kind, post_rows, pre_kind, pre_rows;
  float alpha, beta, eps;
  Drop drop;
  void *o0, *o1, *o2;  // y, h; dx, df, dg
  int64_t ld0, ld1, ld2;
  float *dpost, *dpre;  // a single block's destinations
  float* part;          // [blocks][post_rows + pre_rows][d]
  int add;
};

// s(x) and its derivative s (1 - s), each to some last places of its own: with
// e = exp(-|x|), s and 1 - s are 1 / (1 + e) and e times that. 1 - s formed from s is off
// by half a last place of 1, which is all of it for x = 17.
struct Sigmoid {
  float s, slope;
  __device__ __forceinline__ explicit Sigmoid(float x) {
    const float e = __expf(-fabsf(x)), large = __builtin_amdgcn_rcpf(1.0f + e), small = e * large;
    s = x < 0.f ? small : large;
    slope = small * large;
  }
};

template <class T>
__device__ __forceinline__ float stored(float v) {
  return (float)(T)v;
}

// Threads of a forward block: a row of more than a wavefront has one to itself,
// whose barriers are its sums'
template <int TPR>
constexpr int fwd_threads() {
  return TPR > 64 ? TPR : 256;
}
// RES false: a norm alone, h = w n(x) + b
template <class T, int VEC, int TPR, int NQ, bool ANY, bool RES>
__global__ void __launch_bounds__(fwd_threads<TPR>()) k_residual_fwd(ResArgs a) {
  using R = Row<VEC, TPR, NQ, ANY>;
  constexpr int CPL = R::CPL;
  constexpr int ROWS = fwd_threads<TPR>() / TPR;  // of a block
  __shared__ float red[2][4][16];
  const R row((int)threadIdx.x % TPR, a.d);
  const Scale sc(a.d);
  int turn = 0;
  float wp[CPL], bp[CPL], w[CPL], b[CPL];
  if constexpr (RES) {
    row.load_any(a.post, wp, 1.f);
    row.load_any(a.post_rows == 2 ? a.post + a.d : nullptr, bp, 0.f);
  }
  row.load_any(a.pre, w, 1.f);
  row.load_any(a.pre_rows == 2 ? a.pre + a.d : nullptr, b, 0.f);
  const Philox rng(a.drop);
  for (int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; r < a.rows; r += (int64_t)gridDim.x * ROWS) {
    float y[CPL];
    const int64_t behind = a.rows - 1 - r;
    row.load(static_cast<const T*>(a.x) + r * a.ldx, behind, a.ldx, y);
    if constexpr (RES) {
      float t[CPL];
      row.load(static_cast<const T*>(a.f) + r * a.ldf, behind, a.ldf, t);
      float g[CPL] = {};
      if (a.gate == 2) row.load(static_cast<const T*>(a.g) + r * a.ldg, behind, a.ldg, g);
      const float g1 = a.gate == 1 ? (float)static_cast<const T*>(a.g)[r * a.ldg] : 0.f;
      float dev = 1.f;
      if (a.post_kind != kNoNorm) {
        float s[1] = {0.f};
        if (a.post_kind == kLayer) {
          s[0] = row.part_sum(t, sc);
          row.sums(s, red, turn);
        }
        row.center(t, a.post_kind == kLayer, s[0] * sc.mean, sc);
        s[0] = row.part_dot(t, t);
        row.sums(s, red, turn);
        dev = deviation(s[0], a.eps, sc);
      }
      const float s1 = a.gate == 1 ? sigm(g1) : 1.f;
      typename R::Keep keep;
      row.kept(rng, r, a.drop.cut, keep);
      const float beta = a.beta * a.drop.scale;
#pragma unroll
      for (int k = 0; k < CPL; ++k) {
        const float u = fmaf(wp[k], t[k] * dev, bp[k]) * (a.gate == 2 ? sigm(g[k]) : s1);
        y[k] = fmaf(a.alpha, y[k], keep(k) ? beta * u : 0.f);
        y[k] = stored<T>(y[k]);
      }
      row.store(static_cast<T*>(a.o0) + r * a.ld0, y);
    }
    if (a.pre) {
      float s[1] = {0.f};
      if (a.pre_kind == kLayer) {
        s[0] = row.part_sum(y, sc);
        row.sums(s, red, turn);
      }
      row.center(y, a.pre_kind == kLayer, s[0] * sc.mean, sc);
      s[0] = row.part_dot(y, y);
      row.sums(s, red, turn);
      const float dev = deviation(s[0], a.eps, sc);
#pragma unroll
      for (int k = 0; k < CPL; ++k) y[k] = fmaf(w[k], y[k] * dev, b[k]);
      row.store(static_cast<T*>(a.o1) + r * a.ld1, y);
    }
  }
}

// Threads of a backward block
template <int TPR>
constexpr int bwd_threads() {
  return TPR > 512 ? TPR : 512;
}
// Blocks of a backward launch, which each end in one partial row of the parameters'
// gradients: as many as run at a time, two a compute unit where registers and
// threads allow it
constexpr int kBwdBlocks = 512;
template <class T, int TPR, int NQ, bool RES>
constexpr int bwd_blocks_at_most() {
  return TPR == 1024 || (RES && (sizeof(T) == 2 || NQ > 1)) ? kBwdBlocks / 2 : kBwdBlocks;
}

// Adds the block's sums of one parameter row into `o` (its row of the partial
// sums, or with one block the destination itself): rows of one wavefront by lane
// swaps, rows of several through LDS, in order.
template <int VEC, int TPR, int NQ, bool ANY>
__device__ __forceinline__ void join(const Row<VEC, TPR, NQ, ANY>& row, const float (&acc)[VEC * NQ], float* red, float* o,
                                     bool add) {
  constexpr int W = VEC * TPR * NQ, G = bwd_threads<TPR>() / (TPR > 64 ? TPR : 64);
  const int g = threadIdx.x / (TPR > 64 ? TPR : 64);
  auto put = [&](int c, float s) { o[c] = add ? o[c] + s : s; };
#pragma unroll
  for (int k = 0; k < VEC * NQ; ++k) {
    float v = acc[k];
    const int c = row.col(k / VEC) + k % VEC;
    if (TPR <= 8) v += dpp<0x140>(dpp<0x141>(v));  // lanes 8 apart: mirrored in 16, then in 8
    if (TPR <= 16) v = pl_sum16(v, v);
    if (TPR <= 32) v = pl_sum32(v, v);
    if constexpr (G == 1) {
      if (c < row.d) put(c, v);
    } else {
      if (TPR > 64 || (threadIdx.x & 63) < TPR) red[g * W + c] = v;
    }
  }
  if constexpr (G > 1) {
    __syncthreads();
    for (int c = threadIdx.x; c < row.d; c += bwd_threads<TPR>()) {
      float s = red[c];
#pragma unroll
      for (int w = 1; w < G; ++w) s += red[w * W + c];
      put(c, s);
    }
    __syncthreads();
  }
}

// The next row is loaded before the present one is worked on where a thread has
// registers for it (one group of a row); with 1,024 threads a row, which have 128
// registers each, the norms' parameters make room for it in LDS.
template <class T, int VEC, int TPR, int NQ, bool ANY, bool RES>
__global__ void __launch_bounds__(bwd_threads<TPR>()) k_residual_bwd(ResArgs a) {
  using R = Row<VEC, TPR, NQ, ANY>;
  constexpr int CPL = R::CPL, ROWS = bwd_threads<TPR>() / TPR, G = bwd_threads<TPR>() / (TPR > 64 ? TPR : 64);
  constexpr bool PARAMS_IN_LDS = RES && TPR == 1024 && CPL <= 8, AHEAD = NQ == 1;
  // several rows of more than a wavefront in a block would not meet at the
  // barriers of their sums: each has its own buffers, and all walk as many rows
  __shared__ float red_all[TPR > 64 ? ROWS : 1][2][4][16];
  __shared__ float join_s[G > 1 ? G * VEC * TPR * NQ : 1];
  __shared__ float params[PARAMS_IN_LDS ? 3 : 1][PARAMS_IN_LDS ? VEC * TPR * NQ : 1];
  float(*red)[4][16] = red_all[TPR > 64 ? threadIdx.x / TPR : 0];
  const R row((int)threadIdx.x % TPR, a.d);
  const Scale sc(a.d);
  const float inv_d = 1.0f / (float)a.d;
  int turn = 0;
  float wp[CPL], bp[CPL], w[CPL];
  if constexpr (RES) {
    row.load_any(a.post, wp, 1.f);
    row.load_any(a.post_rows == 2 ? a.post + a.d : nullptr, bp, 0.f);
  }
  row.load_any(a.pre, w, 1.f);
  if constexpr (PARAMS_IN_LDS) {  // (each thread reads what it wrote itself)
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
      params[0][threadIdx.x * CPL + k] = wp[k];
      params[1][threadIdx.x * CPL + k] = bp[k];
      params[2][threadIdx.x * CPL + k] = w[k];
    }
  }
  int lds_at = threadIdx.x * CPL;
  auto param = [&](int which, float (&v)[CPL]) {
    if constexpr (PARAMS_IN_LDS) {
      asm volatile("" : "+v"(lds_at));  // read for each row: kept from moving out of the loop into registers
#pragma unroll
      for (int k = 0; k < CPL; ++k) v[k] = params[which][lds_at + k];
    }
  };
  float awp[CPL] = {}, abp[CPL] = {}, aw[CPL] = {}, ab[CPL] = {};
  const Philox rng(a.drop);
  const int64_t stride = (int64_t)gridDim.x * ROWS;
  struct In {
    typename R::template Raw<T> dy, y, dh, f, g;
    float g1;
  } in;
  auto load = [&](int64_t at) {
    if (a.dy) row.load(static_cast<const T*>(a.dy) + at * a.lddy, a.rows - 1 - at, a.lddy, in.dy);
    if (a.pre) {
      row.load(static_cast<const T*>(a.x) + at * a.ldx, a.rows - 1 - at, a.ldx, in.y);
      row.load(static_cast<const T*>(a.dh) + at * a.lddh, a.rows - 1 - at, a.lddh, in.dh);
    }
    if constexpr (RES) {
      if (a.f) row.load(static_cast<const T*>(a.f) + at * a.ldf, a.rows - 1 - at, a.ldf, in.f);
      if (a.gate == 2) row.load(static_cast<const T*>(a.g) + at * a.ldg, a.rows - 1 - at, a.ldg, in.g);
      if (a.gate == 1) in.g1 = (float)static_cast<const T*>(a.g)[at * a.ldg];
    }
  };
  auto row_of = [&](int64_t first) {  // or the last row again, whose results go nowhere
    const int64_t r = first + threadIdx.x / TPR;
    return r < a.rows ? r : a.rows - 1;
  };
  if (AHEAD && (int64_t)blockIdx.x * ROWS < a.rows) load(row_of((int64_t)blockIdx.x * ROWS));
  for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += stride) {
    const int64_t r = first + threadIdx.x / TPR, at = row_of(first);
    const bool live = r < a.rows;
    float D[CPL] = {}, y[CPL] = {}, dh[CPL] = {}, f[CPL] = {}, g[CPL] = {};
    float g1 = 0.f;
    if constexpr (AHEAD) {
      if (a.dy) row.values(in.dy, D);
      if (a.pre) {
        row.values(in.y, y);
        row.values(in.dh, dh);
      }
      if constexpr (RES) {
        if (a.f) row.values(in.f, f);
        if (a.gate == 2) row.values(in.g, g);
        if (a.gate == 1) g1 = in.g1;
      }
    } else {
      if (a.dy) row.load(static_cast<const T*>(a.dy) + at * a.lddy, a.rows - 1 - at, a.lddy, D);
      if (a.pre) {
        row.load(static_cast<const T*>(a.x) + at * a.ldx, a.rows - 1 - at, a.ldx, y);
        row.load(static_cast<const T*>(a.dh) + at * a.lddh, a.rows - 1 - at, a.lddh, dh);
      }
      if constexpr (RES) {
        if (a.f) row.load(static_cast<const T*>(a.f) + at * a.ldf, a.rows - 1 - at, a.ldf, f);
        if (a.gate == 2) row.load(static_cast<const T*>(a.g) + at * a.ldg, a.rows - 1 - at, a.ldg, g);
        if (a.gate == 1) g1 = (float)static_cast<const T*>(a.g)[at * a.ldg];
      }
    }
    if (AHEAD && first + stride < a.rows) load(row_of(first + stride));
    const bool norm_f = RES && a.post_kind != kNoNorm, pre_layer = a.pre && a.pre_kind == kLayer,
               post_layer = norm_f && a.post_kind == kLayer;
    param(2, w);
    float mean[3] = {0.f, 0.f, 0.f};  // of y, f and w dh
    if (pre_layer || post_layer) {
      if (pre_layer) {
        mean[0] = row.part_sum(y, sc);
        mean[2] = row.part_dot(w, dh);
      }
      if (post_layer) mean[1] = row.part_sum(f, sc);
      row.sums(mean, red, turn);
      mean[0] *= sc.mean;
      mean[1] *= sc.mean;
      mean[2] *= inv_d;
    }
    float dev_f = 1.f;
    {
      float q[3] = {0.f, 0.f, 0.f};  // squares of y and f, product of y and w dh
      if (a.pre) {
        row.center(y, pre_layer, mean[0], sc);
        q[0] = row.part_dot(y, y);
#pragma unroll
        for (int k = 0; k < CPL; ++k) q[2] = fmaf(w[k] * dh[k], y[k], q[2]);
      }
      if (norm_f) {
        row.center(f, post_layer, mean[1], sc);
        q[1] = row.part_dot(f, f);
      }
      if (a.pre || norm_f) row.sums(q, red, turn);
      if (norm_f) dev_f = deviation(q[1], a.eps, sc);
      if (a.pre) {
        const float dev = deviation(q[0], a.eps, sc), r1 = dev * sc.dev;
        const float c = dev > 0.f ? dev * q[2] * inv_d : 0.f;
        if (live && a.pre_rows == 2) {
#pragma unroll
          for (int k = 0; k < CPL; ++k) ab[k] += dh[k];
        }
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
          const float n = y[k] * dev;
          if (live) aw[k] = fmaf(dh[k], n, aw[k]);
          D[k] = fmaf(r1, fmaf(-n, c, fmaf(w[k], dh[k], -mean[2])), D[k]);
        }
      }
    }
    if constexpr (!RES) {
      if (live) row.store(static_cast<T*>(a.o0) + r * a.ld0, D);
    } else {
      typename R::Keep keep;
      row.kept(rng, at, a.drop.cut, keep);
      const float beta = a.beta * a.drop.scale;
      param(0, wp);
      param(1, bp);
      float q[3] = {0.f, 0.f, 0.f};  // of dm, dm n_p, and the one gate's gradient
      if (a.post) {
#pragma unroll
        for (int k = 0; k < CPL; ++k) f[k] *= dev_f;
      }
      // y: the gradient of t
      if (a.gate) {
        const Sigmoid one(g1);
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
          const Sigmoid sg = a.gate == 2 ? Sigmoid(g[k]) : one;
          const float du = beta * D[k];
          g[k] = keep(k) ? du * sg.slope * fmaf(wp[k], f[k], bp[k]) : 0.f;
          y[k] = keep(k) ? du * sg.s : 0.f;
        }
        if (a.gate == 2 && live) row.store(static_cast<T*>(a.o2) + r * a.ld2, g);
        if (a.gate == 1) {
#pragma unroll
          for (int k = 0; k < CPL; ++k) q[2] += row.has(k / VEC, k % VEC) ? g[k] : 0.f;
        }
      } else {
#pragma unroll
        for (int k = 0; k < CPL; ++k) y[k] = keep(k) ? beta * D[k] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < CPL; ++k) D[k] *= a.alpha;
      if (live) row.store(static_cast<T*>(a.o0) + r * a.ld0, D);
      if (a.post) {
        if (!norm_f) {  // what is dropped of f may be anything
#pragma unroll
          for (int k = 0; k < CPL; ++k) f[k] = keep(k) ? f[k] : 0.f;
        }
        if (live) {
#pragma unroll
          for (int k = 0; k < CPL; ++k) awp[k] = fmaf(y[k], f[k], awp[k]);
          if (a.post_rows == 2) {
#pragma unroll
            for (int k = 0; k < CPL; ++k) abp[k] += y[k];
          }
        }
#pragma unroll
        for (int k = 0; k < CPL; ++k) y[k] *= wp[k];
      }
      if (norm_f) {
        if (post_layer)
#pragma unroll
          for (int k = 0; k < CPL; ++k) q[0] += y[k];
        q[1] = row.part_dot(y, f);
      }
      if (norm_f || a.gate == 1) row.sums(q, red, turn);
      if (a.gate == 1 && live && row.j == 0) static_cast<T*>(a.o2)[r * a.ld2] = (T)q[2];
      if (norm_f) {
        const float r1 = dev_f * sc.dev, m0 = q[0] * inv_d, m1 = q[1] * inv_d;
#pragma unroll
        for (int k = 0; k < CPL; ++k) y[k] = r1 * fmaf(-f[k], m1, y[k] - m0);
      }
      if (live) row.store(static_cast<T*>(a.o1) + r * a.ld1, y);
    }
  }
  float* o = a.part + (int64_t)blockIdx.x * (a.post_rows + a.pre_rows) * a.d;
  const bool one = gridDim.x == 1;
  if constexpr (RES) {
    if (a.post) {
      join(row, awp, join_s, one ? a.dpost : o, one && a.add);
      if (a.post_rows == 2) join(row, abp, join_s, one ? a.dpost + a.d : o + a.d, one && a.add);
    }
  }
  if (a.pre) {
    o += a.post_rows * a.d;
    join(row, aw, join_s, one ? a.dpre : o, one && a.add);
    if (a.pre_rows == 2) join(row, ab, join_s, one ? a.dpre + a.d : o + a.d, one && a.add);
  }
}

// out[c] (+)= sum over the n partial rows, in 64 bits: 32 columns a block, 32
// groups of threads each sum every 32nd row, and the groups are added in order.
// The first `split` columns go to out0, the others to out1.
__global__ void __launch_bounds__(1024) k_residual_reduce(const float* __restrict__ part, int n, int count, int split,
                                                          float* __restrict__ out0, float* __restrict__ out1, int add) {
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
  float* o = col < split ? out0 + col : out1 + (col - split);
  *o = add ? *o + (float)s : (float)s;
}

__global__ void __launch_bounds__(256) k_residual_zero(int n, float* __restrict__ p) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

// Calls f with the narrowest layout that holds rows of width d.
template <class T, class F>
int with_layout(int d, bool vec, F&& f) {
  using std::integral_constant;
#define CHG_ROW(V, TPR, NQ)                                                                                              \
  if (d <= V * TPR * NQ) {                                                                                               \
    const integral_constant<int, V> v;                                                                                   \
    const integral_constant<int, TPR> l;                                                                                 \
    const integral_constant<int, NQ> n;                                                                                  \
    return vec ? f(v, l, n, std::false_type{}) : f(v, l, n, std::true_type{});                                           \
  }
  if constexpr (sizeof(T) == 2) {
    CHG_ROW(8, 8, 1)
    CHG_ROW(8, 16, 1)
    CHG_ROW(8, 32, 1)
    CHG_ROW(8, 64, 1)
    CHG_ROW(8, 128, 1)
    CHG_ROW(8, 256, 1)
    CHG_ROW(8, 512, 1)
    CHG_ROW(8, 1024, 1)
    CHG_ROW(8, 1024, 2)
  } else {
    CHG_ROW(4, 8, 1)
    CHG_ROW(4, 16, 1)
    CHG_ROW(4, 32, 1)
    CHG_ROW(4, 64, 1)
    CHG_ROW(4, 64, 2)
    CHG_ROW(4, 256, 1)
    CHG_ROW(4, 256, 2)
    CHG_ROW(4, 512, 2)
    CHG_ROW(4, 1024, 2)
    CHG_ROW(4, 1024, 4)
  }
#undef CHG_ROW
  return fail(CHGNET_EINVAL, "residual: d must be in 1..16384");
}

constexpr int kMostCols = 16384;

int bad(const char* who, const char* what) { return fail(CHGNET_EINVAL, std::string(who) + ": " + what); }

int check_shape(const char* who, int64_t rows, int32_t d, int32_t dtype) {
  if (rows < 0 || rows >= (int64_t(1) << 32)) return bad(who, "rows must be in 0 .. 2^32 - 1");
  if (d < 1 || d > kMostCols) return bad(who, "d must be in 1 .. 16384");
  if (!elem_size(dtype)) return bad(who, "unknown dtype");
  return CHGNET_OK;
}
int check_norm(const char* who, int32_t kind, const float* w, int32_t w_rows, bool none) {
  if (kind != kRms && kind != kLayer && !(none && kind == kNoNorm)) return bad(who, "unknown norm");
  if (w && w_rows != 1 && w_rows != 2) return bad(who, "a norm's parameters are one row (scale) or two (scale, shift)");
  if (!w && !(none && kind == kNoNorm)) return bad(who, "a norm needs its parameters");
  if (!aligned_to(w, 4)) return bad(who, "a norm's parameters are not aligned");
  return CHGNET_OK;
}
int check_cfg(const char* who, const chgnet_residual* c) {
  if (!(c->eps >= 1e-20f && c->eps <= 1.0f)) return bad(who, "eps must be in 1e-20 .. 1");
  if (!(c->p >= 0.0f && c->p <= 1.0f)) return bad(who, "p must be in 0 .. 1");
  if (!aligned_to(c->step, 8)) return bad(who, "step is not aligned");
  return CHGNET_OK;
}
struct Array {
  const void* p;
  int64_t ld, cols;
  bool needed;
};
// pointers, alignment to values and row strides; `vec`: 16-byte accesses are possible
int check_arrays(const char* who, std::initializer_list<Array> arrays, int d, size_t es, bool& vec) {
  vec = d * es % 16 == 0;
  for (const Array& x : arrays) {
    if (!x.p) {
      if (x.needed) return bad(who, "null argument");
      continue;
    }
    if (x.ld < x.cols) return bad(who, "a row stride is below the row's width");
    if (!aligned_to(x.p, es)) return bad(who, "an array is not aligned to its values");
    if (x.cols == d) vec = vec && x.ld * es % 16 == 0 && aligned_to(x.p, 16);
  }
  return CHGNET_OK;
}

// Blocks of a backward launch: rows of a block walked in turn; more than two
// turns are worth a second launch that adds the blocks' sums.
int bwd_blocks(int64_t rows, int rows_a_block, int at_most) {
  const int64_t turns = cdiv(rows, rows_a_block);
  return turns <= 2 ? 1 : (int)std::min<int64_t>(at_most, turns);
}

int launch_fwd(bool res, int32_t dtype, bool vec, const ResArgs& a, hipStream_t st) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_layout<T>(a.d, vec, [&](auto V, auto L, auto N, auto any) -> int {
      constexpr int threads = fwd_threads<L.value>(), rows = threads / L.value;
      const unsigned blocks = (unsigned)std::min<int64_t>(256 * 2048 / threads, cdiv(a.rows, rows));
      if (res)
        KLAUNCH(st, "k_residual_fwd", k_residual_fwd<T, V.value, L.value, N.value, any.value, true><<<blocks, threads, 0, st>>>(a));
      else
        KLAUNCH(st, "k_norm_fwd", k_residual_fwd<T, V.value, L.value, N.value, any.value, false><<<blocks, threads, 0, st>>>(a));
      return CHGNET_OK;
    });
  });
}

int launch_bwd(bool res, int32_t dtype, bool vec, ResArgs a, hipStream_t st) {
  int blocks = 1;
  CHG_TRY(with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_layout<T>(a.d, vec, [&](auto V, auto L, auto N, auto any) -> int {
      constexpr int threads = bwd_threads<L.value>();
      blocks = bwd_blocks(a.rows, threads / L.value,
                          res ? bwd_blocks_at_most<T, L.value, N.value, true>() : bwd_blocks_at_most<T, L.value, N.value, false>());
      if (res)
        KLAUNCH(st, "k_residual_bwd", k_residual_bwd<T, V.value, L.value, N.value, any.value, true><<<blocks, threads, 0, st>>>(a));
      else
        KLAUNCH(st, "k_norm_bwd", k_residual_bwd<T, V.value, L.value, N.value, any.value, false><<<blocks, threads, 0, st>>>(a));
      return CHGNET_OK;
    });
  }));
  const int count = (a.post_rows + a.pre_rows) * a.d;
  if (blocks > 1 && count)
    KLAUNCH(st, "k_residual_reduce", k_residual_reduce<<<(unsigned)cdiv(count, 32), 1024, 0, st>>>(
                                         a.part, blocks, count, a.post_rows * a.d, a.dpost, a.dpre, a.add));
  return CHGNET_OK;
}

int zero_grads(const ResArgs& a, hipStream_t st) {
  if (a.add) return CHGNET_OK;
  if (a.post_rows)
    KLAUNCH(st, "k_residual_zero",
            k_residual_zero<<<(unsigned)cdiv(a.post_rows * a.d, 256), 256, 0, st>>>(a.post_rows * a.d, a.dpost));
  if (a.pre_rows)
    KLAUNCH(st, "k_residual_zero",
            k_residual_zero<<<(unsigned)cdiv(a.pre_rows * a.d, 256), 256, 0, st>>>(a.pre_rows * a.d, a.dpre));
  return CHGNET_OK;
}

}  // namespace

int norm_forward_entry(int64_t rows, int32_t d, int32_t dtype, const void* x, int64_t ldx, int32_t kind, const float* w,
                       int32_t w_rows, float eps, void* h, int64_t ldh, hipStream_t st) {
  const char* who = "norm_forward";
  CHG_TRY(check_shape(who, rows, d, dtype));
  CHG_TRY(check_norm(who, kind, w, w_rows, false));
  if (!(eps >= 1e-20f && eps <= 1.0f)) return bad(who, "eps must be in 1e-20 .. 1");
  if (ldx < d || ldh < d) return bad(who, "a row stride is below the row's width");
  if (rows == 0) return CHGNET_OK;
  bool vec;
  CHG_TRY(check_arrays(who, {{x, ldx, d, true}, {h, ldh, d, true}}, d, elem_size(dtype), vec));
  ResArgs a{};
  a.rows = rows, a.d = d, a.x = x, a.ldx = ldx, a.pre = w, a.pre_kind = kind, a.pre_rows = w_rows, a.eps = eps;
  a.o1 = h, a.ld1 = ldh;
  return launch_fwd(false, dtype, vec, a, st);
}

int residual_backward_workspace_entry(int64_t rows, int32_t d, int32_t w_rows, size_t* bytes) {
  const char* who = "residual_backward_workspace";
  CHG_TRY(check_shape(who, rows, d, CHGNET_F32));
  if (w_rows < 0 || w_rows > 4) return bad(who, "param_rows must be in 0 .. 4");
  if (!bytes) return bad(who, "bytes is NULL");
  *bytes = sizeof(float) * (size_t)w_rows * (size_t)d * (size_t)std::min<int64_t>(kBwdBlocks, std::max<int64_t>(1, rows));
  return CHGNET_OK;
}

static int check_ws(const char* who, int64_t rows, int32_t d, int32_t w_rows, void* ws, size_t ws_bytes) {
  size_t need = 0;
  CHG_TRY(residual_backward_workspace_entry(rows, d, w_rows, &need));
  if (need && (!ws || ws_bytes < need))
    return fail(CHGNET_EWORKSPACE, std::string(who) + ": workspace too small (query chgnet_residual_backward_workspace)");
  if (!aligned_to(ws, 16)) return bad(who, "ws is not 16-byte aligned");
  return CHGNET_OK;
}

int norm_backward_entry(int64_t rows, int32_t d, int32_t dtype, const void* x, int64_t ldx, int32_t kind, const float* w,
                        int32_t w_rows, float eps, const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dw,
                        int accumulate, void* ws, size_t ws_bytes, hipStream_t st) {
  const char* who = "norm_backward";
  CHG_TRY(check_shape(who, rows, d, dtype));
  CHG_TRY(check_norm(who, kind, w, w_rows, false));
  if (!(eps >= 1e-20f && eps <= 1.0f)) return bad(who, "eps must be in 1e-20 .. 1");
  if (ldx < d || lddh < d || lddx < d) return bad(who, "a row stride is below the row's width");
  if (!dw || !aligned_to(dw, 4)) return bad(who, "dw is NULL or not aligned");
  ResArgs a{};
  a.rows = rows, a.d = d, a.pre_rows = w_rows, a.dpre = dw, a.add = accumulate != 0;
  if (rows == 0) return zero_grads(a, st);
  bool vec;
  CHG_TRY(check_arrays(who, {{x, ldx, d, true}, {dh, lddh, d, true}, {dx, lddx, d, true}}, d, elem_size(dtype), vec));
  CHG_TRY(check_ws(who, rows, d, w_rows, ws, ws_bytes));
  a.x = x, a.ldx = ldx, a.dh = dh, a.lddh = lddh, a.pre = w, a.pre_kind = kind, a.eps = eps;
  a.o0 = dx, a.ld0 = lddx, a.part = static_cast<float*>(ws);
  return launch_bwd(false, dtype, vec, a, st);
}

int residual_forward_entry(int64_t rows, int32_t d, int32_t dtype, const chgnet_residual* c, const void* x, int64_t ldx,
                           const void* f, int64_t ldf, const void* g, int64_t ldg, const float* post, const float* pre,
                           void* y, int64_t ldy, void* h, int64_t ldh, hipStream_t st) {
  const char* who = "residual_forward";
  CHG_TRY(check_shape(who, rows, d, dtype));
  if (!c) return bad(who, "cfg is NULL");
  CHG_TRY(check_cfg(who, c));
  CHG_TRY(check_norm(who, c->post_kind, post, c->post_rows, true));
  if (pre) CHG_TRY(check_norm(who, c->pre_kind, pre, c->pre_rows, false));
  if (g && c->gate_cols != 1 && c->gate_cols != d) return bad(who, "gate_cols must be 1 or d");
  if ((pre == nullptr) != (h == nullptr) && rows) return bad(who, "h needs the parameters pre of its norm, and pre an h");
  if (rows == 0) return CHGNET_OK;
  bool vec;
  CHG_TRY(check_arrays(who, {{x, ldx, d, true}, {f, ldf, d, true}, {g, ldg, g ? c->gate_cols : 0, false}, {y, ldy, d, true},
                             {h, ldh, d, false}}, d, elem_size(dtype), vec));
  ResArgs a{};
  a.rows = rows, a.d = d, a.x = x, a.ldx = ldx, a.f = f, a.ldf = ldf, a.g = g, a.ldg = ldg;
  a.gate = !g ? 0 : c->gate_cols == d ? 2 : 1;
  a.post = post, a.post_kind = c->post_kind, a.post_rows = post ? c->post_rows : 0;
  a.pre = pre, a.pre_kind = c->pre_kind, a.pre_rows = pre ? c->pre_rows : 0;
  a.alpha = c->alpha, a.beta = c->beta, a.eps = c->eps, a.drop = make_drop(c->p, c->seed, c->call, c->step);
  a.o0 = y, a.ld0 = ldy, a.o1 = h, a.ld1 = ldh;
  return launch_fwd(true, dtype, vec, a, st);
}

int residual_backward_entry(int64_t rows, int32_t d, int32_t dtype, const chgnet_residual* c, const void* y, int64_t ldy,
                            const void* f, int64_t ldf, const void* g, int64_t ldg, const float* post, const float* pre,
                            const void* dy, int64_t lddy, const void* dh, int64_t lddh, void* dx, int64_t lddx, void* df,
                            int64_t lddf, void* dg, int64_t lddg, float* dpost, float* dpre, int accumulate, void* ws,
                            size_t ws_bytes, hipStream_t st) {
  const char* who = "residual_backward";
  CHG_TRY(check_shape(who, rows, d, dtype));
  if (!c) return bad(who, "cfg is NULL");
  CHG_TRY(check_cfg(who, c));
  CHG_TRY(check_norm(who, c->post_kind, post, c->post_rows, true));
  if (pre) CHG_TRY(check_norm(who, c->pre_kind, pre, c->pre_rows, false));
  if (g && c->gate_cols != 1 && c->gate_cols != d) return bad(who, "gate_cols must be 1 or d");
  if ((post == nullptr) != (dpost == nullptr) || (pre == nullptr) != (dpre == nullptr))
    return bad(who, "dpost and dpre go with post and pre");
  if (!aligned_to(dpost, 4) || !aligned_to(dpre, 4)) return bad(who, "dpost or dpre is not aligned");
  ResArgs a{};
  a.rows = rows, a.d = d, a.add = accumulate != 0;
  a.post = post, a.post_kind = c->post_kind, a.post_rows = post ? c->post_rows : 0, a.dpost = dpost;
  a.pre = pre, a.pre_kind = c->pre_kind, a.pre_rows = pre ? c->pre_rows : 0, a.dpre = dpre;
  if (rows == 0) return zero_grads(a, st);
  if ((pre == nullptr) != (dh == nullptr)) return bad(who, "dh goes with pre");
  if ((g == nullptr) != (dg == nullptr)) return bad(who, "dgate goes with the gate");
  if (!dy && !dh) return bad(who, "neither dy nor dh is given");
  const bool use_f = post || g;
  bool vec;
  CHG_TRY(check_arrays(who, {{y, ldy, d, pre != nullptr}, {f, ldf, d, use_f}, {g, ldg, g ? c->gate_cols : 0, false},
                             {dy, lddy, d, false}, {dh, lddh, d, false}, {dx, lddx, d, true}, {df, lddf, d, true},
                             {dg, lddg, g ? c->gate_cols : 0, false}}, d, elem_size(dtype), vec));
  CHG_TRY(check_ws(who, rows, d, a.post_rows + a.pre_rows, ws, ws_bytes));
  a.x = y, a.ldx = ldy, a.f = use_f ? f : nullptr, a.ldf = ldf, a.g = g, a.ldg = ldg, a.dy = dy, a.lddy = lddy, a.dh = dh, a.lddh = lddh;
  a.gate = !g ? 0 : c->gate_cols == d ? 2 : 1;
  a.alpha = c->alpha, a.beta = c->beta, a.eps = c->eps, a.drop = make_drop(c->p, c->seed, c->call, c->step);
  a.o0 = dx, a.ld0 = lddx, a.o1 = df, a.ld1 = lddf, a.o2 = dg, a.ld2 = lddg, a.part = static_cast<float*>(ws);
  return launch_bwd(true, dtype, vec, a, st);
}

}  // namespace chg
