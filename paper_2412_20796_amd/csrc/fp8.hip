// Matrix products of 8-bit floating point with a power of two for each block of
// 128 values (chgnet_ops.h), and the quantiser that makes their factors.
//
//   code = e4m3(x 2^-e),  2^e the least power of two with max |x| <= 448 2^e in
//   the block, at least 2^-126;  out[m][n] = sum over k of a[m][k] b[n][k]
//
// Powers of two because the matrix instruction multiplies by them: its operands
// carry 8-bit exponents beside the codes, so a block's scale costs no vector
// work and no rounding. In floating-point codes they cost no precision either,
// but for values some 2^-16 of their block's largest.
//
// The instruction adds eight products at a time in steps of 2^-13 of the largest
// one's power of two and cuts off what is below (measured; sums of such eights are
// fp32's). For normal values a result is off by 1.5e-5 of its size, 7e-5 where
// columns are up to hundreds of times as loud as others: inside the half step of a
// 16-bit result (fp16's rounding alone is 2.1e-4). Results in fp32 take the codes as bf16
// values, which hold them and their scales exactly, and its products, which are
// added to fp32's last place, at half of the rate.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "elem.hpp"
#include "rowops.hpp"

namespace chg {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef bf16_t v2b __attribute__((ext_vector_type(2)));
typedef bf16_t v8b __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;   // values under one scale
constexpr int64_t kMostK = 1 << 23, kMostRows = int64_t(1) << 31;

// ---------------------------------------------------------------------------
// Scales and codes
// ---------------------------------------------------------------------------

// Exponent byte (2^(e - 127)) for a block's largest magnitude, as fp32 bits: at
// most 1.75 2^8 in codes. 255, which stands for NaN, where a value is not finite.
__device__ __forceinline__ unsigned scale_byte(unsigned big) {
  const int e = (int)((big + 0x1fffffu) >> 23) - 8;  // one more above a mantissa of 1.75
  return big >= 0x7f800000u ? 255u : (unsigned)(e < 1 ? 1 : e);
}
// 2^-e of such a byte; 0 for NaN, so that the block's codes are 0 (or NaN, which
// the products have anyway)
__device__ __forceinline__ float scale_inverse(unsigned byte) {
  return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);
}
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// four codes, the first in the low byte
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
  unsigned r = 0;
  r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
template <int LPR>
__device__ __forceinline__ unsigned rowmax_bits(unsigned v) {
  auto step = [&](unsigned o) { v = o > v ? o : v; };
  step(__float_as_uint(dpp<0xB1>(__uint_as_float(v))));
  step(__float_as_uint(dpp<0x4E>(__uint_as_float(v))));
  if (LPR >= 8) step(__float_as_uint(dpp<0x141>(__uint_as_float(v))));
  if (LPR >= 16) step(__float_as_uint(dpp<0x140>(__uint_as_float(v))));
  return v;
}
// largest over the four groups of 16 lanes
__device__ __forceinline__ unsigned groupmax_bits(unsigned v) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = a[0] > a[1] ? a[0] : a[1];
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return b[0] > b[1] ? b[0] : b[1];
}

// Eight values of a row as they are stored, in words, and the order of their
// magnitudes without conversions: that of the bits below the sign.
template <class T>
struct Eight {
  static constexpr int NW = 2 * sizeof(T);
  typedef unsigned short pair __attribute__((ext_vector_type(2)));
  unsigned w[NW];
  // (the hardware takes 16 bytes at any address)
  __device__ __forceinline__ void load(const T* p) {
    typedef unsigned words __attribute__((ext_vector_type(4)));
    typedef words any __attribute__((aligned(2)));
#pragma unroll
    for (int q = 0; q < NW / 4; ++q) {
      const words t = reinterpret_cast<const any*>(p)[q];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[4 * q + k] = t[k];
    }
  }
  // the first n of them, 0 for the others
  __device__ __forceinline__ void load_some(const T* p, int64_t n) {
    typedef typename std::conditional<sizeof(T) == 4, unsigned, unsigned short>::type bits;
    const bits* b = reinterpret_cast<const bits*>(p);
#pragma unroll
    for (int q = 0; q < NW; ++q) w[q] = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) w[k * NW / 8] |= (unsigned)b[k] << (sizeof(T) == 2 && k % 2 ? 16 : 0);
  }
  __device__ __forceinline__ float get(int k) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
    else return bits16(k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffffu);
  }
  // the value of 16 bits
  static __device__ __forceinline__ float bits16(unsigned b) {
    if constexpr (std::is_same<T, bf16_t>::value) return __uint_as_float(b << 16);
    else return (float)__builtin_bit_cast(f16_t, (unsigned short)b);
  }
  static __device__ __forceinline__ unsigned below_sign(unsigned w) { return w & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu); }
  // of words without signs, half by half
  static __device__ __forceinline__ unsigned larger(unsigned a, unsigned b) {
    if constexpr (sizeof(T) == 4) return max(a, b);
    else return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(pair, a), __builtin_bit_cast(pair, b)));
  }
  // fp32 bits of the larger value of a word, and of half h
  static __device__ __forceinline__ unsigned largest(unsigned w) {
    if constexpr (sizeof(T) == 4) return w;
    else return __float_as_uint(bits16(max(w & 0xffffu, w >> 16)));
  }
  static __device__ __forceinline__ unsigned half(unsigned w, int h) {
    if constexpr (sizeof(T) == 4) return w;
    else return __float_as_uint(bits16(h ? w >> 16 : w & 0xffffu));
  }
  // kept from being converted once for all uses: the floats of 64 values have no room
  __device__ __forceinline__ void fence() {
#pragma unroll
    for (int q = 0; q < NW; ++q) asm volatile("" : "+v"(w[q]));
  }
};

// Rows under 1 x 128 scales: 16 lanes have a block, 8 values each.
template <class T>
__global__ void __launch_bounds__(256) k_fp8_rows(int64_t rows, int64_t cols, const T* __restrict__ x, int64_t ldx,
                                                  uint8_t* __restrict__ codes, int64_t ldc, uint8_t* __restrict__ scale,
                                                  int64_t lds) {
  const int64_t nb = (cols + kBlock - 1) / kBlock, end = (cols + 15) / 16 * 16;
  const int j = threadIdx.x & 15;
  const int64_t stride = (int64_t)gridDim.x * 16;
  for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < rows * nb; i += stride) {
    const int64_t row = i / nb, b = i - row * nb, c = b * kBlock + 8 * j;
    using E = Eight<T>;
    E v;
    if (c + 8 <= cols) v.load(x + row * ldx + c);
    else v.load_some(x + row * ldx + c, cols - c);
    unsigned big = E::below_sign(v.w[0]);
#pragma unroll
    for (int k = 1; k < E::NW; ++k) big = E::larger(big, E::below_sign(v.w[k]));
    const unsigned byte = scale_byte(rowmax_bits<16>(E::largest(big)));
    const float inv = scale_inverse(byte);
    if (c < end) {
      uint2 q;
      q.x = codes4(v.get(0) * inv, v.get(1) * inv, v.get(2) * inv, v.get(3) * inv);
      q.y = codes4(v.get(4) * inv, v.get(5) * inv, v.get(6) * inv, v.get(7) * inv);
      *reinterpret_cast<uint2*>(codes + row * ldc + c) = q;
    }
    if (j == 0) scale[row * lds + b] = (uint8_t)byte;
  }
}

// Tiles of 128 x 128, `count` (1 or 4) below each other a block: codes of them and
// of their transpose (either may be left out). SQUARE: one scale for a tile, which
// both share; else 1 x 128 of the rows of each. A thread has 8 x 8 values; the
// transposed codes go through LDS, in units of the 8 bytes that a thread has of a
// column, unit u of column c at u ^ (c / 8 % 16), so that 16 lanes write to 16
// banks' pairs. Blocks of four tiles write the transpose's scales in words; single
// bytes far from each other were a third of all writes, as long as rows of codes
// started anywhere. In whole lines of codes blocks of one tile are as fast or faster
// (397,934 x 512 in bf16, both forms: 167 us of one, 180 of four; 16,384 x 16,384: 237
// and 240).
template <class T, bool SQUARE>
__global__ void __launch_bounds__(256, 4) k_fp8_tile(int64_t rows, int64_t cols, const T* __restrict__ x, int64_t ldx,
                                                     uint8_t* __restrict__ codes, int64_t ldc, uint8_t* __restrict__ scale,
                                                     int64_t lds, uint8_t* __restrict__ codes_t, int64_t ldct,
                                                     uint8_t* __restrict__ scale_t, int64_t ldst, int count) {
  __shared__ uint2 tile[128][16];
  __shared__ unsigned colmax[4][128];
  __shared__ unsigned words[128];  // a column's scale bytes in the block's tiles
  const int64_t tiles_c = (cols + 127) / 128, tiles_r = (rows + 127) / 128;
  const int64_t tc = blockIdx.x % tiles_c, tr0 = blockIdx.x / tiles_c * count;
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t c0 = tc * 128 + cg * 8;
  const int64_t end_c = (cols + 15) / 16 * 16, end_r = (rows + 15) / 16 * 16;
  for (int t = 0; t < count && tr0 + t < tiles_r; ++t) {
    asm volatile("" : "+s"(t));  // addresses are formed for each tile, not kept for all
    const int64_t tr = tr0 + t, r0 = tr * 128 + rg * 8;
    using E = Eight<T>;
    constexpr int NW = E::NW;
    E v[8];
    {
      const T* p = x + r0 * ldx + c0;
      const int there = (int)(rows - r0 < 8 ? rows - r0 : 8);  // rows of this thread's (may be none)
      if (c0 + 8 <= cols && there == 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i].load(p + i * ldx);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i].load_some(p + i * ldx, i < there ? cols - c0 : 0);
      }
    }
    unsigned col[NW];
#pragma unroll
    for (int q = 0; q < NW; ++q) {
      col[q] = E::below_sign(v[0].w[q]);
#pragma unroll
      for (int i = 1; i < 8; ++i) col[q] = E::larger(col[q], E::below_sign(v[i].w[q]));
    }
    unsigned whole = 0;
    if constexpr (SQUARE) {
#pragma unroll
      for (int q = 1; q < NW; ++q) col[0] = E::larger(col[0], col[q]);
      whole = groupmax_bits(rowmax_bits<16>(E::largest(col[0])));
      if (lane == 0) colmax[wave][0] = whole;
    } else {
#pragma unroll
      for (int q = 0; q < NW; ++q) {
        const auto a = __builtin_amdgcn_permlane16_swap(col[q], col[q], false, false);
        const unsigned m = E::larger(a[0], a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        if (lane < 16) colmax[wave][cg * NW + q] = E::larger(b[0], b[1]);
      }
    }
    __syncthreads();  // (the last tile's codes are read, too)
    if constexpr (SQUARE) whole = max(max(colmax[0][0], colmax[1][0]), max(colmax[2][0], colmax[3][0]));
    const unsigned all = scale_byte(whole);
    if (codes) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        unsigned byte = all;
        v[i].fence();
        if constexpr (!SQUARE) {
          unsigned big = E::below_sign(v[i].w[0]);
#pragma unroll
          for (int q = 1; q < NW; ++q) big = E::larger(big, E::below_sign(v[i].w[q]));
          byte = scale_byte(rowmax_bits<16>(E::largest(big)));
        }
        const float inv = scale_inverse(byte);
        if (r0 + i < rows) {
          if (c0 < end_c) {
            const E& r = v[i];
            uint2 q;
            q.x = codes4(r.get(0) * inv, r.get(1) * inv, r.get(2) * inv, r.get(3) * inv);
            q.y = codes4(r.get(4) * inv, r.get(5) * inv, r.get(6) * inv, r.get(7) * inv);
            *reinterpret_cast<uint2*>(codes + (r0 + i) * ldc + c0) = q;
          }
          if (!SQUARE && cg == 0) scale[(r0 + i) * lds + tc] = (uint8_t)byte;
        }
      }
      if (SQUARE && threadIdx.x == 0) scale[tr * lds + tc] = (uint8_t)all;
    }
    if (!codes_t) {
      __syncthreads();  // colmax is read
      continue;
    }
    if constexpr (!SQUARE) {
#pragma unroll
      for (int q = 0; q < NW; ++q) {
        const int c = cg * NW + q;
        col[q] = E::larger(E::larger(colmax[0][c], colmax[1][c]), E::larger(colmax[2][c], colmax[3][c]));
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i].fence();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = cg * 8 + k;
      unsigned byte = all;
      if constexpr (!SQUARE) {
        byte = scale_byte(E::half(col[k * NW / 8], k & 1));
        if (rg == 0) words[c] = (t ? words[c] : 0u) | byte << (8 * t);
      }
      const float inv = scale_inverse(byte);
      uint2 q;
      q.x = codes4(v[0].get(k) * inv, v[1].get(k) * inv, v[2].get(k) * inv, v[3].get(k) * inv);
      q.y = codes4(v[4].get(k) * inv, v[5].get(k) * inv, v[6].get(k) * inv, v[7].get(k) * inv);
      tile[c][rg ^ cg] = q;
    }
    if (SQUARE && threadIdx.x == 0) scale_t[tc * ldst + tr] = (uint8_t)all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = i * 256 + threadIdx.x, c = p >> 3, u = p & 7, g = c >> 3;
      const int64_t cc = tc * 128 + c, rr = tr * 128 + u * 16;
      const uint2 a = tile[c][(2 * u) ^ g], b = tile[c][(2 * u + 1) ^ g];
      if (cc < cols && rr < end_r) *reinterpret_cast<uint4*>(codes_t + cc * ldct + rr) = make_uint4(a.x, a.y, b.x, b.y);
    }
  }
  if constexpr (!SQUARE) {
    if (!codes_t || threadIdx.x >= 128 || tc * 128 + threadIdx.x >= cols) return;
    // (the words are this thread's block's: written before its last barrier)
    uint8_t* p = scale_t + (tc * 128 + threadIdx.x) * ldst + tr0;
    const unsigned w = words[threadIdx.x];
    if (count == 4 && tr0 + 4 <= tiles_r) {
      *reinterpret_cast<unsigned*>(p) = w;
    } else {
      for (int t = 0; t < count && tr0 + t < tiles_r; ++t) p[t] = (uint8_t)(w >> (8 * t));
    }
  }
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

// One factor: codes [rows, K] and scale bytes [rows / 128 or rows, K / 128]
struct Factor {
  const uint8_t *codes, *scale;
  int64_t ldc, lds;
  int64_t rows;
  int shift;  // row >> shift has the scales: 7 (a block of 128 rows) or 0
};
struct ProductArgs {
  Factor a, b;
  int64_t K;
  void* out;
  int64_t ldo;
  float* part;  // [split][M][ldp] partial sums, or NULL: `out` is written
  int64_t ldp;
  int splits, kb_split;  // parts of K, and blocks of 128 along it that one has
  int add;
};

// 16 or 4 bytes a lane past the registers: to `l` and the lanes' places behind it
__device__ __forceinline__ void to_lds16(const void* g, void* l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g,
                                   (__attribute__((address_space(3))) void*)l, 16, 0, 0);
}
__device__ __forceinline__ void to_lds4(const void* g, void* l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g,
                                   (__attribute__((address_space(3))) void*)l, 4, 0, 0);
}

// barrier of the block once all but the last COUNT of this wavefront's loads are
// done, and what it wrote to LDS
template <int COUNT>
__device__ __forceinline__ void wait_barrier() {
  static_assert(COUNT < 64, "six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(COUNT) : "memory");
}

// 8 codes as bf16 values, times their scale
__device__ __forceinline__ v8b wide(const uint2& q, float s) {
  const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.x, s, false);
  const v2b b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.x, s, true);
  const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.y, s, false);
  const v2b d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.y, s, true);
  return v8b{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// 2^(byte - 127) for the low byte of a word
__device__ __forceinline__ float scale_value(unsigned word) {
  const unsigned byte = word & 255;
  return byte == 255 ? __builtin_nanf("") : __uint_as_float(byte ? byte << 23 : 0x400000u);
}

// Up to 16 bytes of results of a row, of which the first `left` are the matrix's, at
// any value's address
template <class T, int W>
__device__ __forceinline__ void put(T* p, float (&t)[W], int64_t left, bool add) {
  typedef T vec __attribute__((ext_vector_type(W)));
  typedef vec any __attribute__((aligned(sizeof(T))));
  if (left >= W) {
    vec v;
    if (add) {
      v = *reinterpret_cast<const any*>(p);
#pragma unroll
      for (int k = 0; k < W; ++k) t[k] += (float)v[k];
    }
#pragma unroll
    for (int k = 0; k < W; ++k) v[k] = (T)t[k];
    *reinterpret_cast<any*>(p) = v;
  } else {
#pragma unroll
    for (int k = 0; k < W - 1; ++k)
      if (k < left) p[k] = (T)(add ? (float)p[k] + t[k] : t[k]);
  }
}

// A block has BM x BN results, its WM x WN wavefronts equal parts of them. Both
// factors' codes of 128 values of K go to LDS past the registers, the next ones
// while the present are multiplied. The factors change places in the instruction,
// so that a lane has four results of a row for each operand of b; which column is
// which of an operand's rows is such that these, or those of two operands in 16
// bits, are 16 bytes that follow each other, beside those of the other lane groups.
// A row's 8 pieces of 16 bytes sit at piece ^ key(row), the keys such that the 16
// rows of an operand meet in no bank: 16 lanes read 256 bytes, two rows, at a
// time (with keys of row % 8 a load took twice as long: 8192^3 463 us in place of 420).
// EXACT: products of bf16 values, 32 of a block's 128 at a time.
template <class T, bool EXACT, int BM, int BN, int WM, int WN, int STAGES>
__global__ void __launch_bounds__(64 * WM * WN, (WM * WN) / 4) k_fp8_product(ProductArgs p) {
  constexpr int THREADS = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int PIECES = (BM + BN) * 8 / THREADS;  // of 16 bytes, a thread
  constexpr int W = 16 / sizeof(T);                // results in 16 bytes
  static_assert(TN == 4 && THREADS % 256 == 0, "64 columns a wavefront");
  __shared__ __align__(1024) uint8_t lds[STAGES][(BM + BN) * kBlock];
  __shared__ unsigned words[STAGES][BM + BN];
  const int64_t M = p.a.rows, N = p.b.rows;
  const int64_t tiles_m = (M + BM - 1) / BM, tiles_n = (N + BN - 1) / BN, tiles = tiles_m * tiles_n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  const int nkb = (int)((p.K + kBlock - 1) / kBlock);

  // Items: the tiles of each part of K. Each of the 8 chiplets has a run of tiles,
  // in groups of 8 rows of tiles.
  struct Item {
    int64_t m0, n0;
    int split, kb0, kb1;
  };
  const int64_t items = tiles * p.splits;
  auto item_at = [&](int64_t item) -> Item {
    Item t;
    t.split = (int)(item / tiles);
    int64_t tile = item - t.split * tiles;
    const int64_t q = tiles / 8, r = tiles % 8, x = tile % 8;
    tile = x * q + (x < r ? x : r) + tile / 8;
    const int64_t group = 8 * tiles_n, gr = tile / group, first = gr * 8, size = tiles_m - first < 8 ? tiles_m - first : 8;
    const int64_t in = tile - gr * group;
    t.m0 = (first + in % size) * BM;
    t.n0 = in / size * BN;
    t.kb0 = t.split * p.kb_split;
    t.kb1 = t.kb0 + p.kb_split < nkb ? t.kb0 + p.kb_split : nkb;
    return t;
  };

  // The loads run STAGES - 1 steps ahead of the products, into the next item where
  // this one has no more: its first codes arrive while results are stored.
  // Pieces and scales are at offsets from the item's first rows: rows past the end
  // are the last one again. A word of scales has a row's bytes of four blocks of K.
  constexpr int A_PIECES = BM * 8 / THREADS, WORDS = (BM + BN + THREADS - 1) / THREADS;
  static_assert(BM * 8 % THREADS == 0 && BN * 8 % THREADS == 0, "a step's pieces are of one factor");
  int64_t ahead_item = blockIdx.x;
  int ahead_kb, ahead_kb0, ahead_kb1, ahead_words = 0, issued = 0;
  const uint8_t *codes_a, *codes_b, *scale_a, *scale_b;
  unsigned src[PIECES], word_src[WORDS];
  auto piece = [&](int i) -> unsigned {
    const unsigned key = i < A_PIECES || W == 4 ? threadIdx.x >> 4 & 7 : (threadIdx.x >> 4 & 1) | (threadIdx.x >> 6 & 3) << 1;
    return 16 * ((threadIdx.x & 7) ^ key);
  };
  auto load_item = [&]() {
    const Item t = item_at(ahead_item);
    ahead_kb = ahead_kb0 = t.kb0;
    ahead_kb1 = t.kb1;
    const int last_a = (int)(M - t.m0 < BM ? M - t.m0 : BM) - 1, last_b = (int)(N - t.n0 < BN ? N - t.n0 : BN) - 1;
    codes_a = p.a.codes + t.m0 * p.a.ldc;
    codes_b = p.b.codes + t.n0 * p.b.ldc;
    scale_a = p.a.scale + (t.m0 >> p.a.shift) * p.a.lds;
    scale_b = p.b.scale + (t.n0 >> p.b.shift) * p.b.lds;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int row = (i * THREADS + threadIdx.x) / 8 - (i < A_PIECES ? 0 : BM), last = i < A_PIECES ? last_a : last_b;
      src[i] = (unsigned)(row < last ? row : last) * (unsigned)(i < A_PIECES ? p.a.ldc : p.b.ldc);
    }
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      const int row = i * THREADS + threadIdx.x;
      const bool is_a = row < BM;
      const Factor& f = is_a ? p.a : p.b;
      const int r = is_a ? row : row - BM, last = is_a ? last_a : last_b;
      // (an item starts at a row of blocks)
      word_src[i] = (unsigned)((r < last ? r : last) >> f.shift) * (unsigned)f.lds;
    }
  };
  auto load_step = [&](int buf) {
    if (ahead_item >= items || ahead_kb >= ahead_kb1) return;
    if (((ahead_kb - ahead_kb0) & 3) == 0) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        if (i * THREADS + wave * 64 >= BM + BN) break;
        to_lds4((i * THREADS + wave * 64 < BM ? scale_a : scale_b) + ahead_kb + word_src[i],
                words[ahead_words] + i * THREADS + wave * 64);
      }
      ahead_words = ahead_words + 1 == STAGES ? 0 : ahead_words + 1;
    }
    const int64_t at = (int64_t)ahead_kb * kBlock;
    uint8_t* to = lds[buf] + wave * 1024;
    if (at + kBlock <= p.K) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        to_lds16((i < A_PIECES ? codes_a : codes_b) + at + (src[i] + piece(i)), to + i * THREADS * 16);
    } else {  // pieces past the end of K are zeros (a wavefront has some before it: it counts as many loads)
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        if (at + piece(i) < p.K)
          to_lds16((i < A_PIECES ? codes_a : codes_b) + at + (src[i] + piece(i)), to + i * THREADS * 16);
        else
          *reinterpret_cast<uint4*>(to + i * THREADS * 16 + (threadIdx.x & 63) * 16) = make_uint4(0, 0, 0, 0);
      }
    }
    ++issued;
    if (++ahead_kb == ahead_kb1) {
      ahead_item += gridDim.x;
      if (ahead_item < items) load_item();
    }
  };
  const int r16 = lane & 15, g = lane >> 4;
  unsigned ea[TM], eb[TN];
  v4f acc[TM][TN];
  // half h of a lane's 32 codes of an operand: piece g + 4 h of its row
  auto column = [](int row, int j) { return (row >> 2) * W + (row & 3) + j / (W / 4) * 4 * W + j % (W / 4) * 4; };
  const int key = r16 >> 1;
  auto half_a = [&](int buf, int i, int h) {
    return *reinterpret_cast<const v4i*>(lds[buf] + (wm + 16 * i + r16) * kBlock + ((g + 4 * h) ^ key) * 16);
  };
  auto half_b = [&](int buf, int j, int h) {
    return *reinterpret_cast<const v4i*>(lds[buf] + (BM + wn + column(r16, j)) * kBlock + ((g + 4 * h) ^ key) * 16);
  };
  auto whole = [](const v4i& a, const v4i& b) { return v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; };
  // the first loads, and then for each item its steps and results
  constexpr int MAY = (STAGES - 2) * PIECES, STORES = TM * (16 / W);
  load_item();
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) load_step(i);
  int buf = 0, word = 0, done = 0;
  bool stored = false;  // STORES stores are the last that this wavefront did
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const Item t = item_at(item);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int kb = t.kb0; kb < t.kb1; ++kb) {
      // the codes of this step are there (loads and stores end in order; the loads of
      // the next STAGES - 2 steps and the last item's stores may be under way), and
      // all have read what is loaded over
      if (issued - done <= STAGES - 2) wait_barrier<0>();
      else if (stored) wait_barrier<MAY + STORES>();
      else wait_barrier<MAY>();
      stored = false;
      ++done;
      if (((kb - t.kb0) & 3) == 0) {
        const unsigned* w = words[word];
        word = word + 1 == STAGES ? 0 : word + 1;
#pragma unroll
        for (int i = 0; i < TM; ++i) ea[i] = w[wm + 16 * i + r16];
#pragma unroll
        for (int j = 0; j < TN; ++j) eb[j] = w[BM + wn + column(r16, j)];
      } else {
#pragma unroll
        for (int i = 0; i < TM; ++i) ea[i] >>= 8;
#pragma unroll
        for (int j = 0; j < TN; ++j) eb[j] >>= 8;
      }
      load_step(buf == 0 ? STAGES - 1 : buf - 1);
      constexpr int AHEAD = TM > 2 ? 2 : TM - 1;  // operands of a that are loaded ahead of their products
      if constexpr (EXACT) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v4i a[AHEAD + 1], b[TN];
          v8b bw[TN][2];
#pragma unroll
          for (int j = 0; j < TN; ++j) b[j] = half_b(buf, j, h);
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) a[i] = half_a(buf, i, h);
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            bw[j][0] = wide(make_uint2(b[j][0], b[j][1]), scale_value(eb[j]));
            bw[j][1] = wide(make_uint2(b[j][2], b[j][3]), scale_value(eb[j]));
          }
#pragma unroll
          for (int i = 0; i < TM; ++i) {
            if (i + AHEAD < TM) a[(i + AHEAD) % (AHEAD + 1)] = half_a(buf, i + AHEAD, h);
            const v4i q = a[i % (AHEAD + 1)];
            const v8b w0 = wide(make_uint2(q[0], q[1]), scale_value(ea[i]));
            const v8b w1 = wide(make_uint2(q[2], q[3]), scale_value(ea[i]));
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[j][0], w0, acc[i][j], 0, 0, 0);
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[j][1], w1, acc[i][j], 0, 0, 0);
          }
        }
      } else {
        v8i a[AHEAD + 1], b[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) b[j] = whole(half_b(buf, j, 0), half_b(buf, j, 1));
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) a[i] = whole(half_a(buf, i, 0), half_a(buf, i, 1));
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * (TN + AHEAD), 0);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          if (i + AHEAD < TM) {
            a[(i + AHEAD) % (AHEAD + 1)] = whole(half_a(buf, i + AHEAD, 0), half_a(buf, i + AHEAD, 1));
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          }
#pragma unroll
          for (int j = 0; j < TN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a[i % (AHEAD + 1)], acc[i][j], 0, 0, 0, eb[j], 0,
                                                                         ea[i]);
          __builtin_amdgcn_sched_group_barrier(0x8, TN, 0);
        }
      }
      buf = buf + 1 == STAGES ? 0 : buf + 1;
    }
    T* out = static_cast<T*>(p.out);
    int64_t ld = p.ldo;
    if constexpr (W == 4) {
      if (p.part) {
        out = p.part + (int64_t)t.split * M * p.ldp;
        ld = p.ldp;
      }
    }
    const bool add = p.add && !p.part;
    stored = !add && t.m0 + BM <= M && t.n0 + BN <= N;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = t.m0 + wm + 16 * i + r16;
#pragma unroll
      for (int q = 0; q < 16 / W; ++q) {
        const int64_t n = t.n0 + wn + q * 4 * W + g * W;
        float v[W];
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = acc[i][(q * W + k) / 4][k % 4];
        if (stored) put(out + m * ld + n, v, W, false);
        else if (m < M) put(out + m * ld + n, v, N - n, add);
      }
    }
  }
}

// Up to 16 rows of a, where what takes the time is b's codes: a block has NT x 16
// columns, and its eight wavefronts the blocks of K in turn; b goes from memory to
// registers, up to four blocks of K at a time. QUANT: a is rows of T in place of codes
// (x), quantised by each wavefront as it needs them, which costs less than a launch:
// lane group g of a block of K has the values 32 g .. 32 g + 31 of row lane % 16, and
// the largest of the four groups is the block's.
template <class T, bool EXACT, bool QUANT, int NT>
__global__ void __launch_bounds__(512) k_fp8_few(ProductArgs p, const T* __restrict__ x, int64_t ldx) {
  constexpr int WAVES = 8;
  __shared__ v4f parts[WAVES][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int64_t M = p.a.rows, N = p.b.rows, K = p.K, n0 = (int64_t)blockIdx.x * 16 * NT;
  const int64_t m = r16 < M ? r16 : M - 1;  // rows past the end: the last one again
  const int nkb = (int)((K + kBlock - 1) / kBlock);
  const uint8_t *b[NT], *sb[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t n = n0 + 16 * j + r16 < N ? n0 + 16 * j + r16 : N - 1;
    b[j] = p.b.codes + n * p.b.ldc + 32 * g;
    sb[j] = p.b.scale + (n >> p.b.shift) * p.b.lds;
  }
  const uint8_t* a = QUANT ? nullptr : p.a.codes + m * p.a.ldc;
  const uint8_t* sa = QUANT ? nullptr : p.a.scale + (m >> p.a.shift) * p.a.lds;
  const T* xr = QUANT ? x + m * ldx : nullptr;
  v4f acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j] = v4f{0.f, 0.f, 0.f, 0.f};
  struct In {
    uint4 b[NT][2];
    Eight<T> x[QUANT ? 4 : 1];
    uint4 a[QUANT ? 1 : 2];
    unsigned eb[NT], ea;
  };
  auto load = [&](int kb, In& in) {
    const int64_t c = (int64_t)kb * kBlock + 32 * g;
    const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool there = c + 16 * h < K;  // (bytes between K and the next multiple of 16 are 0)
#pragma unroll
      for (int j = 0; j < NT; ++j)
        in.b[j][h] = there ? *reinterpret_cast<const uint4*>(b[j] + (int64_t)kb * kBlock + 16 * h) : zero;
      if constexpr (!QUANT) in.a[h] = there ? *reinterpret_cast<const uint4*>(a + c + 16 * h) : zero;
    }
    if constexpr (QUANT) {
      if (c + 32 <= K) {
#pragma unroll
        for (int q = 0; q < 4; ++q) in.x[q].load(xr + c + 8 * q);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) in.x[q].load_some(xr + c + 8 * q, K - c - 8 * q);
      }
    } else {
      in.ea = sa[kb];
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) in.eb[j] = sb[j][kb];
  };
  auto multiply = [&](In& in) {
    uint2 qa[4];
    if constexpr (QUANT) {
      using E = Eight<T>;
      unsigned big = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int k = 0; k < E::NW; ++k) big = E::larger(big, E::below_sign(in.x[q].w[k]));
      in.ea = scale_byte(groupmax_bits(E::largest(big)));
      const float inv = scale_inverse(in.ea);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const E& v = in.x[q];
        qa[q].x = codes4(v.get(0) * inv, v.get(1) * inv, v.get(2) * inv, v.get(3) * inv);
        qa[q].y = codes4(v.get(4) * inv, v.get(5) * inv, v.get(6) * inv, v.get(7) * inv);
      }
    } else {
      qa[0] = make_uint2(in.a[0].x, in.a[0].y);
      qa[1] = make_uint2(in.a[0].z, in.a[0].w);
      qa[2] = make_uint2(in.a[1].x, in.a[1].y);
      qa[3] = make_uint2(in.a[1].z, in.a[1].w);
    }
    const v8i wa = {(int)qa[0].x, (int)qa[0].y, (int)qa[1].x, (int)qa[1].y, (int)qa[2].x, (int)qa[2].y, (int)qa[3].x, (int)qa[3].y};
    v8b xa[EXACT ? 4 : 1];
    if constexpr (EXACT) {
#pragma unroll
      for (int q = 0; q < 4; ++q) xa[q] = wide(qa[q], scale_value(in.ea));
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const uint4 lo = in.b[j][0], hi = in.b[j][1];
      if constexpr (EXACT) {
        const float f = scale_value(in.eb[j]);
        const uint2 qb[4] = {make_uint2(lo.x, lo.y), make_uint2(lo.z, lo.w), make_uint2(hi.x, hi.y), make_uint2(hi.z, hi.w)};
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide(qb[q], f), xa[q], acc[j], 0, 0, 0);
      } else {
        const v8i wb = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb, wa, acc[j], 0, 0, 0, in.eb[j], 0, in.ea);
      }
    }
  };
  constexpr int DEPTH = NT == 1 ? 4 : 2;
  In in[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH; ++i)
    if (wave + i * WAVES < nkb) load(wave + i * WAVES, in[i]);
  for (int kb = wave; kb < nkb; kb += DEPTH * WAVES) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      if (kb + i * WAVES >= nkb) break;
      multiply(in[i]);
      if (kb + (i + DEPTH) * WAVES < nkb) load(kb + (i + DEPTH) * WAVES, in[i]);
    }
  }
  // columns n0 + 16 j + 4 g .. of row r16, summed over the wavefronts in order
#pragma unroll
  for (int j = 0; j < NT; ++j) parts[wave][j][lane] = acc[j];
  __syncthreads();
  if (wave >= NT || r16 >= M) return;
  v4f sum = parts[0][wave][lane];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) sum += parts[w][wave][lane];
  const int64_t n = n0 + 16 * wave + 4 * g;
  float t[4] = {sum[0], sum[1], sum[2], sum[3]};
  put(static_cast<T*>(p.out) + r16 * p.ldo + n, t, N - n, p.add != 0);
}

// Linear layer of many rows to up to BN columns: a block has 64 rows of x, each
// read once and quantised on its way to LDS, and all columns. Sixteen threads have
// a row's 128 values of a step; those of the next step arrive while this one's are
// multiplied. Places in LDS and operands are k_fp8_product's. x's codes have one
// buffer, which all read before they multiply: two blocks have room on a compute unit.
// x is not `__restrict__`: a wait counts its loads, and so needs them where they are
// written; the compiler may move loads of memory that nothing else can write past it.
template <class T, bool EXACT, int BN>
__global__ void __launch_bounds__(2 * BN, 4) k_fp8_rows_product(ProductArgs p, const T* x, int64_t ldx) {
  constexpr int BM = 64, WN = BN / 64, THREADS = 2 * BN, TM = 2, TN = 4, W = 16 / sizeof(T);
  constexpr int PIECES = BN * 8 / THREADS, XP = BM * 16 / THREADS, LOADS = XP * sizeof(T) / 2;
  __shared__ __align__(1024) uint8_t la[BM * kBlock], lb[2][BN * kBlock];
  __shared__ uint8_t scales[BM];
  const int64_t M = p.a.rows, N = p.b.rows, K = p.K, m0 = (int64_t)blockIdx.x * BM;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN * 32, wn = wave % WN * 64, r16 = lane & 15, g = lane >> 4, key = r16 >> 1;
  const int nkb = (int)((K + kBlock - 1) / kBlock);
  const bool inside = m0 + BM <= M;

  // b's codes, as in k_fp8_product
  unsigned src[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int row = (i * THREADS + threadIdx.x) / 8, last = (int)N - 1;
    src[i] = (unsigned)(row < last ? row : last) * (unsigned)p.b.ldc;
  }
  const unsigned key_b = W == 4 ? threadIdx.x >> 4 & 7 : (threadIdx.x >> 4 & 1) | (threadIdx.x >> 6 & 3) << 1;
  const unsigned piece = 16 * ((threadIdx.x & 7) ^ key_b);
  auto load_b = [&](int kb) {
    const int64_t at = (int64_t)kb * kBlock;
    uint8_t* to = lb[kb & 1] + wave * 1024;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      if (at + piece < K) to_lds16(p.b.codes + at + (src[i] + piece), to + i * THREADS * 16);
      else *reinterpret_cast<uint4*>(to + i * THREADS * 16 + lane * 16) = make_uint4(0, 0, 0, 0);
    }
  };
  auto column = [](int row, int j) { return (row >> 2) * W + (row & 3) + j / (W / 4) * 4 * W + j % (W / 4) * 4; };
  const uint8_t* sb[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int n = wn + column(r16, j);
    sb[j] = p.b.scale + ((n < N ? n : N - 1) >> p.b.shift) * p.b.lds;
  }
  // rows of x: row xr + i THREADS / 16, values 8 xc ..
  const int xr = threadIdx.x >> 4, xc = threadIdx.x & 15;
  Eight<T> v[XP];
  auto load_x = [&](int kb) {
    const int64_t c = (int64_t)kb * kBlock + 8 * xc;
#pragma unroll
    for (int i = 0; i < XP; ++i) {
      const int64_t m = m0 + xr + i * (THREADS / 16);
      const T* q = x + m * ldx + c;
      if (inside && c + 8 <= K) v[i].load(q);
      else v[i].load_some(q, m < M ? K - c : 0);
    }
  };
  v4f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  if (nkb) {
    load_b(0);
    load_x(0);
  }
  for (int kb = 0; kb < nkb; ++kb) {
#pragma unroll
    for (int i = 0; i < XP; ++i) {
      using E = Eight<T>;
      const int row = xr + i * (THREADS / 16);
      unsigned big = E::below_sign(v[i].w[0]);
#pragma unroll
      for (int q = 1; q < E::NW; ++q) big = E::larger(big, E::below_sign(v[i].w[q]));
      const unsigned byte = scale_byte(rowmax_bits<16>(E::largest(big)));
      const float inv = scale_inverse(byte);
      const E& r = v[i];
      uint2 q;
      q.x = codes4(r.get(0) * inv, r.get(1) * inv, r.get(2) * inv, r.get(3) * inv);
      q.y = codes4(r.get(4) * inv, r.get(5) * inv, r.get(6) * inv, r.get(7) * inv);
      *reinterpret_cast<uint2*>(la + row * kBlock + ((xc >> 1) ^ (row >> 1 & 7)) * 16 + (xc & 1) * 8) = q;
      if (xc == 0) scales[row] = (uint8_t)byte;
    }
    unsigned ea[TM], eb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) eb[j] = sb[j][kb];
    const bool more = kb + 1 < nkb;
    if (more) load_x(kb + 1);
    // b's codes are there (the LOADS loads of x's rows after them may be under way;
    // others among them only lengthen the wait), and all have written theirs of a
    if (more && inside && (int64_t)(kb + 2) * kBlock <= K) wait_barrier<LOADS>();
    else wait_barrier<0>();
    if (more) load_b(kb + 1);
    v4i ra[TM][2];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      ea[i] = scales[wm + 16 * i + r16];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        ra[i][h] = *reinterpret_cast<const v4i*>(la + (wm + 16 * i + r16) * kBlock + ((g + 4 * h) ^ key) * 16);
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // x's codes are read
    auto half_b = [&](int j, int h) {
      return *reinterpret_cast<const v4i*>(lb[kb & 1] + (wn + column(r16, j)) * kBlock + ((g + 4 * h) ^ key) * 16);
    };
    if constexpr (EXACT) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v8b aw[TM][2];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const v4i q = ra[i][h];
          aw[i][0] = wide(make_uint2(q[0], q[1]), scale_value(ea[i]));
          aw[i][1] = wide(make_uint2(q[2], q[3]), scale_value(ea[i]));
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const v4i q = half_b(j, h);
          const v8b b0 = wide(make_uint2(q[0], q[1]), scale_value(eb[j])), b1 = wide(make_uint2(q[2], q[3]), scale_value(eb[j]));
#pragma unroll
          for (int i = 0; i < TM; ++i) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b0, aw[i][0], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b1, aw[i][1], acc[i][j], 0, 0, 0);
          }
        }
      }
    } else {
      v8i a[TM];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const v4i q = ra[i][0], r = ra[i][1];
        a[i] = v8i{q[0], q[1], q[2], q[3], r[0], r[1], r[2], r[3]};
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const v4i q = half_b(j, 0), r = half_b(j, 1);
        const v8i b = {q[0], q[1], q[2], q[3], r[0], r[1], r[2], r[3]};
#pragma unroll
        for (int i = 0; i < TM; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a[i], acc[i][j], 0, 0, 0, eb[j], 0, ea[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = m0 + wm + 16 * i + r16;
#pragma unroll
    for (int q = 0; q < 16 / W; ++q) {
      const int64_t n = wn + q * 4 * W + g * W;
      float t[W];
#pragma unroll
      for (int k = 0; k < W; ++k) t[k] = acc[i][(q * W + k) / 4][k % 4];
      if (m < M) put(static_cast<T*>(p.out) + m * p.ldo + n, t, N - n, false);
    }
  }
}

// The same where all of b's codes have room in LDS beside x's: 256 columns of up to
// 512 values. A block, one a compute unit, keeps them and walks the rows, 64 at a
// time; the values of a step are loaded for the block's next rows as soon as they are
// coded, a whole tile ahead, and a step waits for no load of codes. (397,934 rows of
// 512 to 256 take 133 us in bf16, 4.6 TB/s, and 180 in k_fp8_rows_product, 241 and 306
// in fp32.)
template <class T, bool EXACT>
__global__ void __launch_bounds__(512, 2) k_fp8_rows_resident(ProductArgs p, const T* __restrict__ x, int64_t ldx) {
  constexpr int BM = 64, BN = 256, WN = 4, THREADS = 512, TM = 2, TN = 4, W = 16 / sizeof(T), KB = 4, XP = 2;
  using E = Eight<T>;
  __shared__ __align__(1024) uint8_t lb[KB][BN * kBlock], la[2][BM * kBlock];
  __shared__ uint8_t scales[2][BM];
  const int64_t M = p.a.rows, N = p.b.rows, K = p.K, tiles = (M + BM - 1) / BM;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN * 32, wn = wave % WN * 64, r16 = lane & 15, g = lane >> 4, key = r16 >> 1;
  const int nkb = (int)((K + kBlock - 1) / kBlock);
  auto column = [](int row, int j) { return (row >> 2) * W + (row & 3) + j / (W / 4) * 4 * W + j % (W / 4) * 4; };
  {  // b's codes, as in k_fp8_product
    const unsigned key_b = W == 4 ? threadIdx.x >> 4 & 7 : (threadIdx.x >> 4 & 1) | (threadIdx.x >> 6 & 3) << 1;
    const unsigned piece = 16 * ((threadIdx.x & 7) ^ key_b);
    for (int kb = 0; kb < nkb; ++kb) {
      const int64_t at = (int64_t)kb * kBlock;
      uint8_t* to = lb[kb] + wave * 1024;
#pragma unroll
      for (int i = 0; i < BN * 8 / THREADS; ++i) {
        const int row = (i * THREADS + threadIdx.x) / 8, last = (int)N - 1;
        if (at + piece < K) to_lds16(p.b.codes + (int64_t)(row < last ? row : last) * p.b.ldc + at + piece, to + i * THREADS * 16);
        else *reinterpret_cast<uint4*>(to + i * THREADS * 16 + lane * 16) = make_uint4(0, 0, 0, 0);
      }
    }
  }
  // b's scales: a word has the bytes of the four blocks of K (there are none, and may be
  // no memory, where K = 0)
  unsigned eb[TN] = {};
  if (nkb) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = wn + column(r16, j);
      eb[j] = *reinterpret_cast<const unsigned*>(p.b.scale + ((n < N ? n : N - 1) >> p.b.shift) * p.b.lds);
    }
  }
  // rows of x: row xr + 32 i of a tile, values 8 xc .. of a block of K
  const int xr = threadIdx.x >> 4, xc = threadIdx.x & 15;
  E v[KB][XP];
  auto load_x = [&](int64_t tile, int kb, E (&v)[XP]) {
    const int64_t c = (int64_t)kb * kBlock + 8 * xc;
#pragma unroll
    for (int i = 0; i < XP; ++i) {
      const int64_t m = tile * BM + xr + i * (THREADS / 16);
      const T* q = x + m * ldx + c;
      if (m < M && c + 8 <= K) v[i].load(q);
      else v[i].load_some(q, m < M ? K - c : 0);
    }
  };
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
    if (kb < nkb) load_x(blockIdx.x, kb, v[kb]);
  wait_barrier<0>();  // b's codes are there
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    v4f acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    int step = 0;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if (kb >= nkb) break;
      // (the buffers take turns over the tiles' ends)
      const int buf = (int)((tile / gridDim.x * nkb + step++) & 1);
#pragma unroll
      for (int i = 0; i < XP; ++i) {
        const int row = xr + i * (THREADS / 16);
        const E& r = v[kb][i];
        unsigned big = E::below_sign(r.w[0]);
#pragma unroll
        for (int q = 1; q < E::NW; ++q) big = E::larger(big, E::below_sign(r.w[q]));
        const unsigned byte = scale_byte(rowmax_bits<16>(E::largest(big)));
        const float inv = scale_inverse(byte);
        uint2 q;
        q.x = codes4(r.get(0) * inv, r.get(1) * inv, r.get(2) * inv, r.get(3) * inv);
        q.y = codes4(r.get(4) * inv, r.get(5) * inv, r.get(6) * inv, r.get(7) * inv);
        *reinterpret_cast<uint2*>(la[buf] + row * kBlock + ((xc >> 1) ^ (row >> 1 & 7)) * 16 + (xc & 1) * 8) = q;
        if (xc == 0) scales[buf][row] = (uint8_t)byte;
      }
      if (tile + gridDim.x < tiles) load_x(tile + gridDim.x, kb, v[kb]);
      // x's codes are written (and those of the last step but one read by all)
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      unsigned ea[TM];
      v4i ra[TM][2];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        ea[i] = scales[buf][wm + 16 * i + r16];
#pragma unroll
        for (int h = 0; h < 2; ++h)
          ra[i][h] = *reinterpret_cast<const v4i*>(la[buf] + (wm + 16 * i + r16) * kBlock + ((g + 4 * h) ^ key) * 16);
      }
      auto half_b = [&](int j, int h) {
        return *reinterpret_cast<const v4i*>(lb[kb] + (wn + column(r16, j)) * kBlock + ((g + 4 * h) ^ key) * 16);
      };
      if constexpr (EXACT) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v8b aw[TM][2];
#pragma unroll
          for (int i = 0; i < TM; ++i) {
            aw[i][0] = wide(make_uint2(ra[i][h][0], ra[i][h][1]), scale_value(ea[i]));
            aw[i][1] = wide(make_uint2(ra[i][h][2], ra[i][h][3]), scale_value(ea[i]));
          }
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            const v4i q = half_b(j, h);
            const float f = scale_value(eb[j] >> (8 * kb));
            const v8b b0 = wide(make_uint2(q[0], q[1]), f), b1 = wide(make_uint2(q[2], q[3]), f);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b0, aw[i][0], acc[i][j], 0, 0, 0);
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b1, aw[i][1], acc[i][j], 0, 0, 0);
            }
          }
        }
      } else {
        v8i a[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const v4i q = ra[i][0], r = ra[i][1];
          a[i] = v8i{q[0], q[1], q[2], q[3], r[0], r[1], r[2], r[3]};
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const v4i q = half_b(j, 0), r = half_b(j, 1);
          const v8i b = {q[0], q[1], q[2], q[3], r[0], r[1], r[2], r[3]};
#pragma unroll
          for (int i = 0; i < TM; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a[i], acc[i][j], 0, 0, 0, eb[j] >> (8 * kb), 0, ea[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = tile * BM + wm + 16 * i + r16;
#pragma unroll
      for (int q = 0; q < 16 / W; ++q) {
        const int64_t n = wn + q * 4 * W + g * W;
        float t[W];
#pragma unroll
        for (int k = 0; k < W; ++k) t[k] = acc[i][(q * W + k) / 4][k % 4];
        if (m < M) put(static_cast<T*>(p.out) + m * p.ldo + n, t, N - n, false);
      }
    }
  }
}

// out (+)= the sum of the splits' parts, in order; a thread has four columns
template <class T>
__global__ void __launch_bounds__(256) k_fp8_join(int64_t M, int64_t N, int splits, const float* __restrict__ part,
                                                  int64_t ldp, T* __restrict__ out, int64_t ldo, int add) {
  const int64_t quads = ldp / 4, stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * quads; i += stride) {
    const int64_t m = i / quads, n = 4 * (i - m * quads);
    const float* p = part + m * ldp + n;
    float s[4];
    load_v<4>(p, s);
#pragma unroll 4
    for (int k = 1; k < splits; ++k) {
      float t[4];
      load_v<4>(p + (int64_t)k * M * ldp, t);
#pragma unroll
      for (int c = 0; c < 4; ++c) s[c] += t[c];
    }
    put(out + m * ldo + n, s, N - n, add != 0);
  }
}

int bad(const char* who, const char* what) { return fail(CHGNET_EINVAL, std::string(who) + ": " + what); }

// Shape of one quantised matrix; pointers only where `there`
int check_factor(const char* who, const chgnet_fp8* f, bool there) {
  if (!f) return bad(who, "a matrix is NULL");
  if (f->rows < 0 || f->rows >= kMostRows) return bad(who, "rows must be in 0 .. 2^31 - 1");
  if (f->cols < 0 || f->cols > kMostK) return bad(who, "columns must be in 0 .. 2^23");
  if (f->block_rows != 1 && f->block_rows != kBlock) return bad(who, "block_rows must be 1 or 128");
  if (f->ld < cdiv(f->cols, 16) * 16 || f->ld % 16 || f->ld > kMostK)
    return bad(who, "ld must be a multiple of 16 that holds the columns, at most 2^23");
  if (f->ld_scale < cdiv(f->cols, kBlock) || f->ld_scale % 4 || f->ld_scale > kMostK)
    return bad(who, "ld_scale must be a multiple of 4 that holds a byte for each 128 columns, at most 2^23");
  if (there && f->cols > 0 && (!f->codes || !f->scale)) return bad(who, "null argument");
  if (!aligned_to(f->codes, 16) || !aligned_to(f->scale, 4)) return bad(who, "codes must be 16-byte, scale 4-byte aligned");
  return CHGNET_OK;
}
Factor factor(const chgnet_fp8* f) {
  return {f->codes, f->scale, f->ld, f->ld_scale, f->rows, f->block_rows == kBlock ? 7 : 0};
}

constexpr int64_t kFewRows = 16, kUnits = 256;  // (compute units)

struct Plan {
  int tile;  // of tile x tile results; 0: few rows
  int64_t tiles;
  int splits, kb_split;
};
// The tiles: the largest of which there is one for each compute unit, where K may
// be divided into parts of kLeastSteps blocks or more. 256 x 512 x 397,934 takes
// 135 us in 2 tiles of 256 x 128 parts, 158 in 8 of 128 x 32, 204 in 32 of 64 x
// 16; 512 x 4,096 x 4,096 21 us in 512 tiles of 64, 28 in 128 of 128, 25 in twice
// as many halves; 128 x 8,192 x 8,192 26 us in 256 tiles of 64 and two parts, 31 in one,
// 34 in 64 of 128 and two.
constexpr int64_t kLeastSteps = 24;
// The smallest tiles, where there are fewer than compute units, take parts of 8
// blocks (a linear layer of 1,938 rows of 8,192 to 128 in bf16 30 us with its 62 tiles
// in 2 parts, 24 in 8).
constexpr int64_t kLeastSmallSteps = 8;
Plan plan(int64_t M, int64_t N, int64_t K) {
  const int64_t nkb = std::max<int64_t>(1, cdiv(K, kBlock));
  if (M <= kFewRows) return {0, 0, 1, (int)nkb};
  auto tiles = [&](int t) { return cdiv(M, t) * cdiv(N, t); };
  int64_t most = std::max<int64_t>(1, nkb / kLeastSteps);
  const int tile = tiles(256) * most >= kUnits ? 256 : tiles(128) * most >= kUnits ? 128 : 64;
  if (tile == 64) most = std::max<int64_t>(1, nkb / kLeastSmallSteps);
  const int64_t n = tiles(tile), want = tile == 64 ? 2 * kUnits / n : cdiv(kUnits, n);
  const int64_t s = std::max<int64_t>(1, std::min(want, most));
  const int64_t per = cdiv(cdiv(nkb, s), 4) * 4;  // (of whole words of scales)
  return {tile, n, (int)cdiv(nkb, per), (int)per};
}

// Columns of a block: twice as many where that leaves a block for each compute unit
// (16 rows of 8,192 to 8,192 in bf16: 33 us in blocks of 16 columns, 23 of 32, 26 of
// 64; one row of 4,096 to 4,096: 7.6, 8.6, 12). A launch has fewer than 2^32 threads (of
// more the runtime starts the number modulo 2^32, without an error): more columns than
// kLaunchCols, whole blocks of 128, are taken in turn.
constexpr int64_t kLaunchCols = 1 << 26;
template <class T, bool QUANT>
int launch_few(const ProductArgs& p, const T* x, int64_t ldx, hipStream_t st) {
  constexpr bool exact = std::is_same<T, float>::value;
  auto launch = [&](auto nt) -> int {
    for (int64_t n = 0; n < p.b.rows; n += kLaunchCols) {
      ProductArgs q = p;
      q.b.codes += n * p.b.ldc;
      q.b.scale += (n >> p.b.shift) * p.b.lds;
      q.b.rows = std::min(kLaunchCols, p.b.rows - n);
      q.out = static_cast<T*>(p.out) + n;
      KLAUNCH(st, "k_fp8_few", k_fp8_few<T, exact, QUANT, nt.value>
                               <<<(unsigned)cdiv(q.b.rows, 16 * nt.value), 512, 0, st>>>(q, x, ldx));
    }
    return CHGNET_OK;
  };
  if (p.b.rows >= 32 * kUnits) return launch(std::integral_constant<int, 2>{});
  return launch(std::integral_constant<int, 1>{});
}

// Whether a linear layer quantises its rows on the way: where each is needed once
// and the blocks fill the GPU (us of a call against quantiser and product, bf16: 397,934
// rows of 512 to 256 133 and 227, to 128 116 and 211, 85,274 of 256 to 128 19 and 32; fp32 rows
// 241 and 393, 192 and 353, 27 and 48; 5,000 of 512 to 256 9 and 10, in fp32 12 and 12)
bool on_the_way(int64_t M, int64_t N) { return N <= 256 && cdiv(M, 64) >= kUnits; }
template <class T>
int launch_rows_product(const ProductArgs& p, const T* x, int64_t ldx, hipStream_t st) {
  constexpr bool exact = std::is_same<T, float>::value;
  const unsigned blocks = (unsigned)cdiv(p.a.rows, 64);
  if (p.b.rows > 128 && p.K <= 4 * kBlock)
    KLAUNCH(st, "k_fp8_rows_resident",
            k_fp8_rows_resident<T, exact><<<(unsigned)std::min<int64_t>(blocks, kUnits), 512, 0, st>>>(p, x, ldx));
  else if (p.b.rows <= 128)
    KLAUNCH(st, "k_fp8_rows_product", k_fp8_rows_product<T, exact, 128><<<blocks, 256, 0, st>>>(p, x, ldx));
  else
    KLAUNCH(st, "k_fp8_rows_product", k_fp8_rows_product<T, exact, 256><<<blocks, 512, 0, st>>>(p, x, ldx));
  return CHGNET_OK;
}

int64_t part_ld(int64_t N) { return cdiv(N, 4) * 4; }

}  // namespace

int fp8_quantize_entry(int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t ldx, const chgnet_fp8* q,
                       const chgnet_fp8* t, hipStream_t st) {
  const char* who = "fp8_quantize";
  if (rows < 0 || rows > kMostK || cols < 0 || cols > kMostK) return bad(who, "rows and columns must be in 0 .. 2^23");
  if (!elem_size(dtype)) return bad(who, "unknown dtype");
  if (ldx < cols) return bad(who, "a row stride is below the row's width");
  if (!q && !t) return bad(who, "neither codes nor those of the transpose are asked for");
  if (q) {
    CHG_TRY(check_factor(who, q, rows > 0));
    if (q->rows != rows || q->cols != cols) return bad(who, "the codes are of another shape");
  }
  if (t) {
    CHG_TRY(check_factor(who, t, cols > 0));
    if (t->rows != cols || t->cols != rows) return bad(who, "the transposed codes are of another shape");
  }
  if (q && t && q->block_rows != t->block_rows) return bad(who, "both forms have the same block_rows");
  if (rows == 0 || cols == 0) return CHGNET_OK;
  const size_t es = elem_size(dtype);
  if (!x) return bad(who, "null argument");
  if (!aligned_to(x, es)) return bad(who, "x is not aligned to its values");
  const bool square = (q ? q : t)->block_rows == kBlock;
  return with_type(dtype, [&](auto v) -> int {
    using T = decltype(v);
    const T* p = static_cast<const T*>(x);
    if (!square && !t) {
      const unsigned blocks = (unsigned)std::min<int64_t>(4096, cdiv(rows * cdiv(cols, kBlock), 16));
KLAUNCH(st, "k_fp8_rows",
              k_fp8_rows<T><<<blocks, 256, 0, st>>>(rows, cols, p, ldx, q->codes, q->ld, q->scale, q->ld_scale));
      return CHGNET_OK;
    }
    // four tiles a block only where that leaves four blocks for each compute unit (4,096 x
    // 4,096 in bf16, both forms: 16 us in blocks of one tile, 23 of four)
    const int count = cdiv(rows, 512) * cdiv(cols, 128) >= 4 * kUnits ? 4 : 1;
    const int64_t tiles = cdiv(rows, 128 * count) * cdiv(cols, 128);
    // (a launch has fewer than 2^32 threads, and the runtime does not say so)
    if (tiles >= (int64_t(1) << 24)) return bad(who, "more than 2^40 values");
    const chgnet_fp8 none{}, &a = q ? *q : none, &b = t ? *t : none;
#define CHG_TILE(S)                                                                                                     \
  KLAUNCH(st, "k_fp8_tile", k_fp8_tile<T, S><<<(unsigned)tiles, 256, 0, st>>>(                                          \
                                rows, cols, p, ldx, a.codes, a.ld, a.scale, a.ld_scale, b.codes, b.ld, b.scale, b.ld_scale, \
                                count))
    if (square) CHG_TILE(true);
    else CHG_TILE(false);
#undef CHG_TILE
    return CHGNET_OK;
  });
}

int fp8_matmul_workspace_entry(int64_t M, int64_t N, int64_t K, size_t* bytes) {
  const char* who = "fp8_matmul_workspace";
  if (M < 0 || N < 0 || M >= kMostRows || N >= kMostRows || K < 0 || K > kMostK) return bad(who, "sizes out of range");
  if (!bytes) return bad(who, "bytes is NULL");
  *bytes = 0;
  if (M == 0 || N == 0) return CHGNET_OK;
  const Plan pl = plan(M, N, K);
  if (pl.splits > 1) *bytes = sizeof(float) * (size_t)pl.splits * (size_t)M * (size_t)part_ld(N);
  return CHGNET_OK;
}

int fp8_matmul_entry(const chgnet_fp8* a, const chgnet_fp8* b, int32_t dtype, void* out, int64_t ldout, int accumulate,
                     void* ws, size_t ws_bytes, hipStream_t st) {
  const char* who = "fp8_matmul";
  CHG_TRY(check_factor(who, a, a && a->rows > 0));
  CHG_TRY(check_factor(who, b, b && b->rows > 0));
  if (a->cols != b->cols) return bad(who, "the factors have different numbers of columns");
  if (!elem_size(dtype)) return bad(who, "unknown dtype");
  const int64_t M = a->rows, N = b->rows, K = a->cols;
  if (ldout < N) return bad(who, "a row stride is below the row's width");
  if (M == 0 || N == 0) return CHGNET_OK;
  if (!out) return bad(who, "null argument");
  if (!aligned_to(out, elem_size(dtype))) return bad(who, "out is not aligned to its values");
  size_t need = 0;
  CHG_TRY(fp8_matmul_workspace_entry(M, N, K, &need));
  if (need && (!ws || ws_bytes < need))
    return fail(CHGNET_EWORKSPACE, std::string(who) + ": workspace too small (query chgnet_fp8_matmul_workspace)");
  if (!aligned_to(ws, 16)) return bad(who, "ws is not 16-byte aligned");
  const Plan pl = plan(M, N, K);
  ProductArgs p{factor(a), factor(b), K, out, ldout, pl.splits > 1 ? static_cast<float*>(ws) : nullptr, part_ld(N),
                pl.splits, pl.kb_split, accumulate != 0};
  return with_type(dtype, [&](auto v) -> int {
    using T = decltype(v);
    constexpr bool exact = std::is_same<T, float>::value;
    if (pl.tile == 0) {
      return launch_few<T, false>(p, nullptr, 0, st);
    }
    auto launch = [&](auto part) -> int {
      using P = decltype(part);
      // as many blocks as have room at a time
      auto blocks = [&](int64_t a_unit) { return (unsigned)std::min<int64_t>(pl.tiles * pl.splits, a_unit * kUnits); };
      if (pl.tile == 256)
        KLAUNCH(st, "k_fp8_product", k_fp8_product<P, exact, 256, 256, 2, 4, 2><<<blocks(1), 512, 0, st>>>(p));
      else if (pl.tile == 128)
        KLAUNCH(st, "k_fp8_product", k_fp8_product<P, exact, 128, 128, 2, 2, 2><<<blocks(2), 256, 0, st>>>(p));
      else
        KLAUNCH(st, "k_fp8_product", k_fp8_product<P, exact, 64, 64, 4, 1, 4><<<blocks(2), 256, 0, st>>>(p));
      return CHGNET_OK;
    };
    if (pl.splits == 1) return launch(T{});
    CHG_TRY(launch(float{}));
    KLAUNCH(st, "k_fp8_join", k_fp8_join<T><<<(unsigned)std::min<int64_t>(2048, cdiv(M * part_ld(N) / 4, 256)), 256, 0, st>>>(
                                  M, N, pl.splits, p.part, p.ldp, static_cast<T*>(out), ldout, p.add));
    return CHGNET_OK;
  });
}

// Layout of a linear layer's workspace: codes and scales of x, the product's own
struct LinearWs {
  chgnet_fp8 q;
  size_t product, total;
};
static LinearWs linear_ws(int64_t M, int64_t K, size_t product, void* ws) {
  LinearWs w{};
  w.q.rows = M, w.q.cols = K, w.q.block_rows = 1;
  w.q.ld = K <= kBlock ? cdiv(K, 16) * 16 : cdiv(K, kBlock) * kBlock, w.q.ld_scale = cdiv(cdiv(K, kBlock), 4) * 4;
  const size_t codes = align_up((size_t)M * w.q.ld, 256), scale = align_up((size_t)M * w.q.ld_scale, 256);
  w.q.codes = static_cast<uint8_t*>(ws);
  w.q.scale = static_cast<uint8_t*>(ws) + codes;
  w.product = codes + scale;
  w.total = w.product + product;
  return w;
}

int fp8_linear_workspace_entry(int64_t M, int64_t N, int64_t K, size_t* bytes) {
  size_t product = 0;
  CHG_TRY(fp8_matmul_workspace_entry(M, N, K, &product));
  if (!bytes) return bad("fp8_linear_workspace", "bytes is NULL");
  *bytes = M > kFewRows && N && K && !on_the_way(M, N) ? linear_ws(M, K, product, nullptr).total : 0;
  return CHGNET_OK;
}

int fp8_linear_entry(int64_t rows, int32_t dtype, const void* x, int64_t ldx, const chgnet_fp8* w, void* out, int64_t ldout,
                     void* ws, size_t ws_bytes, hipStream_t st) {
  const char* who = "fp8_linear";
  if (rows < 0 || rows > kMostK) return bad(who, "rows must be in 0 .. 2^23");
  if (!elem_size(dtype)) return bad(who, "unknown dtype");
  CHG_TRY(check_factor(who, w, w && w->rows > 0));
  if (ldx < w->cols || ldout < w->rows) return bad(who, "a row stride is below the row's width");
  if (rows == 0 || w->rows == 0) return CHGNET_OK;
  const size_t es = elem_size(dtype);
  if (!out || (!x && w->cols)) return bad(who, "null argument");
  if (!aligned_to(x, es) || !aligned_to(out, es)) return bad(who, "an array is not aligned to its values");
  if (rows <= kFewRows || on_the_way(rows, w->rows)) {
    ProductArgs p{};
    p.a.rows = rows, p.b = factor(w), p.K = w->cols, p.out = out, p.ldo = ldout;
    return with_type(dtype, [&](auto v) -> int {
      using T = decltype(v);
      const T* t = static_cast<const T*>(x);
      return rows > kFewRows ? launch_rows_product<T>(p, t, ldx, st) : launch_few<T, true>(p, t, ldx, st);
    });
  }
  size_t product = 0;
  CHG_TRY(fp8_matmul_workspace_entry(rows, w->rows, w->cols, &product));
  const LinearWs l = linear_ws(rows, w->cols, product, ws);
  if (w->cols && (!ws || ws_bytes < l.total))
    return fail(CHGNET_EWORKSPACE, "fp8_linear: workspace too small (query chgnet_fp8_linear_workspace)");
  if (!aligned_to(ws, 16)) return bad(who, "ws is not 16-byte aligned");
  CHG_TRY(fp8_quantize_entry(rows, w->cols, dtype, x, ldx, &l.q, nullptr, st));
  return fp8_matmul_entry(&l.q, w, dtype, out, ldout, 0, static_cast<uint8_t*>(ws) + l.product, product, st);
}

}  // namespace chg
