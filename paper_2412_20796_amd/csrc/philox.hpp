// Dropout's mask: which values of a [rows, columns] array a call keeps, from
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as
// 1, 2, 3, SC 2011). A value's bits depend on the seed, the call's number, its
// row and its column only, so that a backward pass forms the mask again and it
// is the same in every layout, type and launch.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

namespace chg {

// What a kernel needs of a dropout: values whose 16 bits are below `cut` are
// dropped (65,536: all), the others multiplied by `scale` = 1 / (1 - cut / 65,536).
// 16 bits a value and not 32: half the generator's multiplications, which at 32
// would take as long as the memory does for 16-bit values; p is off by at most
// 2^-17, and the scale is that of the p that is taken.
struct Drop {
  uint32_t cut;
  float scale;
  uint64_t seed, call;
  const int64_t* step;  // added to `call` (a replayed graph's next number); may be NULL
};
inline Drop make_drop(float p, uint64_t seed, uint64_t call, const int64_t* step) {
  const uint32_t cut = (uint32_t)std::floor((double)p * 65536.0 + 0.5);
  return {cut, cut < 65536 ? (float)(65536.0 / (65536 - cut)) : 0.f, seed, call, step};
}

struct Philox {
  uint32_t k0, k1, c2, c3;
  __device__ __forceinline__ explicit Philox(const Drop& d) {
    const uint64_t call = d.call + (d.step ? (uint64_t)*d.step : 0);
    k0 = (uint32_t)d.seed;
    k1 = (uint32_t)(d.seed >> 32);
    c2 = (uint32_t)call;
    c3 = (uint32_t)(call >> 32);
  }
  // the 16 bits of each of the columns 8 group .. 8 group + 7 of a row: two a
  // word, the lower column in the low half
  __device__ __forceinline__ void words(uint32_t row, uint32_t group, uint32_t (&w)[4]) const {
    uint32_t a0 = group, a1 = row, a2 = c2, a3 = c3, q0 = k0, q1 = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t p = (uint64_t)a0 * 0xD2511F53u, q = (uint64_t)a2 * 0xCD9E8D57u;
      a0 = (uint32_t)(q >> 32) ^ a1 ^ q0;
      a1 = (uint32_t)q;
      a2 = (uint32_t)(p >> 32) ^ a3 ^ q1;
      a3 = (uint32_t)p;
      q0 += 0x9E3779B9u;
      q1 += 0xBB67AE85u;
    }
    w[0] = a0;
    w[1] = a1;
    w[2] = a2;
    w[3] = a3;
  }
  // whether the upper (lower) 16 bits of a word are at least `cut`: one comparison
  // each (a cut of 65,536 is above both)
  static __device__ __forceinline__ bool upper(uint32_t w, uint32_t cut) { return cut <= 65535u && w >= cut << 16; }
  static __device__ __forceinline__ bool lower(uint32_t w, uint32_t cut) {
    return cut <= 65535u && (uint16_t)w >= (uint16_t)cut;
  }
  // bit k: column 8 group + k is kept
  __device__ __forceinline__ uint32_t mask8(uint32_t row, uint32_t group, uint32_t cut) const {
    uint32_t w[4], m = 0;
    words(row, group, w);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m |= (uint32_t)lower(w[k], cut) << (2 * k);
      m |= (uint32_t)upper(w[k], cut) << (2 * k + 1);
    }
    return m;
  }
};

}  // namespace chg
