// Embedding lookup with a scale, and its gradient by sorted tokens
// (chgnet_ops.h).
//
//   out_i = scale W[tok_i - first]       dW_v (+)= scale sum_{tok_i - first = v} dout_i
//
// The lookup is a copy, bound by memory. The gradient reads every row of dout
// once and writes every row of dW once; what it must not do is depend on how
// the tokens are spread, from a table of which most rows have no token to an
// element that is every second atom. So the positions are ordered by token
// first (stably, so that the sums have one order), the ordered positions are
// cut into chunks of equal length, each summed by one group of lanes run by
// run, and the runs that cross a chunk's end are joined from the chunks' partial
// sums, in order. Few tokens skip the ordering: a block finds the tokens of its
// table row by looking at all of them.
//
// Measured, 1,000,003 tokens of 94 rows of 128 in fp32 (a third of them on one
// row): counts 5.6 us, places 17.3, sums 87 (512 MB, 5.9 TB/s), joins 5.9;
// 262,144 tokens of 50,000 rows of 512 in bf16: two passes of 4.8 and 11.1 us,
// sums and zeros 77 (242 MB read, 102 MB written, 4.5 TB/s), joins 6.5. The
// ordering is bound by latency (a pass reads and writes 16 bytes a token), the
// sums by memory.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.hpp"
#include "elem.hpp"

namespace chg {
namespace {

// Table row of a token; `vocab` for a token of no row.
__device__ __forceinline__ int table_row(int tok, int first, int vocab) {
  const int64_t r = (int64_t)tok - first;
  return r >= 0 && r < vocab ? (int)r : vocab;
}

// ---------------------------------------------------------------------------
// Lookup: LPR lanes a row, VEC values a lane and pass; a group of lanes takes
// kFwdRows rows at a time, so that as many loads are in flight. The results go
// past the caches, which keep the table: 83 -> 50 us for 524,288 rows of 256 in
// 16 bits of a table of 50,000.
// ---------------------------------------------------------------------------
constexpr int kFwdRows = 4;

template <class T, int VEC, int LPR>
__global__ void __launch_bounds__(256) k_embed_fwd(int64_t n, int d, int vocab, const int* __restrict__ tok, int first,
                                                   const T* __restrict__ table, int64_t ldt, float scale,
                                                   T* __restrict__ out, int64_t ldo) {
  constexpr int G = 256 / LPR;
  const int j = threadIdx.x % LPR;
  const int g = LPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / LPR) : threadIdx.x / LPR;
  const int64_t stride = (int64_t)gridDim.x * G * kFwdRows;
  int64_t i0 = ((int64_t)blockIdx.x * G + g) * kFwdRows;
  int next[kFwdRows];  // the next rows' tokens, loaded a turn ahead
  auto load_tokens = [&](int64_t i) {
#pragma unroll
    for (int u = 0; u < kFwdRows; ++u) next[u] = i + u < n ? tok[i + u] : -1;
  };
  load_tokens(i0);
  for (; i0 < n; i0 += stride) {
    int r[kFwdRows];
#pragma unroll
    for (int u = 0; u < kFwdRows; ++u) r[u] = table_row(next[u], first, vocab);
    load_tokens(i0 + stride);
    for (int c = j * VEC; c < d; c += LPR * VEC) {
      float v[kFwdRows][VEC];
#pragma unroll
      for (int u = 0; u < kFwdRows; ++u) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[u][k] = 0.f;
        if (r[u] < vocab) load_v<VEC>(table + r[u] * ldt + c, v[u]);
      }
#pragma unroll
      for (int u = 0; u < kFwdRows; ++u) {
        if (i0 + u >= n) break;
        if (r[u] < vocab)
#pragma unroll
          for (int k = 0; k < VEC; ++k) v[u][k] *= scale;
        store_nt<VEC>(out + (i0 + u) * ldo + c, v[u]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Ordering of the positions by table row: passes over digits of at most 8 bits,
// least significant first, each stable. A pass is two launches over at most
// kSortBlocks blocks, each with a contiguous stretch of the tokens: the counts of
// every digit in every stretch, then the places. A block of the second launch
// adds up the counts of the stretches before its own and of the lower digits
// itself (at most 256 x 256 numbers, in L2), so that no scan stands between the
// two.
// ---------------------------------------------------------------------------
constexpr int kSortBlocks = 256, kSortThreads = 1024, kDigits = 256;

struct SortPass {
  int n, vocab, first;
  int shift, bits;          // the pass's digit of the row
  int64_t len;              // tokens of a block's stretch, a multiple of kSortThreads
  const int* tok;           // first pass: the tokens
  const int *row, *pos;     // later passes: rows and positions in the order so far
  int *row_out, *pos_out;
  int* counts;              // [gridDim.x][kDigits]
};

__device__ __forceinline__ int sort_row(const SortPass& s, int i) {
  return s.tok ? table_row(s.tok[i], s.first, s.vocab) : s.row[i];
}

// lanes of the wavefront with the same digit (of `bits` bits) as this one
__device__ __forceinline__ unsigned long long same_digit(int digit, int bits, bool valid) {
  unsigned long long m = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long w = __ballot((digit >> b) & 1);
    m &= (digit >> b) & 1 ? w : ~w;
  }
  return m;
}

__global__ void __launch_bounds__(kSortThreads) k_embed_count(SortPass s) {
  __shared__ int cnt[kDigits];
  const int t = threadIdx.x;
  if (t < kDigits) cnt[t] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * s.len, i1 = min(i0 + s.len, (int64_t)s.n);
  for (int64_t base = i0; base < i1; base += kSortThreads) {
    const int64_t i = base + t;
    const bool valid = i < i1;
    const int digit = valid ? (sort_row(s, (int)i) >> s.shift) & ((1 << s.bits) - 1) : 0;
    const unsigned long long m = same_digit(digit, s.bits, valid);
    if (valid && __ffsll(m) - 1 == (t & 63)) atomicAdd(&cnt[digit], __popcll(m));  // integers: no order shows
  }
  __syncthreads();
  if (t < kDigits) s.counts[blockIdx.x * kDigits + t] = cnt[t];
}

template <int kRounds>
__global__ void __launch_bounds__(kSortThreads) k_embed_place(SortPass s) {
  const int mask = (1 << s.bits) - 1;
  constexpr int W = kSortThreads / 64;
  __shared__ int place[kDigits];     // next place of each digit
  __shared__ int wcnt[W][kDigits];   // counts, then first places, of each wavefront's digits
  __shared__ int total[kDigits];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, nb = gridDim.x;
  {
    // four threads a digit, each a quarter of the stretches
    const int digit = t & (kDigits - 1), q = t / kDigits;
    int before = 0, all = 0;
    const int b1 = nb * (q + 1) / 4;
    for (int b0 = nb * q / 4; b0 < b1; b0 += 32) {
      int c[32];  // loads in flight together: one at a time the launch took 30 us of 1,000,003 tokens
#pragma unroll
      for (int u = 0; u < 32; ++u) c[u] = b0 + u < b1 ? s.counts[(b0 + u) * kDigits + digit] : 0;
#pragma unroll
      for (int u = 0; u < 32; ++u) {
        before += b0 + u < (int)blockIdx.x ? c[u] : 0;
        all += c[u];
      }
    }
    wcnt[q][digit] = before;
    wcnt[4 + q][digit] = all;
  }
  __syncthreads();
  if (t < kDigits) total[t] = wcnt[4][t] + wcnt[5][t] + wcnt[6][t] + wcnt[7][t];
  __syncthreads();
  if (wave == 0) {
    // exclusive scan of the digits' totals, four a lane
    int c[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c[k] = total[4 * lane + k];
      sum += c[k];
    }
    int incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int v = __shfl_up(incl, off);
      if (lane >= off) incl += v;
    }
    int at = incl - sum;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int x = 4 * lane + k;
      place[x] = at + wcnt[0][x] + wcnt[1][x] + wcnt[2][x] + wcnt[3][x];
      at += c[k];
    }
  }
  // kRounds tokens a thread and turn: a wavefront takes kRounds x 64 consecutive
  // tokens in rounds of 64 and counts its digits as it goes, so that the block
  // meets three times for all of them
  const int64_t i0 = (int64_t)blockIdx.x * s.len, i1 = min(i0 + s.len, (int64_t)s.n);
  for (int64_t base = i0; base < i1; base += kSortThreads * kRounds) {
    __syncthreads();
    for (int k = t; k < W * kDigits; k += kSortThreads) (&wcnt[0][0])[k] = 0;
    __syncthreads();
    int row[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int64_t i = base + (wave * kRounds + r) * 64 + lane;
      row[r] = i < i1 ? sort_row(s, (int)i) : -1;
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const bool valid = row[r] >= 0;
      const int digit = (row[r] >> s.shift) & mask;
      const unsigned long long m = same_digit(digit, s.bits, valid);
      const int before = __popcll(m & ((1ull << lane) - 1));
      rank[r] = before + wcnt[wave][digit];
      // (a wavefront's LDS accesses stay in order)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (valid && before == 0) wcnt[wave][digit] += __popcll(m);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    if (t < kDigits) {
      int at = place[t];
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const int c = wcnt[w][t];
        wcnt[w][t] = at;
        at += c;
      }
      place[t] = at;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (row[r] < 0) continue;
      const int i = (int)base + (wave * kRounds + r) * 64 + lane;
      const int to = wcnt[wave][(row[r] >> s.shift) & mask] + rank[r];
      s.row_out[to] = row[r];
      s.pos_out[to] = s.tok ? i : s.pos[i];
    }
  }
}

// ---------------------------------------------------------------------------
// Sums of the ordered rows. Groups of LPR lanes (VEC NQ values a lane; the
// launch's y blocks take further columns) each add the rows of one chunk, eight
// loads in flight, and write a run's sum when it ends. A run that began in an
// earlier chunk or goes on in the next is a partial sum in LDS instead: slot 0 of
// the chunk for a run that began before it, slot 1 for one that begins in it and
// goes on. The block then joins its chunks' partial sums in order, and what
// crosses the block's stretch is one partial row of slot 0 and one of slot 1 in
// the workspace. FAR: the rows, each read once, are loaded past the caches
// (1,000,003 rows of 128 in fp32: 126 -> 114 us the whole gradient). The launch's
// first `nzero` blocks look up 512 table rows each among the ordered ones and
// write the zeros of those that no token has.
// ---------------------------------------------------------------------------
struct RunSums {
  int n, vocab, chunk, stretch, nstretch, d;  // stretch: positions of a block
  const int *row, *pos;
  int64_t ldo, ldw;
  float scale;
  float* dw;
  int add;
  float* part;  // [nstretch][2][d]
  int nzero;
};
constexpr int kRunThreads = 512;

constexpr int kZeroRows = kRunThreads;

// zeros in the rows v0 .. v0 + kZeroRows - 1 without a token, columns [col0, col1)
template <int VEC>
__device__ __forceinline__ void zero_rows(const RunSums& s, int64_t v0, int col0, int col1) {
  __shared__ int none[kZeroRows];
  const int t = threadIdx.x, lane = t & 63;
  const int64_t v = v0 + t;
  if (t < kZeroRows && v < s.vocab) {
    int lo = -1, hi = s.n;  // first position whose row is v or later: hi
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (s.row[mid] < v) lo = mid;
      else hi = mid;
    }
    none[t] = hi == s.n || s.row[hi] != v;
  }
  __syncthreads();
  const int rows = (int)min((int64_t)kZeroRows, s.vocab - v0);
  for (int r = t >> 6; r < rows; r += kRunThreads / 64) {
    if (!none[r]) continue;
    float* w = s.dw + (v0 + r) * s.ldw;
    const float zero[VEC] = {};
    for (int c = col0 + lane * VEC; c < col1; c += 64 * VEC) store_v<VEC>(w + c, zero);
  }
}

template <class T, int VEC, int LPR, int NQ, bool FAR>
__global__ void __launch_bounds__(kRunThreads) k_embed_runs(RunSums s, const int* __restrict__ rows,
                                                            const int* __restrict__ poss, const T* __restrict__ dout) {
  constexpr int G = kRunThreads / LPR, U = 8, CPL = VEC * NQ, C = LPR * CPL;
  __shared__ float part[G][2][C];
  __shared__ int first[G], kind[G];  // kind bits: 1 slot 0 used, 2 slot 1 used, 4 slot 0's run goes on
  // (a wavefront on one row: its chunk is uniform, so indices, comparisons and
  // addresses are scalar)
  const int j = threadIdx.x % LPR;
  const int g = LPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / LPR) : threadIdx.x / LPR;
  const int col0 = blockIdx.y * C;
  const int blk = (int)blockIdx.x - s.nzero;
  if (blk < 0) {
    zero_rows<VEC < 4 ? VEC : 4>(s, (int64_t)blockIdx.x * kZeroRows, col0, min(col0 + C, s.d));
    return;
  }
  const int b0 = blk * s.stretch, b1 = min(b0 + s.stretch, s.n);
  const int p0 = b0 + g * s.chunk, p1 = min(p0 + s.chunk, b1);
  auto column = [&](int q) { return (q * LPR + j) * VEC; };  // within the block's columns
  if (j == 0) kind[g] = 0;
  if (p0 < p1) {
    float acc[CPL];
#pragma unroll
    for (int k = 0; k < CPL; ++k) acc[k] = 0.f;
    int cur = rows[p0];
    if (j == 0) first[g] = cur;
    bool began = p0 == 0 || rows[p0 - 1] != cur;  // the run starts in this chunk
    auto keep = [&](int slot) {
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int k = 0; k < VEC; ++k) part[g][slot][column(q) + k] = acc[q * VEC + k];
    };
    auto flush = [&]() {
      if (cur >= s.vocab) return;
      if (!began) {
        keep(0);
        if (j == 0) kind[g] = 1;
        return;
      }
      float* w = s.dw + cur * s.ldw + col0;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        if (col0 + column(q) >= s.d) continue;
        float v[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = acc[q * VEC + k] * s.scale;
        if (s.add) {
          float o[VEC];
          load_v<VEC>(w + column(q), o);
#pragma unroll
          for (int k = 0; k < VEC; ++k) v[k] += o[k];
        }
        store_v<VEC>(w + column(q), v);
      }
    };
    int nr[U], no[U];  // the next step's rows and positions, loaded a step ahead
    auto load_index = [&](int p) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = min(p + u, p1 - 1);
        nr[u] = rows[x];
        no[u] = poss[x];
      }
    };
    load_index(p0);
    for (int p = p0; p < p1; p += U) {
      int r[U], o[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        r[u] = nr[u];
        o[u] = no[u];
      }
      if (p + U < p1) load_index(p + U);
      float v[U][CPL];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          float x[VEC] = {};
          if (p + u < p1 && r[u] < s.vocab && col0 + column(q) < s.d) {
            const T* src = dout + o[u] * s.ldo + col0 + column(q);
            if constexpr (FAR) load_nt<VEC>(src, x);
            else load_v<VEC>(src, x);
          }
#pragma unroll
          for (int k = 0; k < VEC; ++k) v[u][q * VEC + k] = x[k];
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p + u >= p1) break;
        if (r[u] != cur) {
          flush();
          cur = r[u];
          began = true;
#pragma unroll
          for (int k = 0; k < CPL; ++k) acc[k] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < CPL; ++k) acc[k] += v[u][k];
      }
    }
    if (p1 < s.n && rows[p1] == cur && cur < s.vocab) {
      keep(began ? 1 : 0);
      if (j == 0) kind[g] |= began ? 2 : 5;
    } else {
      flush();
    }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < C && col0 + x < s.d; x += kRunThreads) {
    float acc = 0.f;
    bool open = false, inside = false;  // a run goes on; it began in this block
    for (int k = 0; k < G; ++k) {
      const int kd = kind[k];
      if (kd & 1) {
        acc = open ? acc + part[k][0][x] : part[k][0][x];
        open = true;
        if (!(kd & 4)) {
          if (inside) {
            float* w = s.dw + first[k] * s.ldw + col0 + x;
            *w = s.add ? *w + s.scale * acc : s.scale * acc;
          } else {
            s.part[(int64_t)2 * blk * s.d + col0 + x] = acc;
          }
          open = inside = false;
        }
      }
      if (kd & 2) {
        acc = part[k][1][x];
        open = inside = true;
      }
    }
    if (open) s.part[((int64_t)2 * blk + (inside ? 1 : 0)) * s.d + col0 + x] = acc;
  }
}

// Joins the runs that cross stretches: the block of the stretch in which a run
// begins adds that stretch's slot 1 and slot 0 of the stretches up to the run's
// end. `lanes` (a power of two) lanes a row of VEC columns each; the groups of
// lanes take the partial rows in turn, eight loads in flight, and are added in
// order. One block for all columns, since most have no run to join.
constexpr int kJoinThreads = 512;

template <int VEC>
__global__ void __launch_bounds__(kJoinThreads) k_embed_join(RunSums s, int lanes) {
  constexpr int U = 8;
  __shared__ float red[kJoinThreads * VEC];
  const int c = blockIdx.x;
  const int p0 = c * s.stretch, p1 = p0 + s.stretch;  // p1 < n: one block fewer than stretches
  const int v = s.row[p1], before = s.row[p1 - 1], first = s.row[p0], early = p0 > 0 ? s.row[p0 - 1] : -1;
  if (v >= s.vocab || before != v || (first == v && early == v)) return;  // no run that begins here and goes on
  // last stretch whose first row is v: lo has it, hi does not; most runs end in the next one
  int lo = c + 1, hi = lo + 1;
  while (hi < s.nstretch && s.row[hi * s.stretch] == v) {
    lo = hi;
    hi = min(s.nstretch, hi + 2 * (hi - c));
  }
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (s.row[mid * s.stretch] == v) lo = mid;
    else hi = mid;
  }
  const int m = lo - c + 1;  // partial rows
  const int G = kJoinThreads / lanes, g = threadIdx.x / lanes, j = threadIdx.x % lanes, used = min(m, G);
  for (int col0 = 0; col0 < s.d; col0 += lanes * VEC) {
    const int col = col0 + j * VEC;
    float acc[VEC] = {};
    for (int q0 = g; q0 < m; q0 += G * U) {
      float x[U][VEC];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int q = q0 + u * G;
#pragma unroll
        for (int k = 0; k < VEC; ++k) x[u][k] = 0.f;
        if (q < m && col < s.d) load_v<VEC>(s.part + ((int64_t)2 * (c + q) + (q == 0)) * s.d + col, x[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] += x[u][k];
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) red[threadIdx.x * VEC + k] = acc[k];
    __syncthreads();
    for (int x = threadIdx.x; x < lanes * VEC && col0 + x < s.d; x += kJoinThreads) {
      float t = red[x];
      for (int k = 1; k < used; ++k) t += red[k * lanes * VEC + x];
      float* w = s.dw + v * s.ldw + col0 + x;
      *w = s.add ? *w + s.scale * t : s.scale * t;
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Few tokens: one launch, in which a block finds the tokens of one table row by
// looking at all of them and sums their rows. By row, block v takes row v (and
// writes its zeros if it has no token). By token, for tables with more rows than
// tokens, block b < n takes the row of token b if b is the first of its kind,
// and the blocks after them write the zeros of the other rows. Each of the
// launch's y blocks takes LPR VEC columns.
// ---------------------------------------------------------------------------
constexpr int kFewTokens = 16384, kFewThreads = 1024, kFewZeroRows = 128;
constexpr int kFewEach = kFewTokens / kFewThreads;  // tokens a thread looks at, at most

template <class T, int VEC, int LPR>
__global__ void __launch_bounds__(kFewThreads) k_embed_few(int n, int d, int vocab, const int* __restrict__ tok,
                                                           int first, const T* __restrict__ dout, int64_t ldo,
                                                           float scale, float* __restrict__ dw, int64_t ldw, int add,
                                                           int by_row) {
  constexpr int W = kFewThreads / 64, G = kFewThreads / LPR, U = 8;
  __shared__ unsigned short list[kFewTokens];
  __shared__ int wtot[W], has[kFewZeroRows];
  __shared__ float red[G][LPR * VEC];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int c0 = blockIdx.y * LPR * VEC, c = c0 + t % LPR * VEC;
  if (!by_row && (int)blockIdx.x >= n) {
    const int64_t step = (int64_t)(gridDim.x - n) * kFewZeroRows;
    for (int64_t v0 = (int64_t)(blockIdx.x - n) * kFewZeroRows; v0 < vocab; v0 += step) {
      for (int k = t; k < kFewZeroRows; k += kFewThreads) has[k] = 0;
      __syncthreads();
      for (int i = t; i < n; i += kFewThreads) {
        const int row = table_row(tok[i], first, vocab);
        if (row < vocab && row >= v0 && row < v0 + kFewZeroRows) has[row - v0] = 1;
      }
      __syncthreads();
      const int rows = (int)min((int64_t)kFewZeroRows, vocab - v0);
      for (int r = t / LPR; r < rows; r += G) {
        if (has[r] || c >= d) continue;
        const float none[VEC] = {};
        store_v<VEC>(dw + (v0 + r) * ldw + c, none);
      }
      __syncthreads();
    }
    return;
  }
  const int b = blockIdx.x, v = by_row ? b : table_row(tok[b], first, vocab);
  if (v == vocab) return;
  // the list of the row's tokens in order: each thread looks at `each`
  // consecutive tokens, and a scan over the threads places its hits
  const int each = (n + kFewThreads - 1) / kFewThreads;
  unsigned hits = 0;
#pragma unroll
  for (int k = 0; k < kFewEach; ++k) {
    const int i = t * each + k;
    if (k < each && i < n && table_row(tok[i], first, vocab) == v) hits |= 1u << k;
  }
  const int mine = __popc(hits);
  int incl = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int x = __shfl_up(incl, off);
    if (lane >= off) incl += x;
  }
  if (lane == 63) wtot[wave] = incl;
  __syncthreads();
  int at = incl - mine, m = 0;
  for (int k = 0; k < W; ++k) {
    if (k < wave) at += wtot[k];
    m += wtot[k];
  }
  for (; hits; hits &= hits - 1) list[at++] = (unsigned short)(t * each + __ffs(hits) - 1);
  __syncthreads();
  if (!by_row && list[0] != b) return;  // not the first of its kind
  if (add && m == 0) return;
  // a group's share of the list, at least U rows if there are as many
  const int g = t / LPR, groups = min(G, (m + U - 1) / U);
  const int q0 = g < groups ? (int)((int64_t)m * g / groups) : 0, q1 = g < groups ? (int)((int64_t)m * (g + 1) / groups) : 0;
  float acc[VEC] = {};
  for (int q = q0; q < q1; q += U) {
    float x[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[u][k] = 0.f;
      if (q + u < q1 && c < d) load_v<VEC>(dout + list[q + u] * ldo + c, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < VEC; ++k) acc[k] += x[u][k];
  }
#pragma unroll
  for (int k = 0; k < VEC; ++k) red[g][t % LPR * VEC + k] = acc[k];
  __syncthreads();
  if (t < LPR * VEC && c0 + t < d) {
    float sum = red[0][t];
    for (int k = 1; k < groups; ++k) sum += red[k][t];
    float* w = dw + v * ldw + c0 + t;
    *w = add ? *w + scale * sum : m ? scale * sum : 0.f;
  }
}

// Values a lane: 16 bytes of the type, 4 values of 16 bits where 8 do not fit
// the alignment, else 1. Lanes a row: the fewest of 16, 32 and 64 that hold d
// values (64 lanes take further columns in turn).
int vec_of(int32_t dtype, int32_t d, int64_t lda, int64_t ldb, const void* a, const void* b, size_t bsize) {
  const size_t es = elem_size(dtype);
  for (int v = es == 2 ? 8 : 4; v >= 4; v -= 4)
    if (d % v == 0 && lda % v == 0 && ldb % 4 == 0 && aligned_to(a, v * es) && aligned_to(b, std::min<size_t>(16, v * bsize)) &&
        (bsize == 4 || ldb % v == 0))
      return v;
  return 1;
}
int lanes_of(int32_t d, int vec) { return vec == 1 || d > 32 * vec ? 64 : d > 16 * vec ? 32 : 16; }

template <class T, class F>
int with_lanes(int d, int vec, F&& f) {
  using std::integral_constant;
  const int lanes = lanes_of(d, vec);
  if constexpr (sizeof(T) == 2) {
    if (vec == 8) {
      if (lanes == 16) return f(integral_constant<int, 8>{}, integral_constant<int, 16>{});
      if (lanes == 32) return f(integral_constant<int, 8>{}, integral_constant<int, 32>{});
      return f(integral_constant<int, 8>{}, integral_constant<int, 64>{});
    }
  }
  if (vec == 1) return f(integral_constant<int, 1>{}, integral_constant<int, 64>{});
  if (lanes == 16) return f(integral_constant<int, 4>{}, integral_constant<int, 16>{});
  if (lanes == 32) return f(integral_constant<int, 4>{}, integral_constant<int, 32>{});
  return f(integral_constant<int, 4>{}, integral_constant<int, 64>{});
}

// Whether a call of this layout takes the one launch: the tokens that its blocks
// look at must stay few (fewer where blocks by token do it, most of which find
// that they are not the first of their kind), and so must the rows of a frequent
// token, which the groups of lanes of one block add up alone. With tokens evenly
// spread and with a third of them on one row, against the ordering's four or six
// launches, us a call: of 94 rows 16,384 of 64 fp32 11 and 19 (20 and 22), 12,000
// of 128 7 and 18 (18 and 19), 16,384 of 128 11 and 29 (18 and 20), 8,192 of 512
// 9 and 26 (18 and 19); 8,000 of 1,000 rows of 64 20 and 21 (31 and 30); by token
// 2,000 of 5,000 rows of 64 16 and 15 (27 and 29), of 50,000 rows of 512 in bf16
// 44 and 41 (37 and 38).
bool few_tokens(int64_t n, int64_t vocab, int64_t tiles, int lanes, int vec) {
  if (n > kFewTokens) return false;
  const int64_t looks = (vocab <= n ? vocab : n + cdiv(vocab, kFewZeroRows)) * n * tiles;
  return looks <= (vocab <= n ? 1 << 23 : 1 << 22) && n * lanes * std::max(vec, 4) <= 3 << 19;
}
int64_t tiles_of(int32_t d, int vec) { return cdiv(d, (int64_t)lanes_of(d, vec) * vec); }

int check_embed(const char* who, int64_t n, int32_t d, int64_t vocab, int32_t dtype, int32_t first) {
  const std::string w(who);
  if (n < 0) return fail(CHGNET_EINVAL, w + ": n is negative");
  if (d < 1 || d > 65536) return fail(CHGNET_EINVAL, w + ": d must be in 1..65536");
  if (vocab < 1 || vocab > INT32_MAX) return fail(CHGNET_EINVAL, w + ": vocab must be in 1..2^31-1");
  if (!elem_size(dtype)) return fail(CHGNET_EINVAL, w + ": unknown dtype");
  if (first < 0) return fail(CHGNET_EINVAL, w + ": first is negative");
  return CHGNET_OK;
}

// Length of a chunk of the ordered positions: about 8,192 chunks, whose rows in
// flight fill the chip, of 16 to 256 positions.
int chunk_of(int64_t n) { return (int)std::min<int64_t>(256, std::max<int64_t>(16, cdiv(n, 8192))); }

// Positions of a block of k_embed_runs: a chunk for each of its groups of lanes.
int stretch_of(int64_t n, int lanes) { return chunk_of(n) * (kRunThreads / lanes); }

constexpr int64_t kMaxTokens = 1 << 30;  // positions and the ends of chunks are 32-bit

struct EmbedWs {
  int *row[2], *pos[2], *counts;
  float* part;
};
void carve_embed(Arena& ar, int64_t n, int32_t d, int64_t vocab, EmbedWs& w) {
  // (none for the one launch, if it is taken whichever layout the alignment allows)
  bool few = true;
  for (int vec : {1, 4, 8}) few = few && few_tokens(n, vocab, tiles_of(d, vec), lanes_of(d, vec), vec);
  if (few) return;
  for (int k = 0; k < 2; ++k) {
    w.row[k] = ar.take<int>(n);
    w.pos[k] = ar.take<int>(n);
  }
  w.counts = ar.take<int>((int64_t)kSortBlocks * kDigits);
  w.part = ar.take<float>(2 * cdiv(n, stretch_of(n, 64)) * d);  // (the shortest stretches are those of 64 lanes)
}

}  // namespace

int embed_forward_entry(int64_t n, int32_t d, int64_t vocab, int32_t dtype, const int32_t* tok, int32_t first,
                        const void* table, int64_t ldt, float scale, void* out, int64_t ldo, hipStream_t st) {
  CHG_TRY(check_embed("embed_forward", n, d, vocab, dtype, first));
  if (ldt < d || ldo < d) return fail(CHGNET_EINVAL, "embed_forward: a row stride is below the row's width");
  if (n == 0) return CHGNET_OK;
  if (!tok || !table || !out) return fail(CHGNET_EINVAL, "embed_forward: null argument");
  const size_t es = elem_size(dtype);
  if (!aligned_to(tok, 4) || !aligned_to(table, es) || !aligned_to(out, es))
    return fail(CHGNET_EINVAL, "embed_forward: an array is not aligned to its values");
  const int vec = vec_of(dtype, d, ldt, ldo, table, out, es);
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes<T>(d, vec, [&](auto V, auto L) -> int {
      const unsigned blocks = (unsigned)std::min<int64_t>(4096, cdiv(n, 256 / L.value * kFwdRows));
      KLAUNCH(st, "k_embed_fwd",
              k_embed_fwd<T, V.value, L.value><<<blocks, 256, 0, st>>>(n, d, (int)vocab, tok, first,
                                                                       static_cast<const T*>(table), ldt, scale,
                                                                       static_cast<T*>(out), ldo));
      return CHGNET_OK;
    });
  });
}

size_t embed_backward_bytes(int64_t n, int32_t d, int64_t vocab) {
  Arena ar;
  EmbedWs w;
  carve_embed(ar, n, d, vocab, w);
  return ar.used;
}

int embed_backward_workspace_entry(int64_t n, int32_t d, int64_t vocab, size_t* bytes) {
  CHG_TRY(check_embed("embed_backward_workspace", n, d, vocab, CHGNET_F32, 0));
  if (n > kMaxTokens) return fail(CHGNET_EINVAL, "embed_backward_workspace: n must be at most 2^30");
  if (!bytes) return fail(CHGNET_EINVAL, "embed_backward_workspace: bytes is NULL");
  *bytes = embed_backward_bytes(n, d, vocab);
  return CHGNET_OK;
}

// tag: the launches' name in a profile, in place of their own
int embed_backward_entry(int64_t n64, int32_t d, int64_t vocab64, int32_t dtype, const int32_t* tok, int32_t first,
                         const void* dout, int64_t ldo, float scale, float* dtable, int64_t ldw, int accumulate,
                         void* ws, size_t ws_bytes, hipStream_t st, const char* tag) {
  CHG_TRY(check_embed("embed_backward", n64, d, vocab64, dtype, first));
  if (n64 > kMaxTokens) return fail(CHGNET_EINVAL, "embed_backward: n must be at most 2^30");
  if (ldo < d || ldw < d) return fail(CHGNET_EINVAL, "embed_backward: a row stride is below the row's width");
  if (!dtable || (n64 > 0 && (!tok || !dout))) return fail(CHGNET_EINVAL, "embed_backward: null argument");
  const size_t es = elem_size(dtype);
  if (!aligned_to(tok, 4) || !aligned_to(dout, es) || !aligned_to(dtable, 4))
    return fail(CHGNET_EINVAL, "embed_backward: an array is not aligned to its values");
  const int n = (int)n64, vocab = (int)vocab64;
  const int add = accumulate != 0;
  const int vec = vec_of(dtype, d, ldo, ldw, dout, dtable, 4);
  if (few_tokens(n, vocab, tiles_of(d, vec), lanes_of(d, vec), vec)) {
    if (n == 0 && add) return CHGNET_OK;
    const bool by_row = vocab <= n;
    const unsigned blocks = (unsigned)(by_row ? vocab : n + (add ? 0 : std::min<int64_t>(4096, cdiv(vocab, kFewZeroRows))));
    return with_type(dtype, [&](auto t) {
      using T = decltype(t);
      return with_lanes<T>(d, vec, [&](auto V, auto L) -> int {
        KLAUNCH(st, tag ? tag : "k_embed_few",
                k_embed_few<T, V.value, L.value><<<dim3(blocks, (unsigned)cdiv(d, L.value * V.value)), kFewThreads, 0, st>>>(
                    n, d, vocab, tok, first, static_cast<const T*>(dout), ldo, scale, dtable, ldw, add, by_row));
        return CHGNET_OK;
      });
    });
  }
  size_t need = 0;
  CHG_TRY(embed_backward_workspace_entry(n, d, vocab, &need));
  if (!ws || ws_bytes < need)
    return fail(CHGNET_EWORKSPACE, "embed_backward: workspace too small (query chgnet_embed_backward_workspace)");
  if (!aligned_to(ws, 16)) return fail(CHGNET_EINVAL, "embed_backward: ws is not 16-byte aligned");
  Arena ar{static_cast<char*>(ws), ws_bytes, 0};
  EmbedWs w{};
  carve_embed(ar, n, d, vocab, w);
  // digits of the rows 0 .. vocab (vocab: no row), split evenly over the passes
  int bits = 1;
  while (bits < 31 && (vocab >> bits) != 0) ++bits;
  const int passes = (int)cdiv(bits, 8), width = (int)cdiv(bits, passes);
  SortPass s{};
  s.n = n;
  s.vocab = vocab;
  s.first = first;
  // (kSortBlocks stretches of one round, or as many rounds as that takes)
  const int rounds = n <= kSortBlocks * kSortThreads ? 1 : 4;
  s.len = cdiv(cdiv(n, kSortBlocks), kSortThreads * rounds) * kSortThreads * rounds;
  const int nb = (int)cdiv(n, s.len);
  s.counts = w.counts;
  for (int p = 0; p < passes; ++p) {
    s.shift = p * width;
    s.bits = std::min(width, bits - s.shift);
    s.tok = p == 0 ? tok : nullptr;
    s.row = w.row[(p + 1) & 1];
    s.pos = w.pos[(p + 1) & 1];
    s.row_out = w.row[p & 1];
    s.pos_out = w.pos[p & 1];
    KLAUNCH(st, tag ? tag : "k_embed_count", k_embed_count<<<nb, kSortThreads, 0, st>>>(s));
    if (rounds == 1) KLAUNCH(st, tag ? tag : "k_embed_place", k_embed_place<1><<<nb, kSortThreads, 0, st>>>(s));
    else KLAUNCH(st, tag ? tag : "k_embed_place", k_embed_place<4><<<nb, kSortThreads, 0, st>>>(s));
  }
  RunSums r{};
  r.n = n;
  r.vocab = vocab;
  r.chunk = chunk_of(n);
  r.stretch = stretch_of(n, lanes_of(d, vec));
  r.nstretch = (int)cdiv(n, r.stretch);
  r.d = d;
  r.row = w.row[(passes + 1) & 1];
  r.pos = w.pos[(passes + 1) & 1];
  r.ldo = ldo;
  r.ldw = ldw;
  r.scale = scale;
  r.dw = dtable;
  r.add = add;
  r.part = w.part;
  r.nzero = add ? 0 : (int)cdiv(vocab, kZeroRows);
  CHG_TRY(with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes<T>(d, vec, [&](auto V, auto L) -> int {
      constexpr int NQ = V.value == 1 ? 4 : 1;
      const dim3 grid((unsigned)(r.nzero + r.nstretch), (unsigned)cdiv(d, L.value * V.value * NQ));
      const T* x = static_cast<const T*>(dout);
      if constexpr (V.value > 1) {
        if ((int64_t)n * d * (int64_t)sizeof(T) >= kFarBytes) {
          KLAUNCH(st, tag ? tag : "k_embed_runs",
                  k_embed_runs<T, V.value, L.value, NQ, true><<<grid, kRunThreads, 0, st>>>(r, r.row, r.pos, x));
          return CHGNET_OK;
        }
      }
      KLAUNCH(st, tag ? tag : "k_embed_runs",
              k_embed_runs<T, V.value, L.value, NQ, false><<<grid, kRunThreads, 0, st>>>(r, r.row, r.pos, x));
      return CHGNET_OK;
    });
  }));
  if (r.nstretch > 1) {
    // the partial rows are dense: 16-byte loads where their width allows
    const int v = d % 4 == 0 ? 4 : 1;
    int lanes = 16;
    while (lanes < kJoinThreads && lanes * v < d) lanes *= 2;
    if (v == 4) KLAUNCH(st, tag ? tag : "k_embed_join", k_embed_join<4><<<r.nstretch - 1, kJoinThreads, 0, st>>>(r, lanes));
    else KLAUNCH(st, tag ? tag : "k_embed_join", k_embed_join<1><<<r.nstretch - 1, kJoinThreads, 0, st>>>(r, lanes));
  }
  return CHGNET_OK;
}

}  // namespace chg
