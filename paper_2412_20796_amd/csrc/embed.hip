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
// sums, in order. Few tokens skip the ordering: a block a token finds the
// others like it by comparing all of them.
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
// kFwdRows rows at a time, so that as many loads are in flight.
// ---------------------------------------------------------------------------
constexpr int kFwdRows = 4;

template <class T, int VEC, int LPR>
__global__ void __launch_bounds__(256) k_embed_fwd(int64_t n, int d, int vocab, const int* __restrict__ tok, int first,
                                                   const T* __restrict__ table, int64_t ldt, float scale,
                                                   T* __restrict__ out, int64_t ldo) {
  constexpr int G = 256 / LPR;
  const int j = threadIdx.x % LPR, g = threadIdx.x / LPR;
  const int64_t stride = (int64_t)gridDim.x * G * kFwdRows;
  for (int64_t i0 = ((int64_t)blockIdx.x * G + g) * kFwdRows; i0 < n; i0 += stride) {
    int r[kFwdRows];
#pragma unroll
    for (int u = 0; u < kFwdRows; ++u) r[u] = i0 + u < n ? table_row(tok[i0 + u], first, vocab) : vocab;
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
        store_v<VEC>(out + (i0 + u) * ldo + c, v[u]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Ordering of the positions by table row: passes over digits of at most 8 bits,
// least significant first, each stable. A pass is two launches over at most
// kSortBlocks blocks, each with a contiguous stretch of the tokens, taken 1,024
// at a time: the counts of every digit in every stretch, then the places. A
// block of the second launch adds up the counts of the stretches before its own
// and of the lower digits itself (at most 256 x 256 numbers, in L2), so that no
// scan stands between the two.
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

// Counts of the digits, and (fill blocks, after the counting ones) zeros in the
// table rows: a row's sums overwrite them later.
__global__ void __launch_bounds__(kSortThreads) k_embed_count(SortPass s, int nsort, int64_t zrows, int d, float* zero,
                                                              int64_t ldz) {
  __shared__ int cnt[kDigits];
  const int t = threadIdx.x;
  if ((int)blockIdx.x >= nsort) {
    const int64_t total = zrows * d, step = (int64_t)(gridDim.x - nsort) * kSortThreads;
    int64_t i = (int64_t)(blockIdx.x - nsort) * kSortThreads + t;
    if (ldz == d && total % 4 == 0 && reinterpret_cast<uintptr_t>(zero) % 16 == 0) {
      for (; i < total / 4; i += step) reinterpret_cast<float4*>(zero)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
      for (; i < total; i += step) zero[i / d * ldz + i % d] = 0.f;
    }
    return;
  }
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

__global__ void __launch_bounds__(kSortThreads) k_embed_place(SortPass s) {
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
    for (int b0 = nb * q / 4; b0 < b1; b0 += 16) {
      int c[16];  // loads in flight together: one at a time they took 30 us of 1,000,003 tokens
#pragma unroll
      for (int u = 0; u < 16; ++u) c[u] = b0 + u < b1 ? s.counts[(b0 + u) * kDigits + digit] : 0;
#pragma unroll
      for (int u = 0; u < 16; ++u) {
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
  const int64_t i0 = (int64_t)blockIdx.x * s.len, i1 = min(i0 + s.len, (int64_t)s.n);
  for (int64_t base = i0; base < i1; base += kSortThreads) {
    __syncthreads();
    for (int k = t; k < W * kDigits; k += kSortThreads) (&wcnt[0][0])[k] = 0;
    __syncthreads();
    const int64_t i = base + t;
    const bool valid = i < i1;
    const int row = valid ? sort_row(s, (int)i) : 0;
    const int digit = (row >> s.shift) & ((1 << s.bits) - 1);
    const unsigned long long m = same_digit(digit, s.bits, valid);
    const int rank = __popcll(m & ((1ull << lane) - 1));
    if (valid && rank == 0) wcnt[wave][digit] = __popcll(m);
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
    if (valid) {
      const int to = wcnt[wave][digit] + rank;
      s.row_out[to] = row;
      s.pos_out[to] = s.tok ? (int)i : s.pos[i];
    }
  }
}

// ---------------------------------------------------------------------------
// Sums of the ordered rows. Groups of LPR lanes (VEC NQ values a lane; the
// launch's y blocks take further columns) each add the rows of one chunk, eight
// loads in flight, and write a run's sum when it ends. A run that began in an
// earlier chunk or goes on in the next is a partial sum instead: slot 0 of the
// chunk for a run that began before it, slot 1 for one that begins in it and
// goes on.
// ---------------------------------------------------------------------------
struct RunSums {
  int n, vocab, chunk, nchunks, d;
  const int *row, *pos;
  int64_t ldo, ldw;
  float scale;
  float* dw;
  int add;
  float* part;  // [nchunks][2][d]
};

template <class T, int VEC, int LPR, int NQ>
__global__ void __launch_bounds__(256) k_embed_runs(RunSums s, const T* __restrict__ dout) {
  constexpr int G = 256 / LPR, U = 8, CPL = VEC * NQ;
  const int j = threadIdx.x % LPR;
  const int c = blockIdx.x * G + threadIdx.x / LPR;
  if (c >= s.nchunks) return;
  const int col0 = blockIdx.y * LPR * CPL;
  const int p0 = c * s.chunk, p1 = min(p0 + s.chunk, s.n);
  float acc[CPL];
#pragma unroll
  for (int k = 0; k < CPL; ++k) acc[k] = 0.f;
  int cur = s.row[p0];
  bool began = p0 == 0 || s.row[p0 - 1] != cur;  // the run starts in this chunk
  auto column = [&](int q) { return col0 + (q * LPR + j) * VEC; };
  auto flush = [&](bool goes_on) {
    if (cur >= s.vocab) return;
    if (began && !goes_on) {
      float* w = s.dw + cur * s.ldw;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        if (column(q) >= s.d) continue;
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
    } else {
      float* w = s.part + ((int64_t)2 * c + (began ? 1 : 0)) * s.d;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        if (column(q) >= s.d) continue;
        float v[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = acc[q * VEC + k];
        store_v<VEC>(w + column(q), v);
      }
    }
  };
  int nr[U], no[U];  // the next step's rows and positions, loaded a step ahead
  auto load_index = [&](int p) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = min(p + u, p1 - 1);
      nr[u] = s.row[x];
      no[u] = s.pos[x];
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
        if (p + u < p1 && r[u] < s.vocab && column(q) < s.d) load_v<VEC>(dout + o[u] * s.ldo + column(q), x);
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[u][q * VEC + k] = x[k];
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u >= p1) break;
      if (r[u] != cur) {
        flush(false);
        cur = r[u];
        began = true;
#pragma unroll
        for (int k = 0; k < CPL; ++k) acc[k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < CPL; ++k) acc[k] += v[u][k];
    }
  }
  flush(p1 < s.n && s.row[p1] == cur);
}

// Joins the runs that cross chunks: the block of the chunk in which a run
// begins adds that chunk's slot 1 and slot 0 of the chunks up to the run's end.
// 64 columns a block, 16 lanes a row; the groups of lanes take the partial rows
// in turn, eight loads in flight, and are added in order.
constexpr int kJoinThreads = 512;

template <int VEC>
__global__ void __launch_bounds__(kJoinThreads) k_embed_join(RunSums s) {
  constexpr int G = kJoinThreads / 16, U = 8, C = 16 * VEC;
  __shared__ float red[G][C];
  const int c = blockIdx.x;
  const int p0 = c * s.chunk, p1 = p0 + s.chunk;
  if (p1 >= s.n) return;
  const int v = s.row[p1];
  if (v >= s.vocab || s.row[p1 - 1] != v) return;
  if (s.row[p0] == v && p0 > 0 && s.row[p0 - 1] == v) return;  // begins earlier
  int lo = c + 1, hi = s.nchunks;  // last chunk whose first row is v: lo has it, hi does not
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (s.row[mid * s.chunk] == v) lo = mid;
    else hi = mid;
  }
  const int m = lo - c + 1;  // partial rows
  const int g = threadIdx.x >> 4, j = threadIdx.x & 15, col = blockIdx.y * C + j * VEC;
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
  for (int k = 0; k < VEC; ++k) red[g][j * VEC + k] = acc[k];
  __syncthreads();
  const int x = threadIdx.x, cx = blockIdx.y * C + x, used = min(m, G);
  if (x >= C || cx >= s.d) return;
  float t = red[0][x];
  for (int k = 1; k < used; ++k) t += red[k][x];
  float* w = s.dw + v * s.ldw + cx;
  *w = s.add ? *w + s.scale * t : s.scale * t;
}

// ---------------------------------------------------------------------------
// Few tokens: one launch, in which a block finds the tokens of one table row by
// looking at all of them and sums their rows. By row, block v takes row v (and
// writes its zeros if it has no token). By token, for tables with more rows than
// tokens, block b < n takes the row of token b if b is the first of its kind,
// and the blocks after them write the zeros of the other rows.
// ---------------------------------------------------------------------------
constexpr int kFewTokens = 8192, kFewThreads = 1024, kFewZeroRows = 512;
constexpr int kFewEach = kFewTokens / kFewThreads;  // tokens a thread looks at, at most

template <class T, int VEC, int LPR>
__global__ void __launch_bounds__(kFewThreads) k_embed_few(int n, int d, int vocab, const int* __restrict__ tok,
                                                           int first, const T* __restrict__ dout, int64_t ldo,
                                                           float scale, float* __restrict__ dw, int64_t ldw, int add,
                                                           int by_row) {
  constexpr int W = kFewThreads / 64, G = kFewThreads / LPR, U = 8;
  __shared__ int list[kFewTokens];
  __shared__ int wtot[W], has[kFewZeroRows];
  __shared__ float red[G][LPR * VEC];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
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
      for (int r = wave; r < rows; r += W) {
        if (has[r]) continue;
        float* w = dw + (v0 + r) * ldw;
        const float none[VEC] = {};
        for (int c = lane * VEC; c < d; c += 64 * VEC) store_v<VEC>(w + c, none);
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
  for (; hits; hits &= hits - 1) list[at++] = t * each + __ffs(hits) - 1;
  __syncthreads();
  if (!by_row && list[0] != b) return;  // not the first of its kind
  if (add && m == 0) return;
  const int j = t % LPR, g = t / LPR, groups = min(G, (m + U - 1) / U);
  // a group's share of the list, at least U rows if there are as many
  const int q0 = g < groups ? (int)((int64_t)m * g / groups) : 0, q1 = g < groups ? (int)((int64_t)m * (g + 1) / groups) : 0;
  for (int c0 = 0; c0 < d; c0 += LPR * VEC) {
    const int c = c0 + j * VEC;
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
    for (int k = 0; k < VEC; ++k) red[g][j * VEC + k] = acc[k];
    __syncthreads();
    for (int x = t; x < LPR * VEC && c0 + x < d; x += kFewThreads) {
      float sum = red[0][x];
      for (int k = 1; k < groups; ++k) sum += red[k][x];
      float* w = dw + v * ldw + c0 + x;
      *w = add ? *w + scale * sum : scale * sum;
    }
    __syncthreads();
  }
}

// Whether a call takes the one launch: what its blocks look at must stay small.
bool few_tokens(int64_t n, int64_t vocab) {
  return n <= kFewTokens && std::min(n, vocab) * n <= (1 << 20);
}

// Lanes a row: the fewest of 16, 32 and 64 that hold d values, 4 each.
template <class F>
int with_lanes(int d, bool vec, F&& f) {
  using std::integral_constant;
  if (!vec) return f(integral_constant<int, 1>{}, integral_constant<int, 64>{});
  if (d <= 64) return f(integral_constant<int, 4>{}, integral_constant<int, 16>{});
  if (d <= 128) return f(integral_constant<int, 4>{}, integral_constant<int, 32>{});
  return f(integral_constant<int, 4>{}, integral_constant<int, 64>{});
}

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

constexpr int64_t kMaxTokens = 1 << 30;  // positions and the ends of chunks are 32-bit

struct EmbedWs {
  int *row[2], *pos[2], *counts;
  float* part;
};
void carve_embed(Arena& ar, int64_t n, int32_t d, int64_t vocab, EmbedWs& w) {
  if (few_tokens(n, vocab)) return;
  for (int k = 0; k < 2; ++k) {
    w.row[k] = ar.take<int>(n);
    w.pos[k] = ar.take<int>(n);
  }
  w.counts = ar.take<int>((int64_t)kSortBlocks * kDigits);
  w.part = ar.take<float>(2 * cdiv(n, chunk_of(n)) * d);
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
  const bool vec = d % 4 == 0 && ldt % 4 == 0 && ldo % 4 == 0 && aligned_to(table, 4 * es) && aligned_to(out, 4 * es);
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes(d, vec, [&](auto V, auto L) -> int {
      const unsigned blocks = (unsigned)std::min<int64_t>(4096, cdiv(n, 256 / L.value * kFwdRows));
      KLAUNCH(st, "k_embed_fwd",
              k_embed_fwd<T, V.value, L.value><<<blocks, 256, 0, st>>>(n, d, (int)vocab, tok, first,
                                                                       static_cast<const T*>(table), ldt, scale,
                                                                       static_cast<T*>(out), ldo));
      return CHGNET_OK;
    });
  });
}

int embed_backward_workspace_entry(int64_t n, int32_t d, int64_t vocab, size_t* bytes) {
  CHG_TRY(check_embed("embed_backward_workspace", n, d, vocab, CHGNET_F32, 0));
  if (n > kMaxTokens) return fail(CHGNET_EINVAL, "embed_backward_workspace: n must be at most 2^30");
  if (!bytes) return fail(CHGNET_EINVAL, "embed_backward_workspace: bytes is NULL");
  Arena ar;
  EmbedWs w;
  carve_embed(ar, n, d, vocab, w);
  *bytes = ar.used;
  return CHGNET_OK;
}

int embed_backward_entry(int64_t n64, int32_t d, int64_t vocab64, int32_t dtype, const int32_t* tok, int32_t first,
                         const void* dout, int64_t ldo, float scale, float* dtable, int64_t ldw, int accumulate,
                         void* ws, size_t ws_bytes, hipStream_t st) {
  CHG_TRY(check_embed("embed_backward", n64, d, vocab64, dtype, first));
  if (n64 > kMaxTokens) return fail(CHGNET_EINVAL, "embed_backward: n must be at most 2^30");
  if (ldo < d || ldw < d) return fail(CHGNET_EINVAL, "embed_backward: a row stride is below the row's width");
  if (!dtable || (n64 > 0 && (!tok || !dout))) return fail(CHGNET_EINVAL, "embed_backward: null argument");
  const size_t es = elem_size(dtype);
  if (!aligned_to(tok, 4) || !aligned_to(dout, es) || !aligned_to(dtable, 4))
    return fail(CHGNET_EINVAL, "embed_backward: an array is not aligned to its values");
  const int n = (int)n64, vocab = (int)vocab64;
  const int add = accumulate != 0;
  const bool vec = d % 4 == 0 && ldo % 4 == 0 && ldw % 4 == 0 && aligned_to(dout, 4 * es) && aligned_to(dtable, 16);
  if (few_tokens(n, vocab)) {
    if (n == 0 && add) return CHGNET_OK;
    const bool by_row = vocab <= n;
    const unsigned blocks = (unsigned)(by_row ? vocab : n + (add ? 0 : std::min<int64_t>(4096, cdiv(vocab, kFewZeroRows))));
    return with_type(dtype, [&](auto t) {
      using T = decltype(t);
      return with_lanes(d, vec, [&](auto V, auto L) -> int {
        KLAUNCH(st, "k_embed_few",
                k_embed_few<T, V.value, L.value><<<blocks, kFewThreads, 0, st>>>(
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
  s.len = cdiv(cdiv(n, kSortBlocks), kSortThreads) * kSortThreads;
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
    const int64_t zrows = p == 0 && !add ? vocab : 0;
    const int zb = (int)std::min<int64_t>(512, cdiv(zrows * d, 4 * kSortThreads));
    KLAUNCH(st, "k_embed_count", k_embed_count<<<nb + zb, kSortThreads, 0, st>>>(s, nb, zrows, d, dtable, ldw));
    KLAUNCH(st, "k_embed_place", k_embed_place<<<nb, kSortThreads, 0, st>>>(s));
  }
  RunSums r{};
  r.n = n;
  r.vocab = vocab;
  r.chunk = chunk_of(n);
  r.nchunks = (int)cdiv(n, r.chunk);
  r.d = d;
  r.row = w.row[(passes + 1) & 1];
  r.pos = w.pos[(passes + 1) & 1];
  r.ldo = ldo;
  r.ldw = ldw;
  r.scale = scale;
  r.dw = dtable;
  r.add = add;
  r.part = w.part;
  CHG_TRY(with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes(d, vec, [&](auto V, auto L) -> int {
      constexpr int NQ = V.value == 1 ? 4 : 1;
      const dim3 grid((unsigned)cdiv(r.nchunks, 256 / L.value), (unsigned)cdiv(d, L.value * V.value * NQ));
      KLAUNCH(st, "k_embed_runs", k_embed_runs<T, V.value, L.value, NQ><<<grid, 256, 0, st>>>(r, static_cast<const T*>(dout)));
      return CHGNET_OK;
    });
  }));
  if (r.nchunks > 1) {
    // the partial rows are dense: 16-byte loads where their width allows
    if (d % 4 == 0)
      KLAUNCH(st, "k_embed_join", k_embed_join<4><<<dim3(r.nchunks - 1, (unsigned)cdiv(d, 64)), kJoinThreads, 0, st>>>(r));
    else
      KLAUNCH(st, "k_embed_join", k_embed_join<1><<<dim3(r.nchunks - 1, (unsigned)cdiv(d, 16)), kJoinThreads, 0, st>>>(r));
  }
  return CHGNET_OK;
}

}  // namespace chg
