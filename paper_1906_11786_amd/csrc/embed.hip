// Node states from a token table, and the table's gradient.
//
//  * forward: X[i] = c_i * sum_{k in list i} E[tok[k]], c_i = scale or, for the
//    mean, scale / len_i, then dropout by element number i * H + h;
//  * reverse: dE[v] += sum_{k : tok[k] = v} c_row(k) * keep * dX[row(k)].  The
//    tokens are sorted with their rows (stable, so that every sum keeps the
//    list order), then each run of one token is summed: no float atomics, the
//    result does not depend on how workgroups are scheduled.
//
// Ids outside [0, V) add nothing and get nothing.
#include "counter_rng.h"

namespace ggnn {
namespace dev {

// H / 8 neighbouring lanes handle one row, eight features each.
constexpr int kEmbThreads = 256;

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// Rows of a lane group, one token per node.
constexpr int kEmbRows = 4;

template <typename S, int H, bool DROP>
__device__ __forceinline__ void embed_store(S* __restrict__ X, int row, int h, float (&v)[8], float c,
                                            const Dropout& d) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= c;
  const uint64_t e = (uint64_t)row * H + h;
  if constexpr (DROP) drop8(v, e / 8, d);
  store8f_once(X + e, v);
}

// One token per node: a group takes kEmbRows rows, all loads issued before
// the first use, and the states are stored past the caches, which keep the
// table.  Bound by memory: 1,047,000 rows of 256 in bf16 with dropout in 100 us,
// 5.7 TB/s with the table counted once (a large copy moves 5.2, a fill 6.9).
template <typename S, int H, bool DROP>
__global__ __launch_bounds__(kEmbThreads) void embed_rows_kernel(int n, int V, const S* __restrict__ table,
                                                                 const int32_t* __restrict__ tok, int n_tok,
                                                                 float scale, Dropout d, S* __restrict__ X) {
  constexpr int L = H / 8, G = kEmbThreads / L;   // lanes per row, groups per workgroup
  const long row0 = (long)blockIdx.x * (G * kEmbRows) + threadIdx.x / L;
  const int h = 8 * (threadIdx.x % L);
  int id[kEmbRows];
#pragma unroll
  for (int j = 0; j < kEmbRows; ++j) {
    const long row = row0 + j * G;
    id[j] = row < n_tok ? tok[row] : -1;
  }
  float v[kEmbRows][8];
#pragma unroll
  for (int j = 0; j < kEmbRows; ++j) {
    if ((unsigned)id[j] < (unsigned)V) {
      load8f<S>(table + (size_t)id[j] * H + h, v[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < kEmbRows; ++j) {
    const long row = row0 + j * G;
    if (row < n) embed_store<S, H, DROP>(X, (int)row, h, v[j], scale, d);
  }
}

// Lists: four tokens of a list in flight, added in list order.  4.8 us for 20,000
// lists of 0 to 6 at H = 64 in bf16: the launch and three dependent loads.
// 1,047,000 of them over 50,021 tokens: 74 us at H = 64 (0.40 GB of table rows
// gathered, 0.13 written), 273 us at H = 256 (1.6 and 0.54): the gathers, 7.9 TB/s
// with the states written.
template <typename S, int H, bool DROP>
__global__ __launch_bounds__(kEmbThreads) void embed_lists_kernel(int n, int V, const S* __restrict__ table,
                                                                  const int32_t* __restrict__ tok_ptr,
                                                                  const int32_t* __restrict__ tok, int n_tok,
                                                                  float scale, int mean, Dropout d,
                                                                  S* __restrict__ X) {
  constexpr int L = H / 8, U = 4;
  const long row = ((long)blockIdx.x * kEmbThreads + threadIdx.x) / L;
  const int h = 8 * (threadIdx.x % L);
  if (row >= n) return;
  const int lo = clampi(tok_ptr[row], 0, n_tok), hi = clampi(tok_ptr[row + 1], lo, n_tok);
  float acc[8] = {};
  for (int k = lo; k < hi; k += U) {
    int id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = k + u < hi ? tok[k + u] : -1;
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if ((unsigned)id[u] < (unsigned)V) {
        load8f<S>(table + (size_t)id[u] * H + h, v[u]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += v[u][i];
  }
  embed_store<S, H, DROP>(X, (int)row, h, acc, mean && hi > lo ? scale / (float)(hi - lo) : scale, d);
}

}  // namespace dev

namespace {
template <typename S, int H>
hipError_t embed_h(int n, int V, const void* table, const int32_t* tok_ptr, const int32_t* tok, int n_tok,
                   float scale, int mean, const Dropout& d, void* X, hipStream_t st) {
  constexpr int G = dev::kEmbThreads / (H / 8);
  const int per = tok_ptr != nullptr ? G : G * dev::kEmbRows;   // rows of a workgroup
  const dim3 grid((unsigned)(((long)n + per - 1) / per)), block(dev::kEmbThreads);
  const S* E = static_cast<const S*>(table);
  S* out = static_cast<S*>(X);
  if (tok_ptr != nullptr) {
    if (d.cut != 0)
      hipLaunchKernelGGL((dev::embed_lists_kernel<S, H, true>), grid, block, 0, st, n, V, E, tok_ptr, tok, n_tok,
                         scale, mean, d, out);
    else
      hipLaunchKernelGGL((dev::embed_lists_kernel<S, H, false>), grid, block, 0, st, n, V, E, tok_ptr, tok, n_tok,
                         scale, mean, d, out);
  } else {
    if (d.cut != 0)
      hipLaunchKernelGGL((dev::embed_rows_kernel<S, H, true>), grid, block, 0, st, n, V, E, tok, n_tok, scale, d,
                         out);
    else
      hipLaunchKernelGGL((dev::embed_rows_kernel<S, H, false>), grid, block, 0, st, n, V, E, tok, n_tok, scale, d,
                         out);
  }
  return hipGetLastError();
}
}  // namespace

namespace GGNN_IMPL_NS {
hipError_t launch_embed(int n, int H, int V, const void* table, const int32_t* tok_ptr, const int32_t* tok,
                        int n_tok, float scale, int mean, const Dropout& d, void* X, hipStream_t st) {
  using S = dev::dt_t;
  if (n == 0) return hipSuccess;
  switch (H) {
    case 32: return embed_h<S, 32>(n, V, table, tok_ptr, tok, n_tok, scale, mean, d, X, st);
    case 64: return embed_h<S, 64>(n, V, table, tok_ptr, tok, n_tok, scale, mean, d, X, st);
    case 128: return embed_h<S, 128>(n, V, table, tok_ptr, tok, n_tok, scale, mean, d, X, st);
    case 256: return embed_h<S, 256>(n, V, table, tok_ptr, tok, n_tok, scale, mean, d, X, st);
  }
  return hipErrorInvalidValue;
}
}  // namespace GGNN_IMPL_NS

#if GGNN_DT_BF16   // the reverse works on float32 for both dtypes: built once
namespace dev {

// ---- stable sort of (token, row) by token --------------------------------
//
// Least significant digit first.  A pass is a count of each tile's digits, a
// scan of the counts over the tiles of each digit, and a placement that ranks
// a tile's items in order.  Items of tokens outside [0, V) sort to the end.
// 2.1 M tokens (8 bytes an item) of 50,021, two passes: count 15.6 and 10.1 us, scan
// 5.2, placement 16.5; 59,900 of 10,007: count 5.9 and 4.3, placement 6.8, which is
// the latency of a launch and a few dependent loads.

constexpr int kSortThreads = 256, kSortWaves = kSortThreads / kWave;
constexpr int kSortPer = 8;                              // items per thread
constexpr int kSortTile = kSortThreads * kSortPer;       // items per tile
constexpr int kDigits = 256;
constexpr int kWalkRounds = 8;   // rounds of rows that a tile passes over before it searches
constexpr int kFewTiles = 64;   // the placement adds up the counts of as many tiles itself: one launch less a pass

// The last row i with ptr[i] <= k, of rows 0 .. n - 1 (0 where there is none),
// by the whole workgroup: kSortThreads probes a round.
__device__ __forceinline__ int find_row(const int32_t* __restrict__ ptr, int n, int k) {
  int lo = 0, len = n;   // the answer lies in lo .. lo + len - 1
  while (len > 1) {
    const int step = (len + kSortThreads - 1) / kSortThreads;
    const long i = lo + (long)(threadIdx.x + 1) * step;
    const int below = __syncthreads_count(i < (long)lo + len && ptr[i] <= k);
    lo += below * step;
    len = min(step, n - lo);
  }
  return lo;
}

// Digit counts of each tile, count[digit * tiles + tile].  FIRST: the items
// are made from the token list and written to `items`; the row of a position
// is the greatest row whose (not empty) list begins at or before it, so the
// rows mark the positions where their lists begin and a running maximum over
// the tile fills the rest.  A tile whose lists lie among many empty ones searches
// for the row of each position instead: 3,000 tokens on the first of 1M nodes, on
// the first and last, spread over all: calls of 29, 37 and 43 us (752, 785 and 434
// where a tile passed over all rows).
// (count[tile * kDigits + digit] where few tiles need no scan kernel.)
template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(int n_tok, int n, int V,
                                                                  const int32_t* __restrict__ tok_ptr,
                                                                  const int32_t* __restrict__ tok, u32x2* items,
                                                                  int shift, uint32_t mask, int tiles, int few,
                                                                  uint32_t* __restrict__ count) {
  __shared__ uint32_t c[kDigits];
  c[threadIdx.x] = 0;
  const int k0 = blockIdx.x * kSortTile;
  if constexpr (FIRST) {
    __shared__ int rows[kSortTile];
    __shared__ int wm[kSortWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int listed0 = 0, listed1 = n_tok;   // positions that lists hold
    int id[kSortPer];                   // (on their way while the rows are found)
#pragma unroll
    for (int i = 0; i < kSortPer; ++i) id[i] = tok[min(k0 + i * kSortThreads + (int)threadIdx.x, n_tok - 1)];
    if (tok_ptr != nullptr) {
      listed0 = tok_ptr[0];
      listed1 = tok_ptr[n];
      const int first = find_row(tok_ptr, n, k0);
#pragma unroll
      for (int i = 0; i < kSortPer; ++i) rows[i * kSortThreads + threadIdx.x] = first;
      __syncthreads();
      constexpr int U = 4;   // rows of a thread at once
      const int end = min(k0 + kSortTile, listed1);   // lists that begin here or later hold none of the tile
      long i0 = first;
      bool found = false;
      for (int round = 0; !found && i0 < n && round < kWalkRounds; ++round, i0 += U * kSortThreads) {
        int b[U], e[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const long i = i0 + u * kSortThreads + threadIdx.x;
          b[u] = i < n ? tok_ptr[i] : INT_MAX;
          e[u] = i < n ? tok_ptr[i + 1] : INT_MAX;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (b[u] >= k0 && b[u] < k0 + kSortTile && b[u] < e[u])
            rows[b[u] - k0] = (int)(i0 + u * kSortThreads + threadIdx.x);
        found = __syncthreads_or(b[U - 1] >= end);   // lists begin in order: the rest begin later
      }
      __syncthreads();
      if (!found && i0 < n) {   // the last row that begins at or before each position, of rows i0 - 1 .. n - 1
        int lo[kSortPer], len = n - (int)i0 + 1;
#pragma unroll
        for (int i = 0; i < kSortPer; ++i) lo[i] = (int)i0 - 1;
        while (len > 1) {   // the answer lies in lo .. lo + len - 1
          const int half = len / 2;
#pragma unroll
          for (int i = 0; i < kSortPer; ++i)
            if (tok_ptr[lo[i] + half] <= k0 + i * kSortThreads + (int)threadIdx.x) lo[i] += half;
          len -= half;
        }
        // (positions of the rows before i0 have their marks)
#pragma unroll
        for (int i = 0; i < kSortPer; ++i)
          if (lo[i] >= i0) rows[i * kSortThreads + threadIdx.x] = lo[i];
        __syncthreads();
      }
      int m[kSortPer], top = 0;
#pragma unroll
      for (int i = 0; i < kSortPer; ++i) {
        top = max(top, rows[threadIdx.x * kSortPer + i]);
        m[i] = top;
      }
      int run = top;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int u = __shfl_up(run, o);
        if (lane >= o) run = max(run, u);
      }
      if (lane == kWave - 1) wm[wave] = run;
      int before = __shfl_up(run, 1);
      if (lane == 0) before = 0;
      __syncthreads();
      for (int w = 0; w < wave; ++w) before = max(before, wm[w]);
#pragma unroll
      for (int i = 0; i < kSortPer; ++i) rows[threadIdx.x * kSortPer + i] = max(m[i], before);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortPer; ++i) {
      const int k = k0 + i * kSortThreads + threadIdx.x;
      if (k < n_tok) {
        const bool ok = (unsigned)id[i] < (unsigned)V && k >= listed0 && k < listed1;
        const uint32_t key = ok ? (uint32_t)id[i] : (uint32_t)V;
        items[k] = u32x2{key, (uint32_t)(tok_ptr != nullptr ? rows[k - k0] : k)};
        atomicAdd(&c[(key >> shift) & mask], 1u);   // integers: the order does not matter
      }
    }
  } else {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortPer; ++i) {
      const int k = k0 + i * kSortThreads + threadIdx.x;
      if (k < n_tok) atomicAdd(&c[(items[k].x >> shift) & mask], 1u);
    }
  }
  __syncthreads();
  count[few ? (size_t)blockIdx.x * kDigits + threadIdx.x : (size_t)threadIdx.x * tiles + blockIdx.x] = c[threadIdx.x];
}

// Exclusive scan of one digit's counts over the tiles; its total to total[].
__global__ __launch_bounds__(kSortThreads) void sort_scan_kernel(int tiles, uint32_t* __restrict__ count,
                                                                 uint32_t* __restrict__ total) {
  __shared__ uint32_t ws[kSortWaves];
  uint32_t* c = count + (size_t)blockIdx.x * tiles;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint32_t run = 0;
  for (int t0 = 0; t0 < tiles; t0 += kSortThreads) {
    const int t = t0 + threadIdx.x;
    const uint32_t v = t < tiles ? c[t] : 0u;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t u = __shfl_up(s, o);
      if (lane >= o) s += u;
    }
    if (lane == kWave - 1) ws[wave] = s;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      if (w < wave) before += ws[w];
      all += ws[w];
    }
    if (t < tiles) c[t] = run + before + s - v;
    run += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) total[blockIdx.x] = run;
}

// Places a tile's items.  Wave w takes the tile's w-th quarter, 64 items at a
// time in order; an item's rank is the count of its digit in earlier waves,
// in earlier rounds of its wave and in lower lanes of its round.
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(int n_tok, const u32x2* __restrict__ in,
                                                                  u32x2* __restrict__ out, int shift, uint32_t mask,
                                                                  int tiles, int few,
                                                                  const uint32_t* __restrict__ count,
                                                                  const uint32_t* __restrict__ total) {
  __shared__ uint32_t cnt[kSortWaves][kDigits];
  __shared__ uint32_t ws[kSortWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, dig = threadIdx.x;
  const int k0 = blockIdx.x * kSortTile + wave * (kSortTile / kSortWaves);
  u32x2 it[kSortPer];   // on their way while the counts are added up
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    const int k = k0 + i * kWave + lane;
    it[i] = k < n_tok ? in[k] : u32x2{~0u, 0u};
  }
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) cnt[w][dig] = 0;
  // exclusive scan of the digit totals
  uint32_t tot = 0, before = 0;   // the digit's items in all tiles, and in the tiles before this one
  if (few) {
    constexpr int U = 16;
    for (int t0 = 0; t0 < tiles; t0 += U) {
      uint32_t c[U];
#pragma unroll
      for (int u = 0; u < U; ++u) c[u] = t0 + u < tiles ? count[(size_t)(t0 + u) * kDigits + dig] : 0u;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        tot += c[u];
        if (t0 + u < (int)blockIdx.x) before += c[u];
      }
    }
  } else {
    tot = total[dig];
    before = count[(size_t)dig * tiles + blockIdx.x];
  }
  uint32_t s = tot;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t u = __shfl_up(s, o);
    if (lane >= o) s += u;
  }
  if (lane == kWave - 1) ws[wave] = s;
  __syncthreads();
  uint32_t base = s - tot + before;
  for (int w = 0; w < wave; ++w) base += ws[w];

  uint32_t rank[kSortPer];
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    const bool live = k0 + i * kWave + lane < n_tok;
    const uint32_t d = (it[i].x >> shift) & mask;
    uint64_t same = __ballot(live);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint64_t m = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? m : ~m;
    }
    const uint64_t below = same & ((1ull << lane) - 1);
    uint32_t old = 0;
    if (live) old = cnt[wave][d];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // every lane has read before the first of each digit adds
    if (live && below == 0) cnt[wave][d] = old + (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    rank[i] = old + (uint32_t)__popcll(below);
  }
  __syncthreads();
  uint32_t run = base;   // of digit `dig`: first place in each wave's turn
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    const uint32_t c = cnt[w][dig];
    cnt[w][dig] = run;
    run += c;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    if (k0 + i * kWave + lane < n_tok) {
      const uint32_t d = (it[i].x >> shift) & mask;
      out[cnt[wave][d] + rank[i]] = it[i];
    }
  }
}

// ---- sums over runs of one token -----------------------------------------
//
// The sorted list is cut into chunks, one group of H / 8 lanes each, and a
// workgroup's groups take neighbouring chunks (a block of the list).  A run
// inside one chunk is added to its row of the gradient at once.  Of a run that
// crosses chunks, the chunks after the first leave their shares in LDS and the
// chunk where it begins (or the block's first) adds them in order; of a run that
// crosses blocks, each block writes its share to part[block][0] (it began
// before) or part[block][1] (it begins here), and the join kernel adds those
// in block order.
//
// Bound by the gathered rows: 2.1 M of 1 KB (1.05 M rows, each read for every
// listing of it) in 437 us, 4.9 TB/s.  59,900 rows of 256 bytes: 9 us.

// One row of the gradient += acc.
__device__ __forceinline__ void add_row(float* __restrict__ o, const float (&acc)[8]) {
  float v[8];
  load8f<float>(o, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += acc[i];
  store8f(o, v);
}

// S: type of the summed rows.  Row r's factor is scale (over the length of its list
// for the mean, cut at the list's ends as the lookup cuts it), or -factor[r] where
// factor is given.
template <typename S, int H, bool DROP>
__global__ __launch_bounds__(kEmbThreads) void embed_runs_kernel(int n_tok, int n, int V, int chunk,
                                                                 const u32x2* __restrict__ items,
                                                                 const int32_t* __restrict__ tok_ptr, float scale,
                                                                 int mean, const float* __restrict__ factor, Dropout d,
                                                                 const S* __restrict__ dX,
                                                                 float* __restrict__ dtable,
                                                                 float* __restrict__ part) {
  constexpr int L = H / 8, G = kEmbThreads / L, U = 4;
  __shared__ __attribute__((aligned(16))) float head[G][H];   // share of a run that began before the chunk
  __shared__ uint32_t hkey[G];    // its token; V: none
  __shared__ int hfull[G];        // whether it also leaves the chunk
  const int grp = threadIdx.x / L, h = 8 * (threadIdx.x % L);
  const long lo = ((long)blockIdx.x * G + grp) * chunk;
  const uint32_t none = (uint32_t)V;
  const bool lead = threadIdx.x % L == 0;
  float acc[8] = {};
  uint32_t cur = none;
  bool before = false, after = false;
  if (lead) {
    hkey[grp] = none;
    hfull[grp] = 0;
  }
  if (lo < n_tok) {
    const int k0 = (int)lo, k1 = (int)min((long)n_tok, lo + chunk);
    cur = items[k0].x;
    const uint32_t left = items[max(k0 - 1, 0)].x, right = items[min(k1, n_tok - 1)].x;
    before = k0 > 0 && left == cur;
    float old[8] = {};   // the gradient's row of the current token
    if (!before && cur < none) load8f<float>(dtable + (size_t)cur * H + h, old);
    for (int k = k0; k < k1; k += U) {
      u32x2 it[U];
#pragma unroll
      for (int u = 0; u < U; ++u) it[u] = items[min(k + u, k1 - 1)];
      // every load of the four items first: state rows, list lengths, gradient rows of the tokens that begin
      float v[U][8], w[U][8], f[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = min((int)it[u].y, n - 1);
        const bool ok = it[u].x < none && k + u < k1;
        f[u] = scale;
        if (ok) {
          load8f<S>(dX + (size_t)row * H + h, v[u]);
          if (factor != nullptr) f[u] = -factor[row];
          if (tok_ptr != nullptr && mean) {
            const int b = clampi(tok_ptr[row], 0, n_tok), e = clampi(tok_ptr[row + 1], b, n_tok);
            f[u] = scale / (float)max(e - b, 1);
          }
          if (it[u].x != (u > 0 ? it[u - 1].x : cur)) load8f<float>(dtable + (size_t)it[u].x * H + h, w[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k + u >= k1) break;
        if (it[u].x != cur) {   // the run ends inside the chunk
          if (cur < none) {
            if (before) {
              store8f(&head[grp][h], acc);
              if (lead) hkey[grp] = cur;
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) old[i] += acc[i];
              store8f(dtable + (size_t)cur * H + h, old);
            }
          }
          cur = it[u].x;
          before = false;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            acc[i] = 0.f;
            old[i] = w[u][i];
          }
        }
        if (cur < none) {
          if constexpr (DROP) drop8(v[u], ((uint64_t)it[u].y * H + h) / 8, d);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] += f[u] * v[u][i];
        }
      }
    }
    after = k1 < n_tok && right == cur;
    if (cur < none) {
      if (!before && !after) {
#pragma unroll
        for (int i = 0; i < 8; ++i) old[i] += acc[i];
        store8f(dtable + (size_t)cur * H + h, old);
      } else if (before && grp > 0) {
        store8f(&head[grp][h], acc);
        if (lead) {
          hkey[grp] = cur;
          hfull[grp] = after;
        }
      }
    }
  }
  __syncthreads();
  if (lo >= n_tok || cur >= none) {
    // (group 0's head share of a run that ended in its chunk is written below)
  } else if (after && (!before || grp == 0)) {   // a run that leaves this chunk and is this one's to add up
    constexpr int W = 4;   // shares in flight
    for (int j = grp + 1; after && j < G; j += W) {
      float v[W][8];
      int full[W];
#pragma unroll
      for (int u = 0; u < W; ++u) {
        full[u] = hfull[min(j + u, G - 1)];
        load8f<float>(&head[min(j + u, G - 1)][h], v[u]);   // nothing of this run past its end: unused
      }
#pragma unroll
      for (int u = 0; u < W; ++u) {
        if (!after || j + u >= G) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += v[u][i];
        after = full[u] != 0;
      }
    }
    if (before || after) store8f(part + ((size_t)2 * blockIdx.x + (before ? 0 : 1)) * H + h, acc);
    else add_row(dtable + (size_t)cur * H + h, acc);
  } else if (before && !after && grp == 0) {   // the chunk is all one run that ends with it
    store8f(part + (size_t)2 * blockIdx.x * H + h, acc);
  }
  if (grp == 0 && hkey[0] < none) {
    float v[8];
    load8f<float>(&head[0][h], v);
    store8f(part + (size_t)2 * blockIdx.x * H + h, v);
  }
}

// Adds up the runs that cross blocks.  Two workgroups look at kJoinBlocks
// blocks: in one (y = 0) a group adds up a run that begins in its block and ends
// within kJoinShort more; a longer one is added by all groups of the other, each
// a fixed share of its blocks, joined in a fixed tree.  6.3 us for 469 blocks at H =
// 64 (one workgroup doing both in turn, of 64 blocks: 14), 23 us for 8,183 at H =
// 256.
constexpr int kJoinThreads = 1024, kJoinBlocks = 16, kJoinShort = 16;

template <int H>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(int n_tok, int V, int block, int blocks,
                                                                  const u32x2* __restrict__ items,
                                                                  const float* __restrict__ part,
                                                                  float* __restrict__ dtable) {
  constexpr int L = H / 8, G = kJoinThreads / L;
  __shared__ __attribute__((aligned(16))) float share[G][H];
  __shared__ int is_long[kJoinBlocks];
  const int grp = threadIdx.x / L, h = 8 * (threadIdx.x % L);
  const int b0 = blockIdx.x * kJoinBlocks;
  if (threadIdx.x < kJoinBlocks) is_long[threadIdx.x] = 0;
  __syncthreads();
  auto first = [&](long b) { return items[b * block].x; };   // token at the start of block b < blocks
  for (int b = b0 + grp; b < min(b0 + kJoinBlocks, blocks - 1); b += G) {
    // whether the run at the end of block b goes on and began in it
    const long far = min((long)b + kJoinShort + 1, (long)blocks - 1);
    const uint32_t key = first(b + 1), last = items[((long)b + 1) * block - 1].x, start = first(b),
                   prev = items[max((long)b * block - 1, 0l)].x, farkey = first(far);
    if (key >= (uint32_t)V || last != key || (start == key && b > 0 && prev == key)) continue;
    const bool far_too = b + kJoinShort + 1 < blocks && farkey == key;
    if (far_too != (blockIdx.y == 1)) continue;
    if (far_too) {
      if (h == 0) is_long[b - b0] = 1;
      continue;
    }
    constexpr int U = 6;   // blocks' keys and shares in flight
    float acc[8];
    load8f<float>(part + ((size_t)2 * b + 1) * H + h, acc);
    bool open = true;
    for (long j = b + 1; open; j += U) {
      float w[U][8];
      uint32_t k[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long ju = min(j + u, (long)blocks - 1);
        k[u] = j + u < blocks ? first(ju) : ~0u;
        load8f<float>(part + (size_t)2 * ju * H + h, w[u]);   // not of this run where the key differs: unused
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        open = open && k[u] == key;
        if (open) {
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] += w[u][i];
        }
      }
    }
    add_row(dtable + (size_t)key * H + h, acc);
  }
  if (blockIdx.y == 0) return;
  __syncthreads();
  for (int i = 0; i < kJoinBlocks; ++i) {   // at most one in kJoinShort blocks begins a long run
    if (is_long[i] == 0) continue;
    const int b = b0 + i;
    const uint32_t key = first(b + 1);
    int lo = b + kJoinShort + 1, len = blocks - lo;   // the run's last block lies in lo .. lo + len - 1
    while (len > 1) {                                 // kJoinThreads probes a round
      const int step = (len + kJoinThreads - 1) / kJoinThreads;
      const long j = lo + (long)(threadIdx.x + 1) * step;
      const int same = __syncthreads_count(j < (long)lo + len && first(j) == key);
      lo += same * step;
      len = min(step, blocks - lo);
    }
    float acc[8] = {}, v[8];
    if (grp == 0) load8f<float>(part + ((size_t)2 * b + 1) * H + h, acc);
#pragma unroll 4
    for (long j = b + 1 + grp; j <= lo; j += G) {
      load8f<float>(part + (size_t)2 * j * H + h, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += v[i];
    }
    store8f(&share[grp][h], acc);
    __syncthreads();
    for (int half = G / 2; half >= 1; half /= 2) {
      if (grp < half) {
        load8f<float>(&share[grp][h], acc);
        load8f<float>(&share[grp + half][h], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += v[i];
        store8f(&share[grp][h], acc);
      }
      __syncthreads();
    }
    if (grp == 0) {
      load8f<float>(&share[0][h], acc);
      add_row(dtable + (size_t)key * H + h, acc);
    }
    __syncthreads();
  }
}

}  // namespace dev

namespace {
// Items of a chunk: enough workgroups first, then few shares to join.
int run_chunk(int H, int n_tok) {
  const int groups = dev::kEmbThreads / (H / 8);
  const long c = ((long)n_tok + 1024L * groups - 1) / (1024L * groups);
  return c < 4 ? 4 : c > 32 ? 32 : (int)((c + 3) / 4 * 4);
}

struct EmbedLayout {
  size_t a, b, count, total, part, bytes;
  int tiles, chunk, block, blocks;   // sort tiles; items of a chunk and of a block of the runs kernel
};
EmbedLayout embed_layout(int H, int n_tok) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  EmbedLayout l;
  l.tiles = (int)(((long)n_tok + dev::kSortTile - 1) / dev::kSortTile);
  l.chunk = run_chunk(H, n_tok);
  l.block = l.chunk * (dev::kEmbThreads / (H / 8));
  l.blocks = (int)(((long)n_tok + l.block - 1) / l.block);
  l.a = 0;
  l.b = up((size_t)n_tok * 8);
  l.count = l.b + up((size_t)n_tok * 8);
  l.total = l.count + up((size_t)dev::kDigits * l.tiles * 4);
  l.part = l.total + up((size_t)dev::kDigits * 4);
  l.bytes = l.part + up((size_t)2 * l.blocks * H * 4);
  return l;
}

template <typename S, int H>
hipError_t embed_bwd_h(int n, int V, const int32_t* tok_ptr, const int32_t* tok, int n_tok, float scale, int mean,
                       const float* factor, const Dropout& d, const void* grad, float* dtable, char* ws,
                       hipStream_t st) {
  const S* dX = static_cast<const S*>(grad);
  using namespace dev;
  const EmbedLayout l = embed_layout(H, n_tok);
  u32x2 *a = reinterpret_cast<u32x2*>(ws + l.a), *b = reinterpret_cast<u32x2*>(ws + l.b);
  uint32_t *count = reinterpret_cast<uint32_t*>(ws + l.count), *total = reinterpret_cast<uint32_t*>(ws + l.total);
  float* part = reinterpret_cast<float*>(ws + l.part);
  int bits = 1;
  while (bits < 31 && (V >> bits) != 0) ++bits;   // keys 0 .. V
  const int passes = (bits + 7) / 8, per = (bits + passes - 1) / passes;
  const int few = l.tiles <= kFewTiles;
  for (int p = 0; p < passes; ++p) {
    const int shift = p * per;
    const uint32_t mask = (1u << per) - 1;
    if (p == 0) {
      hipLaunchKernelGGL(sort_count_kernel<true>, dim3(l.tiles), dim3(kSortThreads), 0, st, n_tok, n, V, tok_ptr,
                         tok, a, shift, mask, l.tiles, few, count);
    } else {
      hipLaunchKernelGGL(sort_count_kernel<false>, dim3(l.tiles), dim3(kSortThreads), 0, st, n_tok, n, V, tok_ptr,
                         tok, a, shift, mask, l.tiles, few, count);
    }
    if (!few)
      hipLaunchKernelGGL(sort_scan_kernel, dim3(kDigits), dim3(kSortThreads), 0, st, l.tiles, count, total);
    hipLaunchKernelGGL(sort_place_kernel, dim3(l.tiles), dim3(kSortThreads), 0, st, n_tok, a, b, shift, mask,
                       l.tiles, few, count, total);
    u32x2* t = a;
    a = b;
    b = t;
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  if (d.cut != 0) {
    hipLaunchKernelGGL((embed_runs_kernel<S, H, true>), dim3(l.blocks), dim3(kEmbThreads), 0, st, n_tok, n, V, l.chunk,
                       a, tok_ptr, scale, mean, factor, d, dX, dtable, part);
  } else {
    hipLaunchKernelGGL((embed_runs_kernel<S, H, false>), dim3(l.blocks), dim3(kEmbThreads), 0, st, n_tok, n, V, l.chunk,
                       a, tok_ptr, scale, mean, factor, d, dX, dtable, part);
  }
  if (l.blocks > 1)
    hipLaunchKernelGGL((embed_join_kernel<H>), dim3((l.blocks + kJoinBlocks - 1) / kJoinBlocks, 2), dim3(kJoinThreads),
                       0, st, n_tok, V, l.block, l.blocks, a, part, dtable);
  return hipGetLastError();
}
}  // namespace

size_t embed_bwd_workspace(int H, int n_tok) { return embed_layout(H, n_tok).bytes; }

hipError_t launch_embed_bwd(int n, int H, int V, const int32_t* tok_ptr, const int32_t* tok, int n_tok, float scale,
                            int mean, const Dropout& d, const float* dX, float* dtable, void* ws, hipStream_t st) {
  if (n_tok == 0 || n == 0) return hipSuccess;
  char* w = static_cast<char*>(ws);
  switch (H) {
    case 32: return embed_bwd_h<float, 32>(n, V, tok_ptr, tok, n_tok, scale, mean, nullptr, d, dX, dtable, w, st);
    case 64: return embed_bwd_h<float, 64>(n, V, tok_ptr, tok, n_tok, scale, mean, nullptr, d, dX, dtable, w, st);
    case 128: return embed_bwd_h<float, 128>(n, V, tok_ptr, tok, n_tok, scale, mean, nullptr, d, dX, dtable, w, st);
    case 256: return embed_bwd_h<float, 256>(n, V, tok_ptr, tok, n_tok, scale, mean, nullptr, d, dX, dtable, w, st);
  }
  return hipErrorInvalidValue;
}

size_t target_rows_workspace(int H, int R) { return embed_layout(H, R).bytes; }

hipError_t launch_target_rows(int R, int H, int V, const int32_t* target, const void* x, float scale,
                              const float* factor, float* dW, void* ws, hipStream_t st) {
  const Dropout none{};
  char* w = static_cast<char*>(ws);
  switch (H) {
    case 32: return embed_bwd_h<dev::bf16s, 32>(R, V, nullptr, target, R, scale, 0, factor, none, x, dW, w, st);
    case 64: return embed_bwd_h<dev::bf16s, 64>(R, V, nullptr, target, R, scale, 0, factor, none, x, dW, w, st);
    case 128: return embed_bwd_h<dev::bf16s, 128>(R, V, nullptr, target, R, scale, 0, factor, none, x, dW, w, st);
    case 256: return embed_bwd_h<dev::bf16s, 256>(R, V, nullptr, target, R, scale, 0, factor, none, x, dW, w, st);
  }
  return hipErrorInvalidValue;
}
#endif

}  // namespace ggnn
