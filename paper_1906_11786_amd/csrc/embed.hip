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

template <typename S, int H, bool BAG, bool DROP>
__global__ __launch_bounds__(kEmbThreads) void embed_kernel(int n, int V, const S* __restrict__ table,
                                                            const int32_t* __restrict__ tok_ptr,
                                                            const int32_t* __restrict__ tok, int n_tok, float scale,
                                                            int mean, Dropout d, S* __restrict__ X) {
  constexpr int L = H / 8;
  const int row = (int)(((long)blockIdx.x * kEmbThreads + threadIdx.x) / L);
  const int h = 8 * (threadIdx.x % L);
  if (row >= n) return;
  int lo, hi;
  if constexpr (BAG) {
    lo = clampi(tok_ptr[row], 0, n_tok);
    hi = clampi(tok_ptr[row + 1], lo, n_tok);
  } else {
    lo = row;
    hi = min(row + 1, n_tok);
  }
  float acc[8] = {};
  for (int k = lo; k < hi; ++k) {
    const int id = tok[k];
    if ((unsigned)id < (unsigned)V) {
      float v[8];
      load8f<S>(table + (size_t)id * H + h, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += v[i];
    }
  }
  const float c = BAG && mean && hi > lo ? scale / (float)(hi - lo) : scale;
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] *= c;
  const uint64_t e = (uint64_t)row * H + h;
  if constexpr (DROP) drop8(acc, e / 8, d);
  store8f(X + e, acc);
}

}  // namespace dev

namespace {
template <typename S, int H>
hipError_t embed_h(int n, int V, const void* table, const int32_t* tok_ptr, const int32_t* tok, int n_tok,
                   float scale, int mean, const Dropout& d, void* X, hipStream_t st) {
  const long threads = (long)n * (H / 8);
  const dim3 grid((unsigned)((threads + dev::kEmbThreads - 1) / dev::kEmbThreads)), block(dev::kEmbThreads);
#define EMBED(BAG, DROP)                                                                                       \
  hipLaunchKernelGGL((dev::embed_kernel<S, H, BAG, DROP>), grid, block, 0, st, n, V, static_cast<const S*>(table), \
                     tok_ptr, tok, n_tok, scale, mean, d, static_cast<S*>(X))
  if (tok_ptr != nullptr) {
    if (d.cut != 0) EMBED(true, true); else EMBED(true, false);
  } else {
    if (d.cut != 0) EMBED(false, true); else EMBED(false, false);
  }
#undef EMBED
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

constexpr int kSortThreads = 256, kSortWaves = kSortThreads / kWave;
constexpr int kSortPer = 8;                              // items per thread
constexpr int kSortTile = kSortThreads * kSortPer;       // items per tile
constexpr int kDigits = 256;

// Row whose list holds position k: the last i with ptr[i] <= k.
__device__ __forceinline__ int row_of(const int32_t* __restrict__ ptr, int n, int k) {
  int lo = 0, hi = n;   // ptr[lo] <= k < ptr[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (ptr[mid] <= k) lo = mid; else hi = mid;
  }
  return lo;
}

// Item k of the unsorted list: its key and row.
__device__ __forceinline__ u32x2 first_item(int k, int n, int V, const int32_t* __restrict__ tok_ptr,
                                            const int32_t* __restrict__ tok) {
  const int id = tok[k];
  uint32_t key = (unsigned)id < (unsigned)V ? (uint32_t)id : (uint32_t)V;
  int row = k;
  if (tok_ptr != nullptr) {
    if (k < tok_ptr[0] || k >= tok_ptr[n]) key = (uint32_t)V;   // no row's list holds it
    row = row_of(tok_ptr, n, k);
  }
  return u32x2{key, (uint32_t)row};
}

// Digit counts of each tile, count[digit * tiles + tile].  FIRST: the items
// are made from the token list and written to `items`.
template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(int n_tok, int n, int V,
                                                                  const int32_t* __restrict__ tok_ptr,
                                                                  const int32_t* __restrict__ tok, u32x2* items,
                                                                  int shift, uint32_t mask, int tiles,
                                                                  uint32_t* __restrict__ count) {
  __shared__ uint32_t c[kDigits];
  c[threadIdx.x] = 0;
  __syncthreads();
  const int k0 = blockIdx.x * kSortTile;
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    const int k = k0 + i * kSortThreads + threadIdx.x;
    if (k < n_tok) {
      u32x2 it;
      if constexpr (FIRST) {
        it = first_item(k, n, V, tok_ptr, tok);
        items[k] = it;
      } else {
        it = items[k];
      }
      atomicAdd(&c[(it.x >> shift) & mask], 1u);   // integers: the order does not matter
    }
  }
  __syncthreads();
  count[(size_t)threadIdx.x * tiles + blockIdx.x] = c[threadIdx.x];
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
                                                                  int tiles, const uint32_t* __restrict__ count,
                                                                  const uint32_t* __restrict__ total) {
  __shared__ uint32_t cnt[kSortWaves][kDigits];
  __shared__ uint32_t ws[kSortWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, dig = threadIdx.x;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) cnt[w][dig] = 0;
  // exclusive scan of the digit totals
  const uint32_t tot = total[dig];
  uint32_t s = tot;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t u = __shfl_up(s, o);
    if (lane >= o) s += u;
  }
  if (lane == kWave - 1) ws[wave] = s;
  __syncthreads();
  uint32_t base = s - tot + count[(size_t)dig * tiles + blockIdx.x];
  for (int w = 0; w < wave; ++w) base += ws[w];

  const int k0 = blockIdx.x * kSortTile + wave * (kSortTile / kSortWaves);
  u32x2 it[kSortPer];
  uint32_t rank[kSortPer];
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    const int k = k0 + i * kWave + lane;
    it[i] = k < n_tok ? in[k] : u32x2{~0u, 0u};
  }
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
// The sorted list is cut into chunks of `chunk` items, one group of H / 8
// lanes each.  A run inside one chunk is added to its row of the gradient
// directly.  Of a run that crosses chunks, each chunk writes its share to
// part[chunk][0] (it began before) or part[chunk][1] (it begins here), and the
// join kernel adds the shares in chunk order.

template <int H, bool DROP>
__global__ __launch_bounds__(kEmbThreads) void embed_runs_kernel(int n_tok, int V, int chunk,
                                                                 const u32x2* __restrict__ items,
                                                                 const int32_t* __restrict__ tok_ptr, float scale,
                                                                 int mean, Dropout d, const float* __restrict__ dX,
                                                                 float* __restrict__ dtable,
                                                                 float* __restrict__ part) {
  constexpr int L = H / 8;
  const int c = (int)(((long)blockIdx.x * kEmbThreads + threadIdx.x) / L);
  const int h = 8 * (threadIdx.x % L);
  const long lo = (long)c * chunk;
  if (lo >= n_tok) return;
  const int k0 = (int)lo, k1 = min(n_tok, k0 + chunk);
  uint32_t cur = items[k0].x;
  bool before = k0 > 0 && items[k0 - 1].x == cur;
  float acc[8] = {};
  auto flush = [&](bool after) {
    if (cur >= (uint32_t)V) return;
    if (before || after) {
      store8f(part + ((size_t)2 * c + (before ? 0 : 1)) * H + h, acc);
    } else {
      float* o = dtable + (size_t)cur * H + h;
      float v[8];
      load8f<float>(o, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += acc[i];
      store8f(o, v);
    }
  };
  for (int k = k0; k < k1; ++k) {
    const u32x2 it = items[k];
    if (it.x != cur) {
      flush(false);
      cur = it.x;
      before = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    }
    if (cur < (uint32_t)V) {
      const int row = (int)it.y;
      float f = scale;
      if (tok_ptr != nullptr && mean) f = scale / (float)max(tok_ptr[row + 1] - tok_ptr[row], 1);
      float v[8];
      const uint64_t e = (uint64_t)row * H + h;
      load8f<float>(dX + e, v);
      if constexpr (DROP) drop8(v, e / 8, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += f * v[i];
    }
  }
  flush(k1 < n_tok && items[k1].x == cur);
}

// One group of H / 8 lanes per chunk: adds up a run that begins in the chunk and
// leaves it.
template <int H>
__global__ __launch_bounds__(kEmbThreads) void embed_join_kernel(int n_tok, int V, int chunk,
                                                                 const u32x2* __restrict__ items,
                                                                 const float* __restrict__ part,
                                                                 float* __restrict__ dtable) {
  constexpr int L = H / 8;
  const int c = (int)(((long)blockIdx.x * kEmbThreads + threadIdx.x) / L);
  const int h = 8 * (threadIdx.x % L);
  const long lo = (long)c * chunk;
  const long end = lo + chunk;
  if (end >= n_tok) return;   // the last chunk's runs end in it
  const uint32_t key = items[end - 1].x;
  if (key >= (uint32_t)V || items[end].x != key) return;
  if (items[lo].x == key && lo > 0 && items[lo - 1].x == key) return;   // begins before
  float acc[8], v[8];
  load8f<float>(part + ((size_t)2 * c + 1) * H + h, acc);
  for (long k = end, j = c + 1; k < n_tok && items[k].x == key; k += chunk, ++j) {
    load8f<float>(part + (size_t)2 * j * H + h, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] += v[i];
  }
  float* o = dtable + (size_t)key * H + h;
  load8f<float>(o, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += acc[i];
  store8f(o, v);
}

}  // namespace dev

namespace {
constexpr int kRunChunk = 32;

struct EmbedLayout {
  size_t a, b, count, total, part, bytes;
  int tiles, chunks;
};
EmbedLayout embed_layout(int H, int n_tok) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  EmbedLayout l;
  l.tiles = (int)(((long)n_tok + dev::kSortTile - 1) / dev::kSortTile);
  l.chunks = (int)(((long)n_tok + kRunChunk - 1) / kRunChunk);
  l.a = 0;
  l.b = up((size_t)n_tok * 8);
  l.count = l.b + up((size_t)n_tok * 8);
  l.total = l.count + up((size_t)dev::kDigits * l.tiles * 4);
  l.part = l.total + up((size_t)dev::kDigits * 4);
  l.bytes = l.part + up((size_t)2 * l.chunks * H * 4);
  return l;
}

template <int H>
hipError_t embed_bwd_h(int n, int V, const int32_t* tok_ptr, const int32_t* tok, int n_tok, float scale, int mean,
                       const Dropout& d, const float* dX, float* dtable, char* ws, hipStream_t st) {
  using namespace dev;
  const EmbedLayout l = embed_layout(H, n_tok);
  u32x2 *a = reinterpret_cast<u32x2*>(ws + l.a), *b = reinterpret_cast<u32x2*>(ws + l.b);
  uint32_t *count = reinterpret_cast<uint32_t*>(ws + l.count), *total = reinterpret_cast<uint32_t*>(ws + l.total);
  float* part = reinterpret_cast<float*>(ws + l.part);
  int bits = 1;
  while (bits < 31 && (V >> bits) != 0) ++bits;   // keys 0 .. V
  const int passes = (bits + 7) / 8, per = (bits + passes - 1) / passes;
  for (int p = 0; p < passes; ++p) {
    const int shift = p * per;
    const uint32_t mask = (1u << per) - 1;
    if (p == 0) {
      hipLaunchKernelGGL(sort_count_kernel<true>, dim3(l.tiles), dim3(kSortThreads), 0, st, n_tok, n, V, tok_ptr,
                         tok, a, shift, mask, l.tiles, count);
    } else {
      hipLaunchKernelGGL(sort_count_kernel<false>, dim3(l.tiles), dim3(kSortThreads), 0, st, n_tok, n, V, tok_ptr,
                         tok, a, shift, mask, l.tiles, count);
    }
    hipLaunchKernelGGL(sort_scan_kernel, dim3(kDigits), dim3(kSortThreads), 0, st, l.tiles, count, total);
    hipLaunchKernelGGL(sort_place_kernel, dim3(l.tiles), dim3(kSortThreads), 0, st, n_tok, a, b, shift, mask,
                       l.tiles, count, total);
    u32x2* t = a;
    a = b;
    b = t;
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  const dim3 grid((unsigned)(((long)l.chunks * (H / 8) + kEmbThreads - 1) / kEmbThreads));
  if (d.cut != 0) {
    hipLaunchKernelGGL((embed_runs_kernel<H, true>), grid, dim3(kEmbThreads), 0, st, n_tok, V, kRunChunk, a,
                       tok_ptr, scale, mean, d, dX, dtable, part);
  } else {
    hipLaunchKernelGGL((embed_runs_kernel<H, false>), grid, dim3(kEmbThreads), 0, st, n_tok, V, kRunChunk, a,
                       tok_ptr, scale, mean, d, dX, dtable, part);
  }
  hipLaunchKernelGGL((embed_join_kernel<H>), grid, dim3(kEmbThreads), 0, st, n_tok, V, kRunChunk, a, part, dtable);
  return hipGetLastError();
}
}  // namespace

size_t embed_bwd_workspace(int H, int n_tok) { return embed_layout(H, n_tok).bytes; }

hipError_t launch_embed_bwd(int n, int H, int V, const int32_t* tok_ptr, const int32_t* tok, int n_tok, float scale,
                            int mean, const Dropout& d, const float* dX, float* dtable, void* ws, hipStream_t st) {
  if (n_tok == 0 || n == 0) return hipSuccess;
  char* w = static_cast<char*>(ws);
  switch (H) {
    case 32: return embed_bwd_h<32>(n, V, tok_ptr, tok, n_tok, scale, mean, d, dX, dtable, w, st);
    case 64: return embed_bwd_h<64>(n, V, tok_ptr, tok, n_tok, scale, mean, d, dX, dtable, w, st);
    case 128: return embed_bwd_h<128>(n, V, tok_ptr, tok, n_tok, scale, mean, d, dX, dtable, w, st);
    case 256: return embed_bwd_h<256>(n, V, tok_ptr, tok, n_tok, scale, mean, d, dX, dtable, w, st);
  }
  return hipErrorInvalidValue;
}
#endif

}  // namespace ggnn
