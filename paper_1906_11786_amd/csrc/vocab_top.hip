// The best entries of chosen rows over a vocabulary, under rules, without the
// logits in memory.
//
//   z_iv = x_i . w_v + b_v, changed by the rules (include/ggnn.h)
//   the K largest z_iv of each row, equal ones by the lower entry, and
//   lse_i = log sum_v exp(z_iv / temperature)
//
// The entries are cut into blocks of 16.  A first pass forms all logits on the
// matrix cores and keeps each block's maximum (and the running sum of the
// exponentials).  An entry among a row's K best lies in one of the K blocks that are
// first by (maximum descending, block ascending): each block before its own holds
// an entry that comes before it.  So a second pass picks those blocks, forms their
// 16 K logits again and picks the entries.  The maxima are 1 / 16 of the logits.
//
// Entries that a row's lists name (seen before, or with a bias) are changed one by
// one: the first pass leaves them out, as it leaves out what a mask excludes, and the
// second adds them, changed, to its candidates and to the sum.
#include "vocab_tile.h"

namespace ggnn {
namespace dev {

constexpr int kTopMost = 64;   // K at most: a lane holds one of a wave's best
constexpr int kTopBlock = 16;

// 32-row tiles of a wave: an LDS fragment serves both of two.  (float32 at H = 256
// has no registers for a second one's planes.)
template <typename S>
constexpr int top_tiles(int H) {
  return sizeof(S) == 4 && H >= 256 ? 1 : 2;
}
// Waves of a SIMD, by the registers of a wave's rows and at H >= 128 the buffers.
template <typename S>
constexpr int top_waves(int H) {
  if (sizeof(S) == 4) return H >= 128 ? 1 : H == 64 ? 2 : 3;
  return H >= 256 ? 1 : H == 128 ? 2 : H == 64 ? 3 : 4;
}

// A 32 x 32 tile of logits has entries as its rows.  Entry r of a tile is put on row
// top_row(r), so that a lane (lanes 32 g .. 32 g + 31) holds entries 16 g .. 16 g + 15, one
// block, in order.
__device__ __forceinline__ int top_row(int r) { return 8 * ((r >> 2) & 3) + 4 * (r >> 4) + (r & 3); }
__device__ __forceinline__ int top_entry(int i) { return 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3); }

// As stage_tile, with the places of a row's pieces by its row in the tile of logits
// (the rows that sixteen lanes read at once).
template <int H, int NP, int T>
__device__ __forceinline__ void stage_entries(const bf16s* __restrict__ src, size_t plane, long row0, long last,
                                              uint32_t lds, int wave, int lane) {
  constexpr int CPR = H / 8, EACH = T * CPR / 64, PIECES = NP * EACH;
#pragma unroll
  for (int p = 0; p < (PIECES + kVocWaves - 1) / kVocWaves; ++p) {
    const int piece = p * kVocWaves + wave, q = piece % EACH * 64 + lane;
    if (PIECES % kVocWaves != 0 && piece >= PIECES) break;
    const int r = q / CPR, c = (q % CPR) ^ swz<H>(top_row(r % 32));
    const long row = row0 + r < last ? row0 + r : last;
    dma16(src + piece / EACH * plane + row * H + 8 * c,
          __builtin_amdgcn_readfirstlane(lds + (uint32_t)piece * 1024u));
  }
}

// Bit masks over the entries, one a row: index of[r] (r where of is NULL); one
// outside [0, n) excludes nothing.
struct RowMask {
  const uint32_t* bits;
  const int32_t* of;
  int n, words;
  __device__ __forceinline__ const uint32_t* row(int r, int R) const {
    if (bits == nullptr || r >= R) return nullptr;
    const int i = of != nullptr ? of[r] : r;
    return (unsigned)i < (unsigned)n ? bits + (size_t)i * words : nullptr;
  }
};
// -inf where the entry's bit is 0; a: 16 logits, w: their bits from bit 0 on.
__device__ __forceinline__ void take_out(f32x16& a, uint32_t w) {
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)w, j, 1);
    a[j] = __uint_as_float((__float_as_uint(a[j]) & m) | (0xFF800000u & ~m));
  }
}
__device__ __forceinline__ float max16(const f32x16& a) {
  float t = a[0];
#pragma unroll
  for (int j = 1; j < 16; ++j) t = fmaxf(t, a[j]);
  return t;
}

// Running maximum (times its factor k) and sum of one row's exponentials.
struct RowSum {
  float m, k, l;
};

// First pass.  A workgroup holds 128 NT rows, NT tiles of 32 a wave, and walks a share of
// the vocabulary in tiles staged in LDS, dealt and buffered as in the losses' rows
// pass (csrc/vocab.hip).  Writes block maxima to bmax [R][nbs] and, where LSE, (m, l)
// of a share to pm, pl [slot][128 NT].
template <typename S, int H, bool LSE, bool MASK>
__global__ __launch_bounds__(kVocThreads, top_waves<S>(H)) void vocab_max_kernel(
    int n_nodes, int R, int V, Deal deal, Temper te, const S* __restrict__ X, const bf16s* __restrict__ W,
    const float* __restrict__ bias, const int32_t* __restrict__ node, RowMask rm, float* __restrict__ bmax, int nbs,
    float* __restrict__ pm, float* __restrict__ pl) {
  constexpr int T = voc_tile<S>(), NP = voc_planes<S>(), NT = top_tiles<S>(H), SUB = T / 32, NS = H / 16, NF = NS * NP;
  constexpr int kAhead = NF < 8 ? NF : 8, VS = NS < 8 ? NS : 8;
  constexpr uint32_t ROW = H * 2, PLANE = T * ROW, TILE = NP * PLANE;
  __shared__ __attribute__((aligned(1024))) bf16s tile[kVocBufs][NP * T * H];
  __shared__ __attribute__((aligned(16))) float tb[kVocBufs][T];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = lane / 32;
  const uint32_t lds0 = (uint32_t)(uintptr_t)tile[0];
  typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;

  float nb = 0.f;
  Run run;
  Dealt dealt(deal, blockIdx.x);
  for (int round = 0; dealt.next(deal, blockIdx.x, &run); ++round) {
    const int t0 = run.t0, t1 = run.t1;
    const int row0 = run.i * (kVocRows * NT) + wave * 32 * NT + lane % 32;   // of the lane's first tile
    bf16x8 x[NT][NP][NS];
    RowSum sum[NT];
    const uint32_t* mrow[NT];
    uint32_t word[NT][SUB], next_word[NT][SUB];   // mask bits of the tile in use and of the one on its way
    auto fetch = [&](int t, int buf) {   // start the copies of tile t < t1
      stage_entries<H, NP, T>(W, (size_t)V * H, (long)t * T, V - 1, lds0 + (uint32_t)buf * TILE, wave, lane);
      // (raw values: a use here would wait for the copies too)
      if (bias != nullptr && threadIdx.x < T) nb = bias[min(t * T + (int)threadIdx.x, V - 1)];
      if constexpr (MASK) {
#pragma unroll
        for (int a = 0; a < NT; ++a)
#pragma unroll
          for (int i = 0; i < SUB; ++i)
            next_word[a][i] = mrow[a] != nullptr ? mrow[a][min(t * SUB + i, rm.words - 1)] : ~0u;
      }
    };
    auto land = [&](int t, int buf) {   // and wait for those started last, of tile t
      if (threadIdx.x < T)
        tb[buf][threadIdx.x] = t * T + (int)threadIdx.x >= V || nb <= kMaskedBias ? -INFINITY : nb;
      if constexpr (MASK) {
#pragma unroll
        for (int a = 0; a < NT; ++a)
#pragma unroll
          for (int i = 0; i < SUB; ++i) word[a][i] = next_word[a][i] >> (16 * g);
      }
      wait_copies<0>();
      __syncthreads();
    };
    if (round > 0) __syncthreads();   // every wave has left the buffers of the run before
#pragma unroll
    for (int a = 0; a < NT; ++a) mrow[a] = MASK ? rm.row(row0 + 32 * a, R) : nullptr;
    uint32_t as[VS];   // LDS addresses of the fragments; the other ones lie 256 bytes, rows or planes on
#pragma unroll
    for (int k = 0; k < VS; ++k)
      as[k] = lds0 + (uint32_t)top_entry(lane % 32) * ROW + 16u * ((2 * k + g) ^ swz<H>(lane % 32));
    bf16x8 f[NF];   // at most kAhead are alive
    auto read = [&](int n, int rs) {   // fragment n of the tile rows from rs on: k step n / NP, plane n % NP
      const int kk = n / NP;
      f[n] = __builtin_bit_cast(bf16x8, *(lds_u32x4*)(as[kk % VS] + 256u * (kk / VS) + (uint32_t)rs * ROW +
                                                      (uint32_t)(n % NP) * PLANE));
    };
    f32x16 s[NT];
    float top[NT];
    auto start = [&](f32x16 (&acc)[NT], int buf, int rs) {   // biases of a tile's entries
      f32x16 b;
#pragma unroll
      for (int j4 = 0; j4 < 4; ++j4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(tb[buf] + rs + 16 * g + 4 * j4);
#pragma unroll
        for (int i = 0; i < 4; ++i) b[4 * j4 + i] = v[i];
      }
#pragma unroll
      for (int a = 0; a < NT; ++a) acc[a] = b;
    };
    // acc += logits of the tile rows from rs on; work(i), i < 16 NT, is done alongside
    auto logits = [&](f32x16 (&acc)[NT], int rs, auto work) {
#pragma unroll
      for (int n = 0; n < kAhead; ++n) read(n, rs);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < NF; ++n) {
        if (n + kAhead < NF) read(n + kAhead, rs);
#pragma unroll
        for (int b = 0; b + n % NP < NP; ++b)
#pragma unroll
          for (int a = 0; a < NT; ++a) mma32(acc[a], f[n], x[a][b][n / NP]);
#pragma unroll
        for (int i = n * 16 * NT / NF; i < (n + 1) * 16 * NT / NF; ++i) work(i);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto finish = [&](f32x16 (&acc)[NT], float (&t)[NT], int sub) {
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        if constexpr (MASK) take_out(acc[a], word[a][sub]);
        t[a] = max16(acc[a]);
      }
    };
    // Block maxima: four tiles' are kept, then a row's eight blocks are stored as 32 bytes
    // by its two lanes; at a run's ends, one by one.
    float kept[NT][4];
    int n_kept = 0;
    auto store_kept = [&](int last, bool whole) {   // `last`: tile of kept[.][3]
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        const int r = row0 + 32 * a;
        if (whole) {
          const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(kept[a][0]), __float_as_uint(kept[a][2]),
                                                          false, false);
          const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(kept[a][1]), __float_as_uint(kept[a][3]),
                                                          false, false);
          if (r < R)
            *reinterpret_cast<u32x4*>(bmax + (size_t)r * nbs + 2 * (last - 3) + 4 * g) = u32x4{u[0], u[1], w[0], w[1]};
        } else if (r < R) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < n_kept) bmax[(size_t)r * nbs + 2 * (last - e) + g] = kept[a][3 - e];
        }
      }
      n_kept = 0;
    };
    auto keep = [&](int t) {   // maxima of tile t
#pragma unroll
      for (int a = 0; a < NT; ++a) {
#pragma unroll
        for (int e = 0; e < 3; ++e) kept[a][e] = kept[a][e + 1];
        kept[a][3] = top[a];
      }
      ++n_kept;
      if (t % 4 == 3) store_kept(t, n_kept == 4);
    };

    int buf = 0;
    fetch(t0, 0);
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      load_planes<S, H>(x[a], X, row_node(node, row0 + 32 * a, R, n_nodes), lane);
      sum[a] = RowSum{kNoMax, te.near, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) kept[a][e] = -INFINITY;
    }
    land(t0, 0);
    if (t0 + 1 < t1) fetch(t0 + 1, 1);
    start(s, 0, 0);
    logits(s, 0, [](int) {});
    finish(s, top, 0);
    for (int t = t0; t < t1; ++t) {
      const int nbuf = next_buf(buf);
#pragma unroll
      for (int r0 = 0; r0 < T; r0 += 32) {
        const bool last = r0 + 32 >= T;
        const int rs = last ? 0 : r0 + 32;   // of the next tile (after the last one: of what the buffer holds, not used)
        if (last) {
          land(t + 1, nbuf);
          if (t + 2 < t1) fetch(t + 2, next_buf(nbuf));
#pragma unroll
          for (int k = 0; k < VS; ++k) as[k] += buf_step<TILE>(nbuf);
        }
        f32x16 sn[NT];
        start(sn, last ? nbuf : buf, rs);
        keep(t * SUB + r0 / 32);
        if constexpr (LSE) {
          // (the maximum follows where it would grow by more than 2^8, as in the losses' rows pass)
          bool grows = false;
#pragma unroll
          for (int a = 0; a < NT; ++a) grows |= top[a] * sum[a].k > sum[a].m + 8.f;
          if (__ballot(grows)) {
#pragma unroll
            for (int a = 0; a < NT; ++a) {
              const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top[a]), __float_as_uint(top[a]), false,
                                                               false);
              const float z = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])), kn = exponent_factor(z, te);
              const float mn = fmaxf(sum[a].m, z * kn);
              if (mn > sum[a].m) sum[a].k = kn;
              sum[a].l *= __builtin_amdgcn_exp2f(sum[a].m - mn);
              sum[a].m = mn;
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          logits(sn, rs, [&](int i) {
            const int a = i / 16, j = i % 16;
            sum[a].l += __builtin_amdgcn_exp2f(fmaf(s[a][j], sum[a].k, -sum[a].m));
          });
        } else {
          logits(sn, rs, [](int) {});
        }
        finish(sn, top, last ? 0 : r0 / 32 + 1);
#pragma unroll
        for (int a = 0; a < NT; ++a) s[a] = sn[a];
      }
      buf = nbuf;
    }
    if (n_kept > 0) store_kept(t1 * SUB - 1, false);
    if constexpr (LSE) {
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        const float l = sum[a].l + __shfl_xor(sum[a].l, 32);
        const size_t at = (size_t)run.slot * (kVocRows * NT) + wave * 32 * NT + 32 * a + lane % 32;
        if (g == 0) {
          pm[at] = sum[a].m;
          pl[at] = l;
        }
      }
    }
  }
}

// First pass for at most 32 NT rows: every wave holds the same rows and takes `per`
// tiles of 32 entries, read straight from memory, since no other wave needs them.
template <typename S, int H, int NT, bool LSE, bool MASK>
__global__ __launch_bounds__(kVocThreads) void vocab_max_few_kernel(
    int n_nodes, int R, int V, int per, Temper te, const S* __restrict__ X, const S* __restrict__ W,
    const float* __restrict__ bias, const int32_t* __restrict__ node, RowMask rm, float* __restrict__ bmax, int nbs,
    float* __restrict__ pm, float* __restrict__ pl) {
  const int lane = threadIdx.x % kWave, g = lane / 32, r = lane % 32;
  const int split = blockIdx.x * kVocWaves + threadIdx.x / kWave;
  const int tiles = (V + 31) / 32, t0 = split * per, t1 = min(tiles, t0 + per);
  frag_t<S> xf[NT][H / 16];
  RowSum sum[NT];
  const uint32_t* mrow[NT];
#pragma unroll
  for (int a = 0; a < NT; ++a) {
    load_row<S, H>(xf[a], X, row_node(node, r + 32 * a, R, n_nodes), lane);
    mrow[a] = MASK ? rm.row(r + 32 * a, R) : nullptr;
    sum[a] = RowSum{kNoMax, te.near, 0.f};
  }
  for (int t = t0; t < t1; ++t) {
    frag_t<S> wf[H / 16];
    load_row<S, H>(wf, W, min(t * 32 + top_entry(r), V - 1), lane);
    f32x16 b;
#pragma unroll
    for (int j = 0; j < 16; ++j) b[j] = entry_bias(bias, t * 32 + 16 * g + j, V);
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      uint32_t w = ~0u;
      if (MASK && mrow[a] != nullptr) w = mrow[a][t] >> (16 * g);
      f32x16 s = b;
#pragma unroll
      for (int kk = 0; kk < H / 16; ++kk) mma32(s, wf[kk], xf[a][kk]);
      if constexpr (MASK) take_out(s, w);
      const float top = max16(s);
      if (r + 32 * a < R) bmax[(size_t)(r + 32 * a) * nbs + 2 * t + g] = top;
      if constexpr (LSE) {
        RowSum& q = sum[a];
        const float kn = exponent_factor(top, te), mn = fmaxf(q.m, top * kn);
        if (mn > q.m) q.k = kn;
        q.l *= __builtin_amdgcn_exp2f(q.m - mn);
        q.m = mn;
#pragma unroll
        for (int j = 0; j < 16; ++j) q.l += __builtin_amdgcn_exp2f(fmaf(s[j], q.k, -q.m));
      }
    }
  }
  if constexpr (LSE) {
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      const float m = sum[a].m, m2 = __shfl_xor(m, 32), l2 = __shfl_xor(sum[a].l, 32), mn = fmaxf(m, m2);
      const float l = sum[a].l * __builtin_amdgcn_exp2f(m - mn) + l2 * __builtin_amdgcn_exp2f(m2 - mn);
      const size_t at = (size_t)split * (32 * NT) + 32 * a + r;
      if (g == 0) {
        pm[at] = mn;
        pl[at] = l;
      }
    }
  }
}

// ---- rules: the entries that a row's lists name ------------------------------
//
// One workgroup per row finds the different entries of its lists, how often each was
// seen and the sum of its biases, writes them at the place of their first listing
// (the other places: -1, so the result does not depend on the order of the atomics
// below, which count and take minima) and takes them out of the row's mask.  Entries
// are held in a table in LDS: a hash table while the lists are short; else the
// vocabulary is passed over in parts whose entries have a place each.
constexpr int kTable = 2048, kHashed = kTable / 2;   // places; longest lists that are hashed

struct Listing {
  const int32_t *seen_ptr, *seen, *add_ptr, *add;
  const float* value;
  int n_seen, n_add;
};
// Row r's part [lo, hi) of a list.
__device__ __forceinline__ void list_range(const int32_t* ptr, int n, int r, int& lo, int& hi) {
  lo = ptr != nullptr ? min(max(ptr[r], 0), n) : 0;
  hi = ptr != nullptr ? min(max(ptr[r + 1], lo), n) : 0;
}

template <typename S>   // (the same for both types)
__global__ __launch_bounds__(kVocThreads) void vocab_rules_kernel(int R, int V, Listing list, RowMask rm, int words,
                                                                  uint32_t* __restrict__ out,
                                                                  int32_t* __restrict__ ent_id,
                                                                  uint32_t* __restrict__ ent_count,
                                                                  float* __restrict__ ent_add) {
  __shared__ int key[kTable];
  __shared__ uint32_t first[kTable], seen[kTable], adds[kTable];
  __shared__ float value[kTable];
  const int r = blockIdx.x;
  int slo, shi, alo, ahi;
  list_range(list.seen_ptr, list.n_seen, r, slo, shi);
  list_range(list.add_ptr, list.n_add, r, alo, ahi);
  const int n_seen = shi - slo, n = n_seen + ahi - alo;
  const size_t at = (size_t)slo + alo;   // the row's places
  const uint32_t* mask = rm.row(r, R);
  uint32_t* mine = out + (size_t)r * words;
  const bool hashed = n <= kHashed;
  int bits = 6;
  while (hashed && (1 << bits) < 2 * n) ++bits;
  const int size = hashed ? 1 << bits : kTable;
  const long parts = hashed ? 1 : ((long)V + kTable - 1) / kTable;
  auto token = [&](int i) { return i < n_seen ? list.seen[slo + i] : list.add[alo + i - n_seen]; };
  for (long p = blockIdx.y; p < parts; p += gridDim.y) {
    const int lo = hashed ? 0 : (int)(p * kTable), hi = hashed ? V : (int)min((long)V, (long)lo + kTable);
    for (int i = threadIdx.x; i < size; i += kVocThreads) {
      key[i] = -1;
      first[i] = ~0u;
      seen[i] = adds[i] = 0;
    }
    for (int w = lo / 32 + threadIdx.x; w < (hi + 31) / 32; w += kVocThreads) mine[w] = mask != nullptr ? mask[w] : ~0u;
    __threadfence_block();
    __syncthreads();
    auto place = [&](int id) {   // of an entry that the table has
      if (!hashed) return id - lo;
      uint32_t h = (uint32_t)id * 0x9E3779B1u >> (32 - bits);
      while (key[h] != id) h = (h + 1) & (size - 1);
      return (int)h;
    };
    for (int i = threadIdx.x; i < n; i += kVocThreads) {
      const int id = token(i);
      if (id < lo || id >= hi) continue;
      int h = id - lo;
      if (hashed) {   // at most half of the places are taken, so a free one is found
        h = (int)((uint32_t)id * 0x9E3779B1u >> (32 - bits));
        for (;;) {
          const int old = atomicCAS(&key[h], -1, id);
          if (old == -1 || old == id) break;
          h = (h + 1) & (size - 1);
        }
      }
      atomicMin(&first[h], (uint32_t)i);
      if (i < n_seen) {
        atomicAdd(&seen[h], 1u);
      } else {
        atomicAdd(&adds[h], 1u);
        value[h] = list.value[alo + i - n_seen];   // (used where it is the only one)
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kVocThreads) {
      const int id = token(i);
      const bool known = id >= 0 && id < V;
      if (known ? id < lo || id >= hi : p != 0) continue;   // another part's
      int e = -1;
      if (known) {
        const int h = place(id);
        if (first[h] == (uint32_t)i && (mask == nullptr || (mask[id / 32] >> (id % 32) & 1))) {
          e = id;
          float a = adds[h] == 1 ? value[h] : 0.f;
          if (adds[h] > 1) {   // in list order
            for (int k = alo; k < ahi; ++k)
              if (list.add[k] == id) a += list.value[k];
          }
          ent_count[at + i] = seen[h];
          ent_add[at + i] = a;
          atomicAnd(&mine[id / 32], ~(1u << (id % 32)));
        }
      }
      ent_id[at + i] = e;
    }
    __syncthreads();
  }
}

// ---- second pass -----------------------------------------------------------

// A candidate as one number that orders by value, then by the lower index; 0: none
// (-inf and NaN too).
typedef unsigned long long pick_t;
__device__ __forceinline__ pick_t key_of(float z, uint32_t index) {
  z += 0.f;   // -0 counts as 0
  const uint32_t u = __float_as_uint(z);
  return z > -INFINITY ? (pick_t)(u ^ (u >> 31 ? ~0u : 0x80000000u)) << 32 | (uint32_t)~index : 0;
}
__device__ __forceinline__ uint32_t key_index(pick_t k) { return ~(uint32_t)k; }
__device__ __forceinline__ float key_value(pick_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return k == 0 ? -INFINITY : __uint_as_float(u ^ (u >> 31 ? 0x80000000u : ~0u));
}
__device__ __forceinline__ pick_t key_at(pick_t k, int lane) {   // lane: the same in the whole wave
  return (pick_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}

// The 64 largest keys seen, in descending order over the lanes.
struct Best {
  pick_t k = 0;
  // Bitonic steps over lanes at distances d, d / 2, ... 1 within groups of `group` lanes,
  // descending where the group's number is even.
  static __device__ __forceinline__ void steps(pick_t& v, int group, int d, int lane) {
    for (; d >= 1; d /= 2) {
      const pick_t o = __shfl_xor(v, d);
      const bool low = (lane & d) == 0, down = (lane & group) == 0;
      v = low == down ? max(v, o) : min(v, o);
    }
  }
  static __device__ __forceinline__ void sort(pick_t& v, int lane) {
    for (int group = 2; group <= kWave; group *= 2) steps(v, group, group / 2, lane);
  }
  // Joins another descending list.
  __device__ __forceinline__ void join(pick_t other, int lane) {
    k = max(k, __shfl(other, kWave - 1 - lane));
    steps(k, kWave, kWave / 2, lane);
  }
  // Adds one key a lane; K: how many of the largest matter.
  __device__ __forceinline__ void add(pick_t c, int K, int lane) {
    pick_t least = key_at(k, K - 1);
    uint64_t in = __ballot(c > least);
    if (__popcll(in) > 6) {   // about where sorting all costs less than one at a time
      sort(c, lane);
      join(c, lane);
      return;
    }
    while (in != 0) {
      const pick_t one = key_at(c, (int)__builtin_ctzll(in));
      in &= in - 1;
      const int place = __popcll(__ballot(k > one));
      const pick_t up = __shfl_up(k, 1);
      k = lane < place ? k : lane == place ? one : up;
    }
  }
};

struct TopRows {   // arguments of the second pass
  int n_nodes, R, V, K, nbs, splits, share_rows;
  Deal deal;
  Temper te;
  const float* bias;
  const int32_t* node;
  RowMask rm;
  const float *bmax, *pm, *pl;
  Listing list;
  const int32_t* ent_id;
  const uint32_t* ent_count;
  const float* ent_add;
  float repetition, presence, frequency;
  int32_t* top;
  float *logit, *lse;
};

// Second pass: WPR waves per row (1: four rows a workgroup).  Blocks are picked from
// their maxima, 64 entries at a time are formed as four 16 x 16 tiles (the state in all
// columns, so that each lane finds one entry's logit among its accumulators).
template <typename S, int H, int WPR>
__global__ __launch_bounds__(WPR == 1 ? kVocThreads : kWave* WPR) void vocab_pick_kernel(TopRows c,
                                                                                        const S* __restrict__ X,
                                                                                        const S* __restrict__ W) {
  __shared__ pick_t lists[WPR == 1 ? 1 : WPR][kWave];
  __shared__ float sums[WPR][4];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = WPR == 1 ? blockIdx.x * kVocWaves + wave : blockIdx.x, w0 = WPR == 1 ? 0 : wave;
  if (r >= c.R) return;   // whole waves, and where a workgroup shares a row all of it, leave together
  const int n = row_node(c.node, r, c.R, c.n_nodes), q = lane % 16, kg = lane / 16;
  frag_t<S> x[H / 32];
#pragma unroll
  for (int kk = 0; kk < H / 32; ++kk) {
    if (n >= 0) x[kk] = load8(X + (size_t)n * H + 32 * kk + 8 * kg);
    else x[kk] = frag_t<S>{};
  }
  const uint32_t* mrow = c.rm.row(r, c.R);
  // Joins the waves' lists; every wave has the result.
  auto share = [&](Best& b) {
    if constexpr (WPR > 1) {
      lists[wave][lane] = b.k;
      __syncthreads();
      for (int half = WPR / 2; half >= 1; half /= 2) {
        if (wave < half) {
          b.join(lists[wave + half][lane], lane);
          lists[wave][lane] = b.k;
        }
        __syncthreads();
      }
      b.k = lists[0][lane];
      __syncthreads();
    }
  };

  Best blocks;
  const int nb = (c.V + kTopBlock - 1) / kTopBlock;
  constexpr int U = 4;
  for (int b0 = w0 * kWave; b0 < nb; b0 += WPR * kWave * U) {
    float m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int b = b0 + u * WPR * kWave + lane;
      m[u] = b < nb ? c.bmax[(size_t)r * c.nbs + b] : -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) blocks.add(key_of(m[u], (uint32_t)(b0 + u * WPR * kWave + lane)), c.K, lane);
  }
  share(blocks);

  // 64 entries, entry e of tile u given by lanes e of id[u] (negative: none); each lane
  // gets the logit of entry 4 kg + q % 4 of tile q / 4
  auto form = [&](const int (&id)[4]) {
    f32x4 acc[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      acc[u] = f32x4{};
      frag_t<S> w[H / 32];
#pragma unroll
      for (int kk = 0; kk < H / 32; ++kk) w[kk] = load8(W + (size_t)max(id[u], 0) * H + 32 * kk + 8 * kg);
#pragma unroll
      for (int kk = 0; kk < H / 32; ++kk) mma(acc[u], w[kk], x[kk]);
    }
    float z = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (q == 4 * u + j) z = acc[u][j];
    return z;
  };
  Best best;
  for (int b0 = 4 * w0; b0 < c.K; b0 += 4 * WPR) {
    int id[4], mine = -1;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const pick_t k = key_at(blocks.k, min(b0 + u, kWave - 1));
      const int at = b0 + u < c.K && k != 0 ? (int)key_index(k) * kTopBlock : -1;
      id[u] = at >= 0 && at + q < c.V ? at + q : -1;
      if (q / 4 == u && at >= 0 && at + 4 * kg + q % 4 < c.V) mine = at + 4 * kg + q % 4;
    }
    float z = form(id);
    if (mine >= 0) {
      z += entry_bias(c.bias, mine, c.V);
      if (mrow != nullptr && !(mrow[mine / 32] >> (mine % 32) & 1)) z = -INFINITY;
    }
    best.add(mine >= 0 ? key_of(z, (uint32_t)mine) : 0, c.K, lane);
  }

  // what the lists name
  float m = kNoMax, k = c.te.near, l = 0.f;
  if (c.ent_id != nullptr) {
    int slo, shi, alo, ahi;
    list_range(c.list.seen_ptr, c.list.n_seen, r, slo, shi);
    list_range(c.list.add_ptr, c.list.n_add, r, alo, ahi);
    const int count = shi - slo + ahi - alo;
    const size_t at = (size_t)slo + alo;
    for (int e0 = w0 * kWave; e0 < count; e0 += WPR * kWave) {
      int id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) id[u] = e0 + 16 * u + q < count ? c.ent_id[at + e0 + 16 * u + q] : -1;
      const int e = e0 + 16 * (q / 4) + 4 * kg + q % 4;
      const int mine = e < count ? c.ent_id[at + e] : -1;
      float z = form(id);
      if (mine >= 0) {
        z += entry_bias(c.bias, mine, c.V);
        const uint32_t times = c.ent_count[at + e];
        if (times > 0) {   // each step rounded, none fused
          z = z > 0.f ? __fdiv_rn(z, c.repetition) : __fmul_rn(z, c.repetition);
          z = __fsub_rn(z, __fadd_rn(c.presence, __fmul_rn(c.frequency, (float)times)));
        }
        z = __fadd_rn(z, c.ent_add[at + e]);
        const float kz = exponent_factor(z, c.te), mz = z * kz;
        if (mz > m) {
          l = l * __builtin_amdgcn_exp2f(m - mz) + 1.f;
          m = mz;
          k = kz;
        } else if (z != -INFINITY) {   // (NaN makes the sum NaN)
          l += __builtin_amdgcn_exp2f(fmaf(z, k, -m));
        }
      }
      best.add(mine >= 0 ? key_of(z, (uint32_t)mine) : 0, c.K, lane);
    }
  }
  share(best);
  if ((WPR == 1 || wave == 0) && lane < c.K) {
    c.top[(size_t)r * c.K + lane] = best.k != 0 ? (int32_t)key_index(best.k) : -1;
    c.logit[(size_t)r * c.K + lane] = key_value(best.k);
  }
  if (c.lse == nullptr) return;
  // the log sum: the first pass's shares, each wave every WPR-th, and the lists'
  const int shares = c.splits > 0 ? c.splits : c.deal.shares(r / c.share_rows);
  const size_t at0 = (c.splits > 0 ? 0 : (size_t)c.deal.slot(r / c.share_rows) * c.share_rows) + r % c.share_rows;
  float M, sum;
  RowBest none;
  join_shares<kWave, false>((shares - w0 + WPR - 1) / WPR, at0 + (size_t)w0 * c.share_rows, (size_t)c.share_rows * WPR,
                            lane, c.pm, c.pl, nullptr, M, sum, none);
#pragma unroll
  for (int o = kWave / 2; o >= 1; o /= 2) {
    const float m2 = __shfl_xor(m, o), l2 = __shfl_xor(l, o), mn = fmaxf(m, m2);
    l = l * __builtin_amdgcn_exp2f(m - mn) + l2 * __builtin_amdgcn_exp2f(m2 - mn);
    m = mn;
  }
  const float mn = fmaxf(M, m);
  sum = sum * __builtin_amdgcn_exp2f(M - mn) + l * __builtin_amdgcn_exp2f(m - mn);
  M = mn;
  if constexpr (WPR > 1) {
    if (lane == 0) {
      sums[wave][0] = M;
      sums[wave][1] = sum;
    }
    __syncthreads();
    for (int w = 1; w < WPR && wave == 0; ++w) {
      const float t = fmaxf(M, sums[w][0]);
      sum = sum * __builtin_amdgcn_exp2f(M - t) + sums[w][1] * __builtin_amdgcn_exp2f(sums[w][0] - t);
      M = t;
    }
  }
  if ((WPR == 1 || wave == 0) && lane == 0) c.lse[r] = row_lse(M, sum, c.te);
}

}  // namespace dev

namespace {
// How a call is cut, and where its parts lie in the workspace.
struct TopPlan {
  bool few;
  int nt, splits, per, nbs, words;
  dev::Deal deal;
  size_t id, count, add, mask, bmax, pm, pl, wp, bytes;
};
template <typename S>
TopPlan top_plan(int H, int R, int V, int n_listed) {
  constexpr int T = dev::voc_tile<S>();
  TopPlan p{};
  size_t shares;
  p.few = R <= 64;
  if (p.few) {
    const int tiles = cdiv(V, 32);
    p.nt = R <= 32 ? 1 : 2;
    p.per = cdiv(tiles, 1024);
    p.splits = cdiv(cdiv(tiles, p.per), dev::kVocWaves) * dev::kVocWaves;
    shares = (size_t)p.splits * 32 * p.nt;
  } else {
    p.nt = dev::top_tiles<S>(H);
    p.deal = make_deal(cdiv(R, dev::kVocRows * p.nt), cdiv(V, T), 256 * dev::top_waves<S>(H));
    shares = (size_t)p.deal.all_slots() * dev::kVocRows * p.nt;
  }
  p.nbs = cdiv(cdiv(V, T) * (T / dev::kTopBlock), 8) * 8;
  p.words = cdiv(cdiv(V, 32), 4) * 4;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at = up256(at + bytes);
    return here;
  };
  p.id = take((size_t)n_listed * 4);
  p.count = take((size_t)n_listed * 4);
  p.add = take((size_t)n_listed * 4);
  p.mask = take(n_listed > 0 ? (size_t)R * p.words * 4 : 0);
  p.bmax = take((size_t)R * p.nbs * 4);
  p.pm = take(shares * 4);
  p.pl = take(shares * 4);
  if (sizeof(S) == 4 && !p.few) p.wp = take((size_t)V * H * 6);
  p.bytes = at;
  return p;
}

template <typename S, int H>
hipError_t top_h(const TopArgs& a, hipStream_t st) {
  using namespace dev;
  const TopPlan p = top_plan<S>(H, a.R, a.V, a.n_seen + a.n_add);
  char* ws = static_cast<char*>(a.ws);
  TopRows c{};
  c.n_nodes = a.n_nodes; c.R = a.R; c.V = a.V; c.K = a.K; c.nbs = p.nbs;
  c.splits = p.splits; c.share_rows = p.few ? 32 * p.nt : kVocRows * p.nt; c.deal = p.deal;
  c.te = a.temper; c.bias = a.bias; c.node = a.node;
  c.rm = RowMask{a.mask, a.mask_of, a.n_masks, a.mask_words};
  c.list = Listing{a.seen_ptr, a.seen, a.add_ptr, a.add, a.value, a.n_seen, a.n_add};
  c.repetition = a.repetition; c.presence = a.presence; c.frequency = a.frequency;
  c.top = a.top; c.logit = a.logit; c.lse = a.lse;
  float *bmax = reinterpret_cast<float*>(ws + p.bmax), *pm = reinterpret_cast<float*>(ws + p.pm),
        *pl = reinterpret_cast<float*>(ws + p.pl);
  c.bmax = bmax; c.pm = pm; c.pl = pl;
  if (a.n_seen + a.n_add > 0) {
    int32_t* id = reinterpret_cast<int32_t*>(ws + p.id);
    uint32_t *count = reinterpret_cast<uint32_t*>(ws + p.count), *out = reinterpret_cast<uint32_t*>(ws + p.mask);
    float* add = reinterpret_cast<float*>(ws + p.add);
    // Workgroups of a row: one, but where few rows may have lists that are passed over in parts.
    const int parts = cdiv(a.V, kTable), most = a.R < 1024 ? 1024 / a.R : 1;
    const int each = a.n_seen + a.n_add > kHashed ? (parts < most ? parts : most) : 1;
    hipLaunchKernelGGL(vocab_rules_kernel<S>, dim3(a.R, each), dim3(kVocThreads), 0, st, a.R, a.V, c.list, c.rm, p.words,
                       out, id, count, add);
    c.rm = RowMask{out, nullptr, a.R, p.words};
    c.ent_id = id; c.ent_count = count; c.ent_add = add;
  }
  const S *X = static_cast<const S*>(a.X), *W = static_cast<const S*>(a.W);
  const bf16s* Ws = static_cast<const bf16s*>(a.W);
  if (sizeof(S) == 4 && !p.few) {
    bf16s* planes = reinterpret_cast<bf16s*>(ws + p.wp);
    const hipError_t err = GGNN_IMPL_NS::launch_vocab_planes((size_t)a.V * H, W, planes, st);
    if (err != hipSuccess) return err;
    Ws = planes;
  }
#define MAXIMA(LSE, MASK)                                                                                             \
  do {                                                                                                                \
    if (p.few && p.nt == 1)                                                                                           \
      hipLaunchKernelGGL((vocab_max_few_kernel<S, H, 1, LSE, MASK>), dim3(p.splits / kVocWaves), dim3(kVocThreads), 0, st, \
                         a.n_nodes, a.R, a.V, p.per, a.temper, X, W, a.bias, a.node, c.rm, bmax, p.nbs, pm, pl);       \
    else if (p.few)                                                                                                   \
      hipLaunchKernelGGL((vocab_max_few_kernel<S, H, 2, LSE, MASK>), dim3(p.splits / kVocWaves), dim3(kVocThreads), 0, st, \
                         a.n_nodes, a.R, a.V, p.per, a.temper, X, W, a.bias, a.node, c.rm, bmax, p.nbs, pm, pl);       \
    else                                                                                                              \
      hipLaunchKernelGGL((vocab_max_kernel<S, H, LSE, MASK>), dim3(p.deal.workers), dim3(kVocThreads), 0, st,         \
                         a.n_nodes, a.R, a.V, p.deal, a.temper, X, Ws, a.bias, a.node, c.rm, bmax, p.nbs, pm, pl);     \
  } while (0)
  if (a.lse != nullptr) {
    if (c.rm.bits != nullptr) MAXIMA(true, true); else MAXIMA(true, false);
  } else {
    if (c.rm.bits != nullptr) MAXIMA(false, true); else MAXIMA(false, false);
  }
#undef MAXIMA
  if (a.R <= 64)
    hipLaunchKernelGGL((vocab_pick_kernel<S, H, 16>), dim3(a.R), dim3(16 * kWave), 0, st, c, X, W);
  else if (a.R <= 2048)
    hipLaunchKernelGGL((vocab_pick_kernel<S, H, 4>), dim3(a.R), dim3(4 * kWave), 0, st, c, X, W);
  else
    hipLaunchKernelGGL((vocab_pick_kernel<S, H, 1>), dim3(cdiv(a.R, kVocWaves)), dim3(kVocThreads), 0, st, c, X, W);
  return hipGetLastError();
}
}  // namespace

namespace GGNN_IMPL_NS {
size_t top_workspace(int H, int R, int V, int n_listed) { return top_plan<dev::dt_t>(H, R, V, n_listed).bytes; }

hipError_t launch_top(int H, const TopArgs& a, hipStream_t st) {
  using S = dev::dt_t;
  switch (H) {
    case 32: return top_h<S, 32>(a, st);
    case 64: return top_h<S, 64>(a, st);
    case 128: return top_h<S, 128>(a, st);
    case 256: return top_h<S, 256>(a, st);
  }
  return hipErrorInvalidValue;
}
}  // namespace GGNN_IMPL_NS

}  // namespace ggnn
