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
// Workgroups of a launch along x, at most: a dimension takes fewer than 2^32 threads, which 2^24 rows of
// 256 (or 2^30 pairs, four threads each) would reach.  The rest goes to a further dimension.
constexpr int kGridX = 1 << 21;

// The first pass walks the entries in units of 128, in LDS chunks of top_chunk.
constexpr int kTopUnit = 128;
template <typename S>
constexpr int top_chunk(int H) {
  return sizeof(S) == 2 || H <= 64 ? 128 : H == 128 ? 64 : 32;
}
// 32-row tiles of a wave: an LDS fragment serves both of two.
template <typename S>
constexpr int top_tiles(int H) {
  return sizeof(S) == 4 ? (H >= 128 ? 1 : 2) : H >= 256 ? 2 : 1;
}
// Waves of a workgroup, which share its LDS chunks, and its rows.
template <typename S>
constexpr int top_group(int H) {
  return sizeof(S) == 4 && H >= 256 ? 4 : 8;
}
template <typename S>
constexpr int top_rows(int H) {
  return 32 * top_tiles<S>(H) * top_group<S>(H);
}
// Waves of a SIMD, by the registers of a wave's rows and the buffers.
template <typename S>
constexpr int top_waves(int H) {
  return sizeof(S) == 4 ? (H >= 256 ? 1 : 2) : H >= 256 ? 2 : 4;
}

// A 32 x 32 tile of logits has entries as its rows.  Row i holds entry top_entry(i) of its
// 32, so that a lane (lanes 32 g .. 32 g + 31) holds entries 16 g .. 16 g + 15, one block, in
// order.
__device__ __forceinline__ int top_entry(int i) { return 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3); }

// dma16 (csrc/lds_dma.h) from a wave-uniform address and each lane's offset in bytes.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop

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
// The bits of 32 entries from e0 on that the vocabulary has.  Lanes beyond it hold the last entry's logits, which
// the starting -inf does not cover where its row is masked and holds NaN: they are taken out whatever a mask says there.
__device__ __forceinline__ uint32_t entry_bits(int e0, int V) {
  return V - e0 >= 32 ? ~0u : V > e0 ? (1u << (V - e0)) - 1u : 0u;
}
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

// First pass.  A workgroup holds its waves' rows (NT tiles of 32 a wave) and
// walks a share of the vocabulary, dealt in units of 128 entries as the losses' passes
// deal theirs (csrc/vocab.hip).  Writes block maxima to bmax [R][nbs] and, where LSE,
// (m, l) of a share to pm, pl [slot][rows of a workgroup].
//
// There is no second product here, so a step is its products and then its
// exponentials, and the waves that share a SIMD fill each other's.  LDS holds the
// entries in the order in which lanes read them as fragments, 1 KB a fragment, so
// that a read's place is a constant; the copies, 32 bytes a row each, pay for that
// order, and their addresses are constants too but in the last chunk.
//
// 12,001 rows over 50,021 entries at H = 256: 291 us, 1.06 PFLOP/s (a plain 8,192^3 product
// 1.39), matrix cores 53% busy and vector issue 41% at 2.0 GHz; without the log sum 247.
// (Products and exponentials of two tiles interleaved in one wave a SIMD, three buffers:
// 349; rows of the tile in LDS, 64 entries a barrier: 308.)  2,999 rows at H = 128: 52,
// 0.74 PFLOP/s, matrix cores 31%, vector issue 46%, waiting 36%; without the log sum 43.
// 3,001 rows over 10,007 at H = 64 with masks 17.9, waiting 46%: four units a workgroup
// (two of twice the workgroups: 1.5 us more).
// Block maxima: 10% of these times.
template <typename S, int H, bool LSE, bool MASK>
__global__ __launch_bounds__(kWave* top_group<S>(H), top_waves<S>(H)) void vocab_max_kernel(
    int n_nodes, int R, int V, Deal deal, Temper te, const S* __restrict__ X, const bf16s* __restrict__ W,
    const float* __restrict__ bias, const int32_t* __restrict__ node, RowMask rm, float* __restrict__ bmax, int nbs,
    float* __restrict__ pm, float* __restrict__ pl) {
  constexpr int T = top_chunk<S>(H), NP = voc_planes<S>(), NT = top_tiles<S>(H), NS = H / 16, NF = NS * NP;
  constexpr int SUB = T / 32, CH = kTopUnit / T, ROWS = top_rows<S>(H), WAVES = top_group<S>(H);
  constexpr int kAhead = NF < 4 ? NF : 4, STEPS = kTopUnit / 32;
  constexpr uint32_t ROW = H * 2, CHUNK = SUB * NF * 1024;   // bytes of a row and of a buffer
  __shared__ __attribute__((aligned(1024))) char buffer[2][CHUNK];
  __shared__ __attribute__((aligned(16))) float tb[2][T];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = lane / 32;
  const uint32_t lds0 = (uint32_t)(uintptr_t)buffer[0];
  typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;

  const uint32_t from = (uint32_t)top_entry(lane % 32) * ROW + 16u * g;   // of a lane's copies, from a step's first row
  float nb = 0.f;
  Run run;
  Dealt dealt(deal, blockIdx.x);
  while (dealt.next(deal, blockIdx.x, &run)) {
    const int q0 = run.t0 * CH, q1 = run.t1 * CH;                  // chunks
    const int row0 = run.i * ROWS + wave * 32 * NT + lane % 32;   // of the lane's first tile
    bf16x8 x[NT][NP][NS];
    RowSum sum[NT];
    const uint32_t* mrow[NT];
    uint32_t word[NT][SUB], next_word[NT][SUB];   // mask bits of the chunk in use and of the one on its way
    auto fetch = [&](int q) {   // start the copies of chunk q
      const char* src = reinterpret_cast<const char*>(W) + (size_t)q * T * ROW;
      const uint32_t to = lds0 + (uint32_t)(q & 1) * CHUNK;
      const bool whole = (q + 1) * T <= V;
#pragma unroll
      for (int p = 0; p < (SUB * NF + WAVES - 1) / WAVES; ++p) {
        const int i = p * WAVES + wave, s = i / NF, n = i % NF;
        if (SUB * NF % WAVES != 0 && i >= SUB * NF) break;
        const size_t at = (size_t)(n % NP) * V * ROW + (uint32_t)(32 * s) * ROW + 32u * (n / NP);
        if (whole) {
          dma16(src + at, from, to + (uint32_t)i * 1024u);
        } else {   // the last entry's row in place of those beyond
          const int row = min(q * T + 32 * s + top_entry(lane % 32), V - 1);
          dma16(W + (size_t)(n % NP) * V * H + (size_t)row * H + 16 * (n / NP) + 8 * g, to + (uint32_t)i * 1024u);
        }
      }
      // (raw values: a use here would wait for the copies too)
      if (bias != nullptr && threadIdx.x < T) nb = bias[min(q * T + (int)threadIdx.x, V - 1)];
      if constexpr (MASK) {
#pragma unroll
        for (int a = 0; a < NT; ++a)
#pragma unroll
          for (int i = 0; i < SUB; ++i)
            next_word[a][i] = mrow[a] != nullptr ? mrow[a][min(q * SUB + i, rm.words - 1)] : ~0u;
      }
    };
    auto land = [&](int q) {   // and wait for those of chunk q; every wave has left the other buffer
      if (threadIdx.x < T)
        tb[q & 1][threadIdx.x] = q * T + (int)threadIdx.x >= V || nb <= kMaskedBias ? -INFINITY : nb;
      if constexpr (MASK) {
#pragma unroll
        for (int a = 0; a < NT; ++a)
#pragma unroll
          for (int i = 0; i < SUB; ++i) word[a][i] = (next_word[a][i] & entry_bits(q * T + 32 * i, V)) >> (16 * g);
      }
      wait_copies<0>();
      __syncthreads();
    };
    const uint32_t place = (uint32_t)(lane % 32) * (uint32_t)nbs + 4u * g;   // in bmax, from the wave's first row on
    float* wave_max = bmax + (size_t)(run.i * ROWS + wave * 32 * NT) * nbs;

    __syncthreads();   // every wave has left the buffers of the run before
#pragma unroll
    for (int a = 0; a < NT; ++a) mrow[a] = MASK ? rm.row(row0 + 32 * a, R) : nullptr;
    fetch(q0);
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      load_planes<S, H>(x[a], X, row_node(node, row0 + 32 * a, R, n_nodes), lane);
      sum[a] = RowSum{kNoMax, te.near, 0.f};
    }
#pragma unroll 1
    for (int q = q0; q < q1; q += CH) {
      float kept[NT][STEPS];   // block maxima of the unit
#pragma unroll
      for (int step = 0; step < STEPS; ++step) {
        const int c = q + step / SUB, sub = step % SUB;
        if (sub == 0) {
          land(c);
          if (c + 1 < q1) fetch(c + 1);
        }
        const uint32_t at = lds0 + (uint32_t)(c & 1) * CHUNK + 16u * lane;
        bf16x8 f[NF];   // at most kAhead are alive
        auto read = [&](int n) {   // fragment n: k step n / NP, plane n % NP
          f[n] = __builtin_bit_cast(bf16x8, *(lds_u32x4*)(at + (uint32_t)(sub * NF + n) * 1024u));
        };
#pragma unroll
        for (int n = 0; n < kAhead; ++n) read(n);
        f32x16 s[NT], b;
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(tb[c & 1] + 32 * sub + 16 * g + 4 * j4);
#pragma unroll
          for (int i = 0; i < 4; ++i) b[4 * j4 + i] = v[i];
        }
#pragma unroll
        for (int a = 0; a < NT; ++a) s[a] = b;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NF; ++n) {
          if (n + kAhead < NF) read(n + kAhead);
#pragma unroll
          for (int p = 0; p + n % NP < NP; ++p)
#pragma unroll
            for (int a = 0; a < NT; ++a) mma32(s[a], f[n], x[a][p][n / NP]);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int a = 0; a < NT; ++a) {
          if constexpr (MASK) take_out(s[a], word[a][sub]);
          kept[a][step] = max16(s[a]);
        }
        if constexpr (LSE) {
          // (the maximum follows where it would grow by more than 2^8, as in the losses' rows pass)
          bool grows = false;
#pragma unroll
          for (int a = 0; a < NT; ++a) grows |= kept[a][step] * sum[a].k > sum[a].m + 8.f;
          if (__ballot(grows)) {
#pragma unroll
            for (int a = 0; a < NT; ++a) {
              const uint32_t own = __float_as_uint(kept[a][step]);
              const auto sw = __builtin_amdgcn_permlane32_swap(own, own, false, false);
              const float z = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])), kn = exponent_factor(z, te);
              const float mn = fmaxf(sum[a].m, z * kn);
              if (mn > sum[a].m) sum[a].k = kn;
              sum[a].l *= __builtin_amdgcn_exp2f(sum[a].m - mn);
              sum[a].m = mn;
            }
          }
#pragma unroll
          for (int a = 0; a < NT; ++a)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              sum[a].l += __builtin_amdgcn_exp2f(fmaf(s[a][j], sum[a].k, -sum[a].m));
              if (j % 8 == 7) {   // (or all arguments are held at once, and the next step's products come first)
                keep_here(sum[a].l);
                __builtin_amdgcn_sched_barrier(0);
              }
            }
        } else {
#pragma unroll
          for (int a = 0; a < NT; ++a) keep_here(kept[a][step]);
        }
      }
      // A row's eight maxima are stored as 32 bytes by its two lanes.
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(kept[a][0]), __float_as_uint(kept[a][2]), false,
                                                        false);
        const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(kept[a][1]), __float_as_uint(kept[a][3]), false,
                                                        false);
        if (row0 + 32 * a < R)
          *reinterpret_cast<u32x4*>(wave_max + (size_t)(32 * a) * nbs + (q / CH) * (kTopUnit / kTopBlock) + place) =
              u32x4{u[0], u[1], w[0], w[1]};
      }
    }
    if constexpr (LSE) {
#pragma unroll
      for (int a = 0; a < NT; ++a) {
        const float l = sum[a].l + __shfl_xor(sum[a].l, 32);
        const size_t at = (size_t)run.slot * ROWS + wave * 32 * NT + 32 * a + lane % 32;
        if (g == 0) {
          pm[at] = sum[a].m;
          pl[at] = l;
        }
      }
    }
  }
}

// First pass for at most 32 NT rows: every wave holds the same rows and takes `per`
// tiles of 32 entries, read straight from memory, since no other wave needs them.  4.0 us
// for one row over 10,007 entries at H = 64 (the launch), 10.0 over 50,021 at H = 256 with a
// mask (25.6 MB, 2.6 TB/s: one or two round trips to memory a wave).  (float32 at H = 256
// with two tiles holds more than a lane's registers, 171 to 244 of them in scratch: the call
// for 64 rows over 10,007 entries takes 48 us, for 32 rows 32.)
template <typename S, int H, int NT, bool LSE, bool MASK>
__global__ __launch_bounds__(kVocThreads) void vocab_max_few_kernel(
    int n_nodes, int R, int V, int per, Temper te, const S* __restrict__ X, const S* __restrict__ W,
    const float* __restrict__ bias, const int32_t* __restrict__ node, RowMask rm, float* __restrict__ bmax, int nbs,
    float* __restrict__ pm, float* __restrict__ pl) {
  const int lane = threadIdx.x % kWave, g = lane / 32, r = lane % 32;
  const int split = blockIdx.x * kVocWaves + threadIdx.x / kWave;
  const int tiles = (V + 31) / 32, t0 = split * per, t1 = min(tiles, t0 + per);
  // a tile's rows of W and biases are on their way while the one before is worked on, the first one's before
  // the rows' nodes are known
  frag_t<S> xf[NT][H / 16], next[H / 16];
  float next_bias[16];
  auto fetch = [&](int t) {
    load_row<S, H>(next, W, min(t * 32 + top_entry(r), V - 1), lane);
#pragma unroll
    for (int j = 0; j < 16; ++j) next_bias[j] = bias != nullptr ? bias[min(t * 32 + 16 * g + j, V - 1)] : 0.f;
  };
  fetch(min(t0, tiles - 1));
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
    f32x16 b;
#pragma unroll
    for (int kk = 0; kk < H / 16; ++kk) wf[kk] = next[kk];
#pragma unroll
    for (int j = 0; j < 16; ++j)
      b[j] = t * 32 + 16 * g + j >= V || next_bias[j] <= kMaskedBias ? -INFINITY : next_bias[j];
    if (t + 1 < t1) fetch(t + 1);
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      uint32_t w = ~0u;
      if (MASK && mrow[a] != nullptr) w = mrow[a][t];
      w = (w & entry_bits(32 * t, V)) >> (16 * g);
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
constexpr int kTable = 4096, kHashed = kTable / 2;   // places; longest lists that are hashed

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

// THREADS a row.  Latency: 6.7 us for one row of 24 listings, 9 us for 64 rows of 780
// (1,024 threads; 256 threads and a hash table of half the places 21), 13 us for 3,001 rows
// of 58: a chain of loads, table look-ups and barriers, a few rows a compute unit.
template <typename S, int THREADS>   // (the same for both types S)
__global__ __launch_bounds__(THREADS) void vocab_rules_kernel(int R, int V, Listing list, RowMask rm, int words,
                                                              int table, uint32_t* __restrict__ out,
                                                              int32_t* __restrict__ ent_id,
                                                              uint32_t* __restrict__ ent_count,
                                                              float* __restrict__ ent_add) {
  // Entry, place of its first listing, times seen (low half: hashed lists have at most
  // 2048 listings) and biases (high half), a bias; a table without hashing holds the
  // biases' count in place of the entry.
  extern __shared__ uint32_t lds[];
  uint32_t *key = lds, *first = lds + table, *seen = lds + 2 * table;
  float* value = reinterpret_cast<float*>(lds + 3 * table);
  const int r = blockIdx.z * kGridX + blockIdx.x;
  if (r >= R) return;   // whole workgroups leave
  int slo, shi, alo, ahi;
  list_range(list.seen_ptr, list.n_seen, r, slo, shi);
  list_range(list.add_ptr, list.n_add, r, alo, ahi);
  const int n_seen = shi - slo, n = n_seen + ahi - alo;
  const size_t at = (size_t)slo + alo;   // the row's places
  const uint32_t* mask = rm.row(r, R);
  uint32_t* mine = out + (size_t)r * words;
  const bool hashed = n <= table / 2;
  int bits = 6;
  while (hashed && (1 << bits) < 2 * n) ++bits;
  const int size = hashed ? 1 << bits : table;
  const long parts = hashed ? 1 : ((long)V + table - 1) / table;
  constexpr int kKeep = 2;   // listings that a thread keeps from the first look to the second
  int id[kKeep];
#pragma unroll
  for (int u = 0; u < kKeep; ++u) {
    const int i = u * THREADS + threadIdx.x;
    const int s = list.n_seen > 0 ? list.seen[min(slo + min(i, max(n_seen - 1, 0)), list.n_seen - 1)] : -1;
    const int a = list.n_add > 0 ? list.add[min(alo + max(i - n_seen, 0), list.n_add - 1)] : -1;
    id[u] = i >= n ? -1 : i < n_seen ? s : a;
  }
  auto token = [&](int u, int i) {
    if (u == 0) return id[0];
    if (u == 1) return id[1];
    return i < n_seen ? list.seen[slo + i] : list.add[alo + i - n_seen];
  };
  auto hash = [&](int e) { return (uint32_t)e * 0x9E3779B1u >> (32 - bits); };
  for (long p = blockIdx.y; p < parts; p += gridDim.y) {
    const int lo = hashed ? 0 : (int)(p * table), hi = hashed ? V : (int)min((long)V, (long)lo + table);
    for (int i = threadIdx.x; i < size; i += THREADS) {
      key[i] = hashed ? ~0u : 0u;
      first[i] = ~0u;
      seen[i] = 0;
    }
    for (int w = lo / 32 + threadIdx.x; w < (hi + 31) / 32; w += THREADS) mine[w] = mask != nullptr ? mask[w] : ~0u;
    __threadfence_block();
    __syncthreads();
    for (int i = threadIdx.x, u = 0; i < n; i += THREADS, ++u) {
      const int e = token(u, i);
      if (e < lo || e >= hi) continue;
      uint32_t h = (uint32_t)(e - lo);
      if (hashed) {   // at most half of the places are taken, so a free one is found
        h = hash(e);
        for (;;) {
          const uint32_t old = atomicCAS(&key[h], ~0u, (uint32_t)e);
          if (old == ~0u || old == (uint32_t)e) break;
          h = (h + 1) & (size - 1);
        }
      }
      atomicMin(&first[h], (uint32_t)i);
      if (i < n_seen) {
        atomicAdd(&seen[h], 1u);
      } else {
        if (hashed) atomicAdd(&seen[h], 1u << 16);
        else atomicAdd(&key[h], 1u);
        value[h] = list.value[alo + i - n_seen];   // (used where it is the only one)
      }
    }
    __syncthreads();
    auto place = [&](int e) {   // of an entry that the table has
      if (!hashed) return (uint32_t)(e - lo);
      uint32_t h = hash(e);
      while (key[h] != (uint32_t)e) h = (h + 1) & (size - 1);
      return h;
    };
    auto adds = [&](uint32_t h) { return hashed ? seen[h] >> 16 : key[h]; };
    // Entries with several biases: zero, then added up in list order, a wave at a time.
    int again = 0;
    for (int i = alo + threadIdx.x; i < ahi; i += THREADS) {
      const int e = list.add[i];
      if (e < lo || e >= hi) continue;
      const uint32_t h = place(e);
      if (adds(h) > 1) {
        value[h] = 0.f;
        again = 1;
      }
    }
    if (__syncthreads_or(again)) {
      for (int i0 = alo; i0 < ahi; i0 += kWave) {
        if (i0 / kWave % (THREADS / kWave) == threadIdx.x / kWave) {
          const int i = i0 + threadIdx.x % kWave, e = i < ahi ? list.add[i] : -1;
          const float v = i < ahi ? list.value[i] : 0.f;
          int h = -1;
          if (e >= lo && e < hi) {
            h = (int)place(e);
            if (adds((uint32_t)h) < 2) h = -1;
          }
          uint64_t left = __ballot(h >= 0);
          while (left != 0) {
            const int one = __builtin_amdgcn_readlane(h, (int)__builtin_ctzll(left));
            uint64_t same = __ballot(h == one);
            left &= ~same;
            float sum = value[one];
            for (; same != 0; same &= same - 1)
              sum += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), (int)__builtin_ctzll(same)));
            value[one] = sum;   // (the same from every lane)
          }
        }
        __syncthreads();
      }
    }
    for (int i = threadIdx.x, u = 0; i < n; i += THREADS, ++u) {
      const int e = token(u, i);
      const bool known = e >= 0 && e < V;
      if (known ? e < lo || e >= hi : p != 0) continue;   // another part's
      int found = -1;
      if (known) {
        const uint32_t h = place(e);
        if (first[h] == (uint32_t)i && (mask == nullptr || (mask[e / 32] >> (e % 32) & 1))) {
          found = e;
          ent_count[at + i] = hashed ? seen[h] & 0xFFFFu : seen[h];
          ent_add[at + i] = adds(h) > 0 ? value[h] : 0.f;
          atomicAnd(&mine[e / 32], ~(1u << (e % 32)));
        }
      }
      ent_id[at + i] = found;
    }
    __syncthreads();
  }
}

// ---- second pass -----------------------------------------------------------

// A float as a whole number that orders alike, 0 for -inf and NaN; -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float z) {
  z += 0.f;
  const uint32_t u = __float_as_uint(z);
  return z > -INFINITY ? u ^ (u >> 31 ? ~0u : 0x80000000u) : 0u;
}
// A candidate as one number that orders by value, then by the lower index; 0: none.
typedef unsigned long long pick_t;
__device__ __forceinline__ pick_t pick_of(uint32_t order, uint32_t index) {
  return order != 0 ? (pick_t)order << 32 | (uint32_t)~index : 0;
}
__device__ __forceinline__ uint32_t pick_index(pick_t k) { return ~(uint32_t)k; }
__device__ __forceinline__ float pick_value(pick_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return k == 0 ? -INFINITY : __uint_as_float(u ^ (u >> 31 ? 0x80000000u : ~0u));
}
__device__ __forceinline__ pick_t pick_at(pick_t k, int lane) {   // lane: the same in the whole wave
  return (pick_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}
// A bound that K or more of the wave's numbers a and b reach, bit by bit: the K-th
// largest, or any between it and the next; 0 where fewer are not 0.  Four bits between
// two looks whether it is reached by just K (the call for one row over 10,007 entries:
// 13.6 us; a look each bit 18.0, all 32 bits without one 14.9).
__device__ __forceinline__ uint32_t kth_of(uint32_t a, uint32_t b, int K) {
  uint32_t t = 0;
#pragma unroll 1
  for (int shift = 28; shift >= 0; shift -= 4) {
#pragma unroll
    for (int bit = 3; bit >= 0; --bit) {
      const uint32_t c = t | 1u << (shift + bit);
      if (__popcll(__ballot(a >= c)) + __popcll(__ballot(b >= c)) >= K) t = c;
    }
    if (__popcll(__ballot(a >= t)) + __popcll(__ballot(b >= t)) == K) break;
  }
  return t;
}

// The 64 largest picks seen, in descending order over the lanes.
struct Best {
  pick_t k = 0;
  // Bitonic steps over lanes at distances d, d / 2, ... 1, descending where the number of
  // a group of `group` lanes is even.
  static __device__ __forceinline__ void steps(pick_t& v, int group, int d, int lane) {
    for (; d >= 1; d /= 2) {
      const pick_t o = __shfl_xor(v, d);
      const bool low = (lane & d) == 0, down = (lane & group) == 0;
      v = low == down ? max(v, o) : min(v, o);
    }
  }
  static __device__ __forceinline__ void sort(pick_t& v, int lane) {
#pragma unroll
    for (int group = 2; group <= kWave; group *= 2) steps(v, group, group / 2, lane);
  }
  // Joins another descending list.
  __device__ __forceinline__ void join(pick_t other, int lane) {
    k = max(k, __shfl(other, kWave - 1 - lane));
    steps(k, kWave, kWave / 2, lane);
  }
  // Adds one pick a lane; K: how many of the largest matter.
  __device__ __forceinline__ void add(pick_t c, int K, int lane) {
    uint64_t in = __ballot(c > pick_at(k, K - 1));
    if (__popcll(in) > 6) {   // about where sorting all costs less than one at a time
      sort(c, lane);
      join(c, lane);
      return;
    }
    while (in != 0) {
      const pick_t one = pick_at(c, (int)__builtin_ctzll(in));
      in &= in - 1;
      const int place = __popcll(__ballot(k > one));
      const pick_t up = __shfl_up(k, 1);
      k = lane < place ? k : lane == place ? one : up;
    }
  }
};

// Writes a row's answers from its n <= 64 picks in LDS, in no order: each lane counts
// how many come before its own.
__device__ __forceinline__ void answer(const pick_t* picks, int n, int r, int K, int lane, int32_t* __restrict__ top,
                                       float* __restrict__ logit) {
  const pick_t own = lane < n ? picks[lane] : 0;
  int rank = 0;
#pragma unroll 8
  for (int i = 0; i < n; ++i) rank += picks[i] > own;
  if (lane < n && rank < K) {
    top[(size_t)r * K + rank] = (int32_t)pick_index(own);
    logit[(size_t)r * K + rank] = pick_value(own);
  }
  if (lane >= n && lane < K) {
    top[(size_t)r * K + lane] = -1;
    logit[(size_t)r * K + lane] = -INFINITY;
  }
}
// The same from a list in order, one pick a lane.
__device__ __forceinline__ void answer_list(pick_t k, int r, int K, int lane, int32_t* __restrict__ top,
                                            float* __restrict__ logit) {
  if (lane >= K) return;
  top[(size_t)r * K + lane] = k != 0 ? (int32_t)pick_index(k) : -1;
  logit[(size_t)r * K + lane] = pick_value(k);
}

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
  uint32_t* ent_count;   // taken over for order_of the ruled logits
  const float* ent_add;
  float repetition, presence, frequency;
  int32_t* top;
  float *logit, *lse;
};

// A row's state, and the logits of 64 entries at a time, one a lane, as four tiles of
// 16 x 16 whose entries lie along the rows: lane l holds row l % 16, k group l / 16.  In
// bf16 the state stands in all columns of the other operand, so that each lane
// finds one entry's logit among the accumulators.  In float32, where that would take
// 32 cycles for 64 useful products, each lane adds up its own and four lanes join.
template <typename S, int H>
struct RowState {
  static constexpr bool kMatrix = sizeof(S) == 2;
  frag_t<S> x[H / 32];
  int lane;
  __device__ __forceinline__ RowState(const S* __restrict__ X, int n, int lane) : lane(lane) {
#pragma unroll
    for (int kk = 0; kk < H / 32; ++kk) {
      if (n >= 0) x[kk] = load8(X + (size_t)n * H + 32 * kk + 8 * (lane / 16));
      else x[kk] = frag_t<S>{};
    }
  }
  // Tile of the lane's entry, and its row there.
  __device__ __forceinline__ int tile() const { return kMatrix ? lane % 16 / 4 : lane / 16; }
  __device__ __forceinline__ int entry() const { return kMatrix ? 4 * (lane / 16) + lane % 4 : lane % 16; }
  // Largest of the tile's sixteen values; whether the lane is the tile's first.
  __device__ __forceinline__ uint32_t tile_max(uint32_t m) const {
    m = max(m, __shfl_xor(m, 1));
    m = max(m, __shfl_xor(m, 2));
    m = max(m, __shfl_xor(m, kMatrix ? 16 : 4));
    return max(m, __shfl_xor(m, kMatrix ? 32 : 8));
  }
  __device__ __forceinline__ bool leads() const { return kMatrix ? lane < 16 && lane % 4 == 0 : lane % 16 == 0; }
  // id[u], lanes l % 16: the entries of tile u < tiles (negative: none).  Two tiles' rows
  // of W are on their way at a time.
  __device__ __forceinline__ float form(const S* __restrict__ W, const int (&id)[4], int tiles) const {
    float z = 0.f;
#pragma unroll
    for (int u0 = 0; u0 < 4; u0 += 2) {
      if (u0 >= tiles) break;
      frag_t<S> w[2][H / 32];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int kk = 0; kk < H / 32; ++kk)
          w[u][kk] = load8(W + (size_t)max(id[u0 + u], 0) * H + 32 * kk + 8 * (lane / 16));
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if constexpr (kMatrix) {
          f32x4 acc = {};
#pragma unroll
          for (int kk = 0; kk < H / 32; ++kk) mma(acc, w[u][kk], x[kk]);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (lane % 16 == 4 * (u0 + u) + j) z = acc[j];
        } else {
          float part[2] = {};
#pragma unroll
          for (int kk = 0; kk < H / 32; ++kk)
#pragma unroll
            for (int i = 0; i < 8; ++i) part[i % 2] = fmaf(w[u][kk][i], x[kk][i], part[i % 2]);
          float a = part[0] + part[1];
          a += __shfl_xor(a, 16);
          a += __shfl_xor(a, 32);
          if (lane / 16 == u0 + u) z = a;
        }
      }
    }
    return z;
  }
};

// The logit of an entry that a row's lists name, from the raw one z.
__device__ __forceinline__ float ruled(const TopRows& c, float z, uint32_t times, float add) {
  if (times > 0) {   // each step rounded, none fused
    z = z > 0.f ? __fdiv_rn(z, c.repetition) : __fmul_rn(z, c.repetition);
    z = __fsub_rn(z, __fadd_rn(c.presence, __fmul_rn(c.frequency, (float)times)));
  }
  return __fadd_rn(z, add);
}
__device__ __forceinline__ void add_exponential(RowSum& s, float z, const Temper& te) {
  const float kz = exponent_factor(z, te), mz = z * kz;
  if (mz > s.m) {
    s.l = s.l * __builtin_amdgcn_exp2f(s.m - mz) + 1.f;
    s.m = mz;
    s.k = kz;
  } else if (z != -INFINITY) {   // (NaN makes the sum NaN)
    s.l += __builtin_amdgcn_exp2f(fmaf(z, s.k, -s.m));
  }
}

// The ruled logits of what row r's lists name: wave w of `waves` takes every waves-th 16
// places, four at a time.  Adds their exponentials to `own`, leaves order_of them in
// ent_count and calls visit(order, entry) with a lane's (0: none) in step.
template <typename S, int H, typename Visit>
__device__ __forceinline__ void rule_lists(const TopRows& c, const RowState<S, H>& row, const S* __restrict__ W, int r,
                                           int w, int waves, RowSum& own, Visit visit) {
  int slo, shi, alo, ahi;
  list_range(c.list.seen_ptr, c.list.n_seen, r, slo, shi);
  list_range(c.list.add_ptr, c.list.n_add, r, alo, ahi);
  const int count = shi - slo + ahi - alo, lane = row.lane;
  const size_t at = (size_t)slo + alo;
  for (int e0 = 16 * w; e0 < count; e0 += 64 * waves) {
    // one load of the 64 names, passed on between the lanes; what changes them is on its way with it
    const int e = e0 + 16 * waves * row.tile() + row.entry();
    const int all = c.ent_id[at + min(e0 + 16 * waves * (lane / 16) + lane % 16, count - 1)];
    const uint32_t times = c.ent_count[at + min(e, count - 1)];
    const float add = c.ent_add[at + min(e, count - 1)];
    int ids[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int id = __shfl(all, 16 * u + lane % 16);
      ids[u] = e0 + 16 * waves * u + lane % 16 < count ? id : -1;
    }
    const int own_id = __shfl(all, 16 * row.tile() + row.entry()), mine = e < count ? own_id : -1;
    const float b = entry_bias(c.bias, max(mine, 0), c.V);
    float v = row.form(W, ids, (count - e0 + 16 * waves - 1) / (16 * waves)) + b;
    uint32_t o = 0;
    if (mine >= 0) {
      v = ruled(c, v, times, add);
      add_exponential(own, v, c.te);
      o = order_of(v);
      c.ent_count[at + e] = o;
    }
    visit(o, (uint32_t)mine);
  }
}
// The same places again, from what rule_lists left (by the same waves).
template <typename S, int H, typename Visit>
__device__ __forceinline__ void ruled_lists(const TopRows& c, const RowState<S, H>& row, int r, int w, int waves,
                                            Visit visit) {
  int slo, shi, alo, ahi;
  list_range(c.list.seen_ptr, c.list.n_seen, r, slo, shi);
  list_range(c.list.add_ptr, c.list.n_add, r, alo, ahi);
  const int count = shi - slo + ahi - alo;
  const size_t at = (size_t)slo + alo;
  for (int e0 = 16 * w; e0 < count; e0 += 64 * waves) {
    const int e = e0 + 16 * waves * row.tile() + row.entry(), mine = e < count ? c.ent_id[at + e] : -1;
    visit(mine >= 0 ? c.ent_count[at + e] : 0u, (uint32_t)mine);
  }
}
// Joins the lanes' sums, and with them the row's share (M, sum).
__device__ __forceinline__ void join_own(RowSum own, float& M, float& sum) {
#pragma unroll
  for (int o = kWave / 2; o >= 1; o /= 2) {
    const float m2 = __shfl_xor(own.m, o), l2 = __shfl_xor(own.l, o), t = fmaxf(own.m, m2);
    own.l = own.l * __builtin_amdgcn_exp2f(own.m - t) + l2 * __builtin_amdgcn_exp2f(m2 - t);
    own.m = t;
  }
  const float t = fmaxf(M, own.m);
  sum = sum * __builtin_amdgcn_exp2f(M - t) + own.l * __builtin_amdgcn_exp2f(own.m - t);
  M = t;
}

// Second pass, all in one: a workgroup of WPR waves per row.
//
// Both choices, of blocks and of entries, begin with a bound below the K-th largest:
// the K-th largest of numbers that are maxima of disjoint parts.  What reaches it is
// seldom much more than K, and goes to LDS as one list; where it does not fit 64
// places (many equal ones), the waves' own lists are joined instead.
//
// One row over 10,007 entries: 6.9 us, of which two barriers' waits and four dependent
// round trips to memory are most (an insertion into sorted lists in registers 15.0); 64
// rows of 780 listings 19; 1,229 rows in float32, K = 16, 30 (161 MB gathered, 5 TB/s).
template <typename S, int H, int WPR>
__global__ __launch_bounds__(kWave* WPR) void vocab_pick_kernel(TopRows c, const S* __restrict__ X,
                                                                const S* __restrict__ W) {
  constexpr int U = 4;
  __shared__ pick_t lists[WPR][kWave];
  __shared__ uint32_t tops[kWave];
  __shared__ float sums[WPR][2];
  __shared__ int n_blocks, n_best;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r = blockIdx.x;
  const RowState<S, H> row(X, row_node(c.node, r, c.R, c.n_nodes), lane);
  const uint32_t* mrow = c.rm.row(r, c.R);
  // Joins the waves' lists; every wave has the result.
  auto share = [&](Best& b) {
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
  };

  // Blocks.  Wave w looks at every WPR-th 64 of them.
  const float* bm = c.bmax + (size_t)r * c.nbs;
  const int nb = (c.V + kTopBlock - 1) / kTopBlock, first = wave * kWave + lane;
  auto load = [&](uint32_t (&o)[U], int b0) {
    float m[U];   // (all on their way before the first is looked at)
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = b0 + u * WPR * kWave < nb ? bm[b0 + u * WPR * kWave] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) o[u] = b0 + u * WPR * kWave < nb ? order_of(m[u]) : 0u;
  };
  uint32_t head[U], most = 0;   // the first of them stay in registers
  load(head, first);
  // the first pass's shares of the sum: each wave takes every WPR-th
  float M = kNoMax, sum = 0.f;
  if (c.lse != nullptr) {
    const int shares = c.splits > 0 ? c.splits : c.deal.shares(r / c.share_rows);
    const size_t at0 = (c.splits > 0 ? 0 : (size_t)c.deal.slot(r / c.share_rows) * c.share_rows) + r % c.share_rows;
    RowBest none;
    join_shares<kWave, false>((shares - wave + WPR - 1) / WPR, at0 + (size_t)wave * c.share_rows,
                              (size_t)c.share_rows * WPR, lane, c.pm, c.pl, nullptr, M, sum, none);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) most = max(most, head[u]);
  for (int b0 = first + U * WPR * kWave; b0 < nb + lane; b0 += U * WPR * kWave) {
    uint32_t o[U];
    load(o, b0);
#pragma unroll
    for (int u = 0; u < U; ++u) most = max(most, o[u]);
  }
  uint32_t* maxima = reinterpret_cast<uint32_t*>(lists);
  maxima[threadIdx.x] = most;
  if (threadIdx.x == 0) n_blocks = n_best = 0;
  __syncthreads();
  uint32_t even = 0, odd = 0;
#pragma unroll
  for (int w = 0; w < WPR; w += 2) {
    even = max(even, maxima[w * kWave + lane]);
    odd = max(odd, maxima[(w + 1) * kWave + lane]);
  }
  uint32_t bound = max(kth_of(even, odd, c.K), 1u);
  __syncthreads();
  pick_t* chosen = lists[0];
  auto gather = [&](int* counter, uint32_t o, uint32_t index) {   // what reaches the bound
    if (o < bound) return;
    const int at = atomicAdd(counter, 1);
    if (at < kWave) chosen[at] = pick_of(o, index);
  };
#pragma unroll
  for (int u = 0; u < U; ++u) gather(&n_blocks, head[u], (uint32_t)(first + u * WPR * kWave));
  for (int b0 = first + U * WPR * kWave; b0 < nb + lane; b0 += U * WPR * kWave) {
    uint32_t o[U];
    load(o, b0);
#pragma unroll
    for (int u = 0; u < U; ++u) gather(&n_blocks, o[u], (uint32_t)(b0 + u * WPR * kWave));
  }
  __syncthreads();
  int n = n_blocks;
  pick_t block = 0;   // one a lane
  if (n <= kWave) {
    // the K first of them, in order: each lane counts how many come before its own
    block = lane < n ? chosen[lane] : 0;
    int rank = lane;
    if (lane < n) {
      rank = 0;
#pragma unroll 8
      for (int i = 0; i < n; ++i) rank += chosen[i] > block;
    }
    block = (pick_t)(uint32_t)__builtin_amdgcn_ds_permute(4 * rank, (int)(block >> 32)) << 32 |
            (uint32_t)__builtin_amdgcn_ds_permute(4 * rank, (int)block);
    n = min(n, c.K);
    __syncthreads();
  } else {
    __syncthreads();
    Best b;
    for (int b0 = first; b0 < nb + lane; b0 += WPR * kWave)
      b.add(b0 < nb ? pick_of(order_of(bm[b0]), (uint32_t)b0) : 0, c.K, lane);
    share(b);
    n = c.K;
    block = lane < n ? b.k : 0;
  }

  // Their entries: each wave takes every WPR-th block, four at a time.
  constexpr int G = kWave / 4 / WPR;
  uint32_t z[G], id[G];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int b0 = wave + 4 * WPR * i, tiles = (n - b0 + WPR - 1) / WPR;
    z[i] = 0;
    id[i] = 0;
    if (tiles > 0) {
      int ids[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const pick_t k = pick_at(block, min(b0 + WPR * u, kWave - 1));
        const int e = (int)pick_index(k) * kTopBlock + lane % 16;
        ids[u] = u < tiles && k != 0 && e < c.V ? e : -1;
      }
      const int at = b0 + WPR * row.tile();
      const pick_t k = __shfl(block, min(at, kWave - 1));
      const int e = (int)pick_index(k) * kTopBlock + row.entry();
      const bool is = at < n && k != 0 && e < c.V;
      const float b = entry_bias(c.bias, is ? e : 0, c.V);   // (on their way before the rows of W)
      const uint32_t may = mrow != nullptr ? mrow[is ? e / 32 : 0] : ~0u;
      const float raw = row.form(W, ids, tiles);
      if (is && (may >> (e % 32) & 1)) {
        z[i] = order_of(raw + b);
        id[i] = (uint32_t)e;
      }
      const uint32_t m = row.tile_max(z[i]);
      if (row.leads() && at < n) tops[at] = m;
    }
  }
  __syncthreads();
  bound = max(kth_of(lane < n ? tops[lane] : 0u, 0u, c.K), 1u);
#pragma unroll
  for (int i = 0; i < G; ++i) gather(&n_best, z[i], id[i]);
  RowSum own{kNoMax, c.te.near, 0.f};
  if (c.ent_id != nullptr)
    rule_lists(c, row, W, r, wave, WPR, own, [&](uint32_t o, uint32_t e) { gather(&n_best, o, e); });
  if (c.lse != nullptr) {
    join_own(own, M, sum);
    if (lane == 0) {
      sums[wave][0] = M;
      sums[wave][1] = sum;
    }
  }
  __syncthreads();
  const int picked = n_best;
  if (picked > kWave) {
    __syncthreads();
    Best best;
#pragma unroll
    for (int i = 0; i < G; ++i) best.add(pick_of(z[i], id[i]), c.K, lane);
    if (c.ent_id != nullptr)
      ruled_lists(c, row, r, wave, WPR, [&](uint32_t o, uint32_t e) { best.add(pick_of(o, e), c.K, lane); });
    share(best);
    if (wave == 0) answer_list(best.k, r, c.K, lane, c.top, c.logit);
  } else if (wave == 0) {
    answer(chosen, picked, r, c.K, lane, c.top, c.logit);
  }
  if (wave != WPR - 1 || c.lse == nullptr) return;
  M = sums[0][0];
  sum = sums[0][1];
  for (int w = 1; w < WPR; ++w) {
    const float t = fmaxf(M, sums[w][0]);
    sum = sum * __builtin_amdgcn_exp2f(M - t) + sums[w][1] * __builtin_amdgcn_exp2f(sums[w][0] - t);
    M = t;
  }
  if (lane == 0) c.lse[r] = row_lse(M, sum, c.te);
}

// ---- second pass over many rows ---------------------------------------------
//
// A block's 16 rows of W are 16 times a state, so where many rows pick blocks it is
// the states that move: the picked (row, block) pairs are sorted by block, and a wave
// forms the logits of 16 pairs, mostly of one block, as one 16 x 16 tile.  12,001 rows, K =
// 32, H = 256: blocks 42 us (150 MB of maxima), sort 34, pairs 54 (420 MB of states, rows of
// W and logits through the L2s, 7.8 TB/s), answers 28; gathering 3.1 GB of W in one
// launch took 415.

// The K best blocks of each row, one wave a row: block [R][K], -1 from where none is
// left.
constexpr int kReach = 2 * kWave;   // blocks that reach the bound, at most
// The first 512 GROUPS blocks are held in registers, the rest is read twice.
template <typename S, int GROUPS>   // (the same for both types S)
__global__ __launch_bounds__(kVocThreads) void vocab_blocks_kernel(int R, int nb, int nbs, int K,
                                                                   const float* __restrict__ bmax,
                                                                   int32_t* __restrict__ block) {
  constexpr int U = 8;
  __shared__ u32x2 reach[kVocWaves][kReach];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = blockIdx.x * kVocWaves + wave;
  if (r >= R) return;   // whole waves leave together
  const float* bm = bmax + (size_t)r * nbs;
  int32_t* out = block + (size_t)r * K;
  auto load = [&](float (&m)[U], int b0) {   // (all on their way before the first is looked at)
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = bm[min(b0 + u * kWave + lane, nb - 1)];
  };
  auto order = [&](float m, int b) { return b < nb ? order_of(m) : 0u; };
  float held[GROUPS][U];
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) load(held[g], g * U * kWave);
  uint32_t most[2] = {};
#pragma unroll
  for (int g = 0; g < GROUPS; ++g)
#pragma unroll
    for (int u = 0; u < U; ++u) most[u % 2] = max(most[u % 2], order(held[g][u], (g * U + u) * kWave + lane));
  for (int b0 = GROUPS * U * kWave; b0 < nb; b0 += U * kWave) {
    float m[U];
    load(m, b0);
#pragma unroll
    for (int u = 0; u < U; ++u) most[u % 2] = max(most[u % 2], order(m[u], b0 + u * kWave + lane));
  }
  const uint32_t bound = max(kth_of(most[0], most[1], K), 1u);
  const uint64_t below = (1ull << lane) - 1;
  int n = 0;
  auto take = [&](float m, int b) {
    const uint32_t o = order(m, b);
    const uint64_t in = __ballot(o >= bound);
    if (in == 0) return;
    const int at = n + __popcll(in & below);
    if (o >= bound && at < kReach) reach[wave][at] = u32x2{o, (uint32_t)b};
    n += __popcll(in);
  };
#pragma unroll
  for (int g = 0; g < GROUPS; ++g)
#pragma unroll
    for (int u = 0; u < U; ++u) take(held[g][u], (g * U + u) * kWave + lane);
  for (int b0 = GROUPS * U * kWave; b0 < nb; b0 += U * kWave) {
    float m[U];
    load(m, b0);
#pragma unroll
    for (int u = 0; u < U; ++u) take(m[u], b0 + u * kWave + lane);
  }
  if (n > kReach) {   // many equal ones
    Best best;
    for (int b0 = 0; b0 < nb; b0 += kWave) {
      const int b = b0 + lane;
      best.add(b < nb ? pick_of(order_of(bm[b]), (uint32_t)b) : 0, K, lane);
    }
    if (lane < K) out[lane] = best.k != 0 ? (int32_t)pick_index(best.k) : -1;
    return;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // in the order of their blocks: those above the K-th largest, then the first of its equals
  const u32x2 a = lane < n ? reach[wave][lane] : u32x2{}, b = lane + kWave < n ? reach[wave][lane + kWave] : u32x2{};
  const uint32_t kth = kth_of(a[0], b[0], K);
  const bool above_a = a[0] > kth, above_b = b[0] > kth, same_a = a[0] == kth && kth != 0, same_b = b[0] == kth && kth != 0;
  const uint64_t ma = __ballot(above_a), mb = __ballot(above_b), sa = __ballot(same_a), sb = __ballot(same_b);
  const int na = __popcll(ma), above = na + __popcll(mb), equal_a = __popcll(sa);
  const int pa = above_a ? __popcll(ma & below) : above + __popcll(sa & below);
  const int pb = above_b ? na + __popcll(mb & below) : above + equal_a + __popcll(sb & below);
  if ((above_a || same_a) && pa < K) out[pa] = (int32_t)a[1];
  if ((above_b || same_b) && pb < K) out[pb] = (int32_t)b[1];
  const int all = above + equal_a + __popcll(sb);
  if (lane >= all && lane < K) out[lane] = -1;
}

// The logits of the picked blocks' entries, z [R][K][16], from the sorted pairs (block,
// row and place).
template <typename S, int H>
__global__ __launch_bounds__(kVocThreads) void vocab_pairs_kernel(TopRows c, const u32x2* __restrict__ pairs, int n_pairs,
                                                                  const S* __restrict__ X, const S* __restrict__ W,
                                                                  float* __restrict__ z) {
  const int lane = threadIdx.x % kWave, q = lane % 16, kg = lane / 16;
  const int group = blockIdx.y * kGridX + blockIdx.x, nb = (c.V + kTopBlock - 1) / kTopBlock;
  const int i = (group * kVocWaves + threadIdx.x / kWave) * 16 + q;   // fewer than 2^30 + 64 kGridX
  const u32x2 pair = i < n_pairs ? pairs[i] : u32x2{(uint32_t)nb, 0u};
  const int b = (int)pair[0];
  uint64_t left = __ballot(b < nb) & 0xFFFFu;
  if (left == 0) return;   // whole waves leave together
  const int r = (int)pair[1] / c.K, n = b < nb ? row_node(c.node, r, c.R, c.n_nodes) : -1;
  frag_t<S> x[H / 32];
#pragma unroll
  for (int kk = 0; kk < H / 32; ++kk) {
    if (n >= 0) x[kk] = load8(X + (size_t)n * H + 32 * kk + 8 * kg);
    else x[kk] = frag_t<S>{};
  }
  const uint32_t* mrow = b < nb ? c.rm.row(r, c.R) : nullptr;
  const uint32_t may = mrow != nullptr ? mrow[b / 2] >> (16 * (b & 1) + 4 * kg) : ~0u;
  while (left != 0) {
    const int one = __builtin_amdgcn_readlane(b, (int)__builtin_ctzll(left));
    left &= ~__ballot(b == one);
    const int e0 = one * kTopBlock;
    frag_t<S> w[H / 32];
#pragma unroll
    for (int kk = 0; kk < H / 32; ++kk) w[kk] = load8(W + (size_t)min(e0 + q, c.V - 1) * H + 32 * kk + 8 * kg);
    f32x4 acc = {};
#pragma unroll
    for (int kk = 0; kk < H / 32; ++kk) mma(acc, w[kk], x[kk]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[j] += entry_bias(c.bias, e0 + 4 * kg + j, c.V);
      if (!(may >> j & 1)) acc[j] = -INFINITY;
    }
    if (b == one) *reinterpret_cast<f32x4*>(z + (size_t)pair[1] * kTopBlock + 4 * kg) = acc;
  }
}

// The answers from those logits, one wave a row.
template <typename S, int H>
__global__ __launch_bounds__(kVocThreads) void vocab_answer_kernel(TopRows c, const int32_t* __restrict__ block,
                                                                   const float* __restrict__ z,
                                                                   const S* __restrict__ X, const S* __restrict__ W) {
  __shared__ pick_t picks[kVocWaves][kWave];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = blockIdx.x * kVocWaves + wave;
  if (r >= c.R) return;   // whole waves leave together
  const int32_t* bl = block + (size_t)r * c.K;
  const float* zr = z + (size_t)r * c.K * kTopBlock;
  constexpr int G = kTopMost * kTopBlock / kWave;   // 64 entries, of four blocks, at a time
  // all blocks hold an entry that reaches the least of their maxima, and there are K
  uint32_t o[G], bound = ~0u;
  float zs[G];
  int of[G];   // (all on their way before the first is looked at)
#pragma unroll
  for (int i = 0; i < G; ++i) {
    if (4 * i < c.K) {
      of[i] = bl[min(4 * i + lane / 16, c.K - 1)];
      zs[i] = zr[min(64 * i + lane, c.K * kTopBlock - 1)];
    }
  }
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int at = 4 * i + lane / 16;
    o[i] = 0;
    if (4 * i < c.K) {
      o[i] = at < c.K && of[i] >= 0 ? order_of(zs[i]) : 0u;
      uint32_t m = o[i];
#pragma unroll
      for (int d = 1; d < 16; d *= 2) m = max(m, __shfl_xor(m, d));
      if (at < c.K) bound = min(bound, m);
    }
  }
#pragma unroll
  for (int d = 16; d < kWave; d *= 2) bound = min(bound, __shfl_xor(bound, d));
  bound = max(bound, 1u);
  Best best;
  bool spilled = false;
  int n = 0;
  const uint64_t below = (1ull << lane) - 1;
  auto take = [&](uint32_t v, uint32_t e) {   // what reaches the bound, to the list, which goes to `best` when full
    const uint64_t in = __ballot(v >= bound);
    if (in == 0) return;
    const int m = __popcll(in);
    if (n + m > kWave) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      best.add(lane < n ? picks[wave][lane] : 0, c.K, lane);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      n = 0;
      spilled = true;
    }
    if (v >= bound) picks[wave][n + __popcll(in & below)] = pick_of(v, e);
    n += m;
  };
#pragma unroll
  for (int i = 0; i < G; ++i) {
    if (4 * i < c.K) take(o[i], (uint32_t)(of[i] * kTopBlock + lane % 16));
  }
  RowSum own{kNoMax, c.te.near, 0.f};
  if (c.ent_id != nullptr) {
    const RowState<S, H> row(X, row_node(c.node, r, c.R, c.n_nodes), lane);
    rule_lists(c, row, W, r, 0, 1, own, take);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (spilled) {
    best.add(lane < n ? picks[wave][lane] : 0, c.K, lane);
    answer_list(best.k, r, c.K, lane, c.top, c.logit);
  } else {
    answer(picks[wave], n, r, c.K, lane, c.top, c.logit);
  }
  if (c.lse == nullptr) return;
  const int shares = c.deal.shares(r / c.share_rows);
  const size_t at0 = (size_t)c.deal.slot(r / c.share_rows) * c.share_rows + r % c.share_rows;
  float M, sum;
  RowBest none;
  join_shares<kWave, false>(shares, at0, c.share_rows, lane, c.pm, c.pl, nullptr, M, sum, none);
  join_own(own, M, sum);
  if (lane == 0) c.lse[r] = row_lse(M, sum, c.te);
}

}  // namespace dev

namespace {
// How a call is cut, and where its parts lie in the workspace.
struct TopPlan {
  bool few, sorted;
  int nt, splits, per, nbs, words;
  dev::Deal deal;
  size_t id, count, add, mask, bmax, pm, pl, wp, block, z, sort, bytes;
};
// Up to so many rows have a first pass of their own (vocab_max_few_kernel).  It against that
// of many rows, the whole call in us at K = 16, 1, 32 and 64 rows: bf16, H = 64, V = 10,007
// 11.3, 12.0, 12.8 / 12.7, 13.3, 13.5; H = 256, V = 50,021 23.4, 24.9, 27.9 / 31.7, 32.0,
// 32.6; float32, H = 64, V = 10,007 13.5, 14.4, 16.6 / 25.4, 25.7, 25.9; H = 256, V =
// 50,021 37.9, 40.2, 66.0 / 66.6, 67.0, 67.2, V = 5,000 27.6, 31.1, 46.2 / 38.9, 39.4, 40.7
// (33 to 64 float32 rows at H = 256 taken to be the other way).
constexpr int kTopFew = 64;
// Whether the picked blocks are sorted, which takes seven launches in place of one: by the
// bytes of W that they would gather, and kPairBytes for the rest of one launch's work a pair,
// against kSortBytes for the launches (both fitted to the times below; V, on which the sort
// and the blocks' launch depend a little, is left out).  One launch against seven, the whole
// call in us: bf16, V = 10,007, H = 64, K = 16, 1,000 rows 24 / 44, 3,001 44 / 55; V =
// 50,021, H = 128, K = 32, 1,500 rows 69 / 82, 2,999 118 / 110; H = 256, K = 16, 1,000
// rows 68 / 89, 2,000 108 / 111 (taken to be the other way), K = 8, 4,000 rows 159 / 156; V
// = 4,999, H = 32, K = 16, 8,000 rows 75 / 69; V = 50,021, K = 4, 129 / 141; float32, V =
// 4,999, H = 128, K = 16, 1,229 rows 56 / 59, 2,000 77 / 69.
constexpr double kPairBytes = 1000, kSortBytes = 2.55e8;
bool pairs_sorted(int es, int H, int R, int K) {
  return R > kTopFew && (double)R * K * (dev::kTopBlock * H * es + kPairBytes) > kSortBytes;   // (at most 2^30 pairs)
}
template <typename S>
TopPlan top_plan(int H, int R, int V, int K, int n_listed) {
  TopPlan p{};
  size_t shares;
  p.few = R <= kTopFew;
  if (p.few) {
    const int tiles = cdiv(V, 32);
    p.nt = R <= 32 ? 1 : 2;
    p.per = cdiv(tiles, 1024);
    p.splits = cdiv(cdiv(tiles, p.per), dev::kVocWaves) * dev::kVocWaves;
    shares = (size_t)p.splits * 32 * p.nt;
  } else {
    p.nt = dev::top_tiles<S>(H);
    p.deal = make_deal(cdiv(R, dev::top_rows<S>(H)), cdiv(V, dev::kTopUnit),
                       256 * dev::top_waves<S>(H) * 4 / dev::top_group<S>(H));
    shares = (size_t)p.deal.all_slots() * dev::top_rows<S>(H);
  }
  p.nbs = cdiv(V, dev::kTopUnit) * (dev::kTopUnit / dev::kTopBlock);
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
  p.sorted = pairs_sorted(sizeof(S), H, R, K);
  if (p.sorted) {
    p.block = take((size_t)R * K * 4);
    p.z = take((size_t)R * K * dev::kTopBlock * 4);
    p.sort = take(sort_workspace(R * K));
  }
  p.bytes = at;
  return p;
}

template <typename S, int H>
hipError_t top_h(const TopArgs& a, hipStream_t st) {
  using namespace dev;
  const TopPlan p = top_plan<S>(H, a.R, a.V, a.K, a.n_seen + a.n_add);
  char* ws = static_cast<char*>(a.ws);
  TopRows c{};
  c.n_nodes = a.n_nodes; c.R = a.R; c.V = a.V; c.K = a.K; c.nbs = p.nbs;
  c.splits = p.splits; c.share_rows = p.few ? 32 * p.nt : top_rows<S>(H); c.deal = p.deal;
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
    // A row's threads and its table's places by how long the lists are on average; its
    // workgroups: one, but where few rows may have lists that are passed over in parts.
    const int listed = a.n_seen + a.n_add;
    const bool longer = listed / a.R > 256;
    const int table = longer ? kTable : kTable / 4;
    const int parts = cdiv(a.V, table), most = a.R < 1024 ? 1024 / a.R : 1;
    const dim3 grid(a.R < kGridX ? a.R : kGridX, listed > table / 2 ? (parts < most ? parts : most) : 1,
                    cdiv(a.R, kGridX));
    const size_t lds = (size_t)table * 16;
    if (longer)
      hipLaunchKernelGGL((vocab_rules_kernel<S, 1024>), grid, dim3(1024), lds, st, a.R, a.V, c.list, c.rm, p.words, table,
                         out, id, count, add);
    else
      hipLaunchKernelGGL((vocab_rules_kernel<S, 256>), grid, dim3(256), lds, st, a.R, a.V, c.list, c.rm, p.words, table, out,
                         id, count, add);
    c.rm = RowMask{out, nullptr, a.R, p.words};
    c.ent_id = id; c.ent_count = count; c.ent_add = add;
    const hipError_t err = hipGetLastError();   // (the passes take entries from what this launch wrote)
    if (err != hipSuccess) return err;
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
      hipLaunchKernelGGL((vocab_max_kernel<S, H, LSE, MASK>), dim3(p.deal.workers), dim3(kWave* top_group<S>(H)), 0, st, \
                         a.n_nodes, a.R, a.V, p.deal, a.temper, X, Ws, a.bias, a.node, c.rm, bmax, p.nbs, pm, pl);     \
  } while (0)
  if (a.lse != nullptr) {
    if (c.rm.bits != nullptr) MAXIMA(true, true); else MAXIMA(true, false);
  } else {
    if (c.rm.bits != nullptr) MAXIMA(false, true); else MAXIMA(false, false);
  }
#undef MAXIMA
  if (p.sorted) {
    int32_t* block = reinterpret_cast<int32_t*>(ws + p.block);
    float* z = reinterpret_cast<float*>(ws + p.z);
    const int nb = cdiv(a.V, kTopBlock), pairs = a.R * a.K;
#define BLOCKS(GROUPS)                                                                                              \
  hipLaunchKernelGGL((vocab_blocks_kernel<S, GROUPS>), dim3(cdiv(a.R, kVocWaves)), dim3(kVocThreads), 0, st, a.R, nb, \
                     p.nbs, a.K, bmax, block)
    if (nb <= 512) BLOCKS(1);
    else if (nb <= 1024) BLOCKS(2);
    else if (nb <= 2048) BLOCKS(4);
    else BLOCKS(7);
#undef BLOCKS
    const void* sorted;
    const hipError_t err = launch_sort(pairs, nb, block, ws + p.sort, &sorted, st);
    if (err != hipSuccess) return err;
    const int groups = cdiv(pairs, 16 * kVocWaves);
    hipLaunchKernelGGL((vocab_pairs_kernel<S, H>), dim3(groups < kGridX ? groups : kGridX, cdiv(groups, kGridX)),
                       dim3(kVocThreads), 0, st, c, static_cast<const u32x2*>(sorted), pairs, X, W, z);
    hipLaunchKernelGGL((vocab_answer_kernel<S, H>), dim3(cdiv(a.R, kVocWaves)), dim3(kVocThreads), 0, st, c, block, z, X, W);
    return hipGetLastError();
  }
  if (p.few)
    hipLaunchKernelGGL((vocab_pick_kernel<S, H, 8>), dim3(a.R), dim3(8 * kWave), 0, st, c, X, W);
  else
    hipLaunchKernelGGL((vocab_pick_kernel<S, H, 4>), dim3(a.R), dim3(4 * kWave), 0, st, c, X, W);
  return hipGetLastError();
}
}  // namespace

namespace GGNN_IMPL_NS {
size_t top_workspace(int H, int R, int V, int K, int n_listed) {
  return top_plan<dev::dt_t>(H, R, V, K, n_listed).bytes;
}

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
