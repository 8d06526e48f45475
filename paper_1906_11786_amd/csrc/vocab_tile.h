// Parts that the passes over a vocabulary share (csrc/vocab.hip: the losses and their gradients; csrc/vocab_top.hip: the
// best entries): tiles of rows copied into LDS, rows as matrix-core fragments, exponents of logits of any size, how work
// is dealt to workgroups, and how shares of a row's sum are joined.
#pragma once

#include "device_common.h"
#include "kernels.h"
#include "lds_dma.h"

namespace ggnn {
namespace dev {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kVocThreads = 256, kVocWaves = 4;
constexpr int kVocRows = 128;              // rows (or vocabulary entries) of a workgroup, 32 per wave
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMaskedBias = -1e30f;      // a bias at or below takes its entry out
constexpr float kNoMax = -3e38f;           // running maximum before the first logit

// Exponents of a row's terms are z * k - m with m = z_max * k, in one fused
// multiply-add: k = near = log2 e / temperature, and the rounding of m is one factor of
// all terms, which the log sum takes out again.  From a logit of 2^29 temperatures on
// (`limit`) that rounding would pass the range of an exponential.  There k = far, the
// power of two above near (2 at a temperature of 1), which makes m exact: logits of this
// size are equal or at least 32 temperatures apart, so that any k gives the terms 1 and
// (to 2^-46) 0.  Maxima of both sizes keep their order, and differences that vanish,
// when compared as m.
__device__ __forceinline__ float exponent_factor(float z, const Temper& te) {
  return fabsf(z) >= te.limit ? te.far : te.near;
}
// The log sum of a row, of logits over the temperature, from its m and the sum of its terms.
__device__ __forceinline__ float log_of(float m, float sum, const Temper& te) {
  const float s = __log2f(sum);
  return fabsf(m) >= te.far * te.limit ? te.back * m + s * kLn2 : (m + s) * kLn2;
}

// The same in units of the logits, rounded once: what probabilities exp2(near (z - it)) start from.
// (log_of times the temperature has up to five roundings, U |lse| of a probability each;
// and from 2^29 temperatures on, where one step of it is many temperatures, a row's
// largest logit has to come back as it was, which M / far does.)
__device__ __forceinline__ float log_of_logits(float m, float sum, const Temper& te) {
  const double s = __log2f(sum);
  return (float)(fabsf(m) >= te.far * te.limit ? (double)(m / te.far) + s / te.near : (m + s) / te.near);
}

// float32 states and rows enter the matrix cores as three bf16 each (x = x0 +
// x1 + x2, exact), with the six products of order 2^-16 and up: 24 bits at 6
// bf16 products, where the float32 matrix instructions take 16 times a bf16
// product's time.  Probabilities, likewise, as three parts (two in bf16).
template <typename S> constexpr int voc_planes() { return sizeof(S) == 2 ? 1 : 3; }
template <typename S> constexpr int voc_parts() { return sizeof(S) == 2 ? 2 : 3; }
// Entries of an LDS tile: 64 in bf16, 32 in float32 (three times the bytes).
template <typename S> constexpr int voc_tile() { return sizeof(S) == 2 ? 64 : 32; }

__device__ __forceinline__ void mma32(f32x16& acc, const bf16x8& a, const bf16x8& b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
}
// (vocab_few_kernel's in float32, which waits for memory)
__device__ __forceinline__ void mma32(f32x16& acc, const f32x8& a, const f32x8& b) {
#pragma unroll
  for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], acc, 0, 0, 0);
}

// LDS tile: planes of T rows of H bf16 in 16-byte pieces; piece c of row r lies
// at place c ^ swz(r) of its row.  Sixteen rows read at one piece (fragments along
// H) and four rows times four pieces (fragments across rows) then both fall on
// different banks, without padding, so that the copies into LDS stay linear.
template <int H>
__device__ __forceinline__ int swz(int r) {
  constexpr int CPR = H / 8;
  if constexpr (CPR >= 16) return ((r & 3) << 2) | ((r >> 2) & 3);
  if constexpr (CPR == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  return (r >> 2) & 3;
}

// Copies rows row0 .. row0 + T - 1 (the last one's where beyond) of each plane
// to LDS; a plane holds `plane` elements.
template <int H, int NP, int T>
__device__ __forceinline__ void stage_tile(const bf16s* __restrict__ src, size_t plane, long row0, long last,
                                           uint32_t lds, int wave, int lane) {
  constexpr int CPR = H / 8, EACH = T * CPR / 64, PIECES = NP * EACH;   // 1 KB copies of a plane, and in all
#pragma unroll
  for (int p = 0; p < (PIECES + kVocWaves - 1) / kVocWaves; ++p) {
    const int piece = p * kVocWaves + wave, q = piece % EACH * 64 + lane;
    if (PIECES % kVocWaves != 0 && piece >= PIECES) break;
    const int r = q / CPR, c = (q % CPR) ^ swz<H>(r);
    const long row = row0 + r < last ? row0 + r : last;
    dma16(src + piece / EACH * plane + row * H + 8 * c,
          __builtin_amdgcn_readfirstlane(lds + (uint32_t)piece * 1024u));
  }
}

// Keeps the compiler from moving what forms v past this point.
template <typename V>
__device__ __forceinline__ void keep_here(V& v) { asm volatile("" : "+v"(v)); }

__device__ __forceinline__ float entry_bias(const float* bias, int v, int V) {
  if (v >= V) return -INFINITY;
  const float b = bias != nullptr ? bias[v] : 0.f;
  return b <= kMaskedBias ? -INFINITY : b;
}

// Accumulator start values: a[8 (j / 4) + 4 (lane / 32) + j % 4] of 32 floats in LDS.
__device__ __forceinline__ void start32(f32x16& acc, const float* a, int lane) {
#pragma unroll
  for (int j4 = 0; j4 < 4; ++j4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(a + 8 * j4 + 4 * (lane / 32));
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[4 * j4 + i] = v[i];
  }
}

struct RowBest {   // largest logit so far and the lowest entry that has it
  float z;
  int v;
};
__device__ __forceinline__ void take_best(RowBest& b, float z, int v) {
  if (z > b.z || (z == b.z && v < b.v)) b = RowBest{z, v};
}

// The row a lane stands for: its node, or -1 (beyond R, or outside the graph).
__device__ __forceinline__ int row_node(const int32_t* __restrict__ node, int r, int R, int n_nodes) {
  if (r >= R) return -1;
  const int i = node != nullptr ? node[r] : r;
  return (unsigned)i < (unsigned)n_nodes ? i : -1;
}
// A row's fragments along H, as they lie in memory (row < 0: zero).
template <typename S, int H>
__device__ __forceinline__ void load_row(frag_t<S> (&f)[H / 16], const S* __restrict__ X, long row, int lane) {
#pragma unroll
  for (int kk = 0; kk < H / 16; ++kk) {
    if (row >= 0) f[kk] = load8(X + row * H + 16 * kk + 8 * (lane / 32));
    else f[kk] = frag_t<S>{};
  }
}
// The same as planes of bf16.
template <typename S, int H>
__device__ __forceinline__ void load_planes(bf16x8 (&f)[voc_planes<S>()][H / 16], const S* __restrict__ X, long row,
                                            int lane) {
  frag_t<S> v[H / 16];
  load_row<S, H>(v, X, row, lane);
#pragma unroll
  for (int kk = 0; kk < H / 16; ++kk) {
    if constexpr (sizeof(S) == 2) {
      f[0][kk] = v[kk];
    } else {
#pragma unroll
      for (int a = 0; a < 3; ++a) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = pk2(v[kk][2 * i], v[kk][2 * i + 1]);
          v[kk][2 * i] -= lo_f(w[i]);
          v[kk][2 * i + 1] -= hi_f(w[i]);
        }
        f[a][kk] = __builtin_bit_cast(bf16x8, w);
      }
    }
  }
}
// Four elements as planes, `plane` elements apart.
__device__ __forceinline__ void store_planes(bf16s* p, size_t plane, f32x4 v, float) {
#pragma unroll
  for (int a = 0; a < 3; ++a) {
    const u32x2 w = u32x2{pk2(v[0], v[1]), pk2(v[2], v[3])};
    *reinterpret_cast<u32x2*>(p + a * plane) = w;
    v -= f32x4{lo_f(w[0]), hi_f(w[0]), lo_f(w[1]), hi_f(w[1])};
  }
}
__device__ __forceinline__ void store_planes(bf16s* p, size_t, f32x4 v, bf16s) { store4(p, v[0], v[1], v[2], v[3]); }

// Work is dealt in units of one LDS tile against one tile of 128 rows (or, in
// the columns pass, entries).  Many 128-tiles: `workers` workgroups first take
// whole ones, one each a round; those left over are laid end to end and cut into
// equal runs of units, so that all workgroups end together.  Few: each is cut
// into `parts` runs, one a worker, so that no worker starts twice.  A 128-tile is
// thus one share, or several workers' shares, joined afterwards in their order.
// (60,001 rows over 50,021 entries, 469 and 391 128-tiles for 256 workgroups: a
// round of whole tiles alone would leave the chip half idle in the last one.)
struct Deal {
  int workers, tiles;   // workgroups; LDS tiles against one 128-tile
  int whole, rest;      // 128-tiles dealt whole (a multiple of workers), and cut up
  int slots;            // shares of a 128-tile, at most
  int parts;            // of each 128-tile of the rest, or 0: cut end to end
  uint32_t each, more;  // units of a worker (or a part); the first `more` have one more
  __host__ __device__ uint32_t begin(uint32_t w) const { return w * each + (w < more ? w : more); }
  __host__ __device__ int owner(uint32_t u) const {   // worker that has unit u of the rest (parts = 0)
    const uint32_t k = more * (each + 1);
    return (int)(u < k ? u / (each + 1) : more + (u - k) / each);
  }
  // Where share 0 of 128-tile i is written: a whole one is one share, each of the
  // rest has room for `slots`.
  __host__ __device__ int slot(int i) const { return i < whole ? i : whole + (i - whole) * slots; }
  __host__ __device__ int all_slots() const { return whole + rest * slots; }
  // Shares of 128-tile i; share s of it is written to slot(i) + s.
  __host__ __device__ int shares(int i) const {
    if (i < whole) return 1;
    if (parts > 0) return parts;
    const uint32_t u = (uint32_t)(i - whole) * tiles;
    return owner(u + tiles - 1) - owner(u) + 1;
  }
};
// The next run of worker w: 128-tile, LDS tiles t0 .. t1 - 1, its slot.
struct Run {
  int i, t0, t1, slot;
};
struct Dealt {
  int step = 0;         // 128-tiles dealt whole so far
  uint32_t u, end;      // units of the rest (parts: the worker's run, once)
  __device__ __forceinline__ Dealt(const Deal& d, int w)
      : u(d.begin(d.parts > 0 ? w % d.parts : w)), end(d.begin((d.parts > 0 ? w % d.parts : w) + 1)) {}
  __device__ __forceinline__ bool next(const Deal& d, int w, Run* r) {
    if (step * d.workers < d.whole) {
      const int i = step * d.workers + w;
      *r = Run{i, 0, d.tiles, d.slot(i)};
      ++step;
      return true;
    }
    if (u >= end) return false;
    if (d.parts > 0) {
      *r = Run{w / d.parts, (int)u, (int)end, d.slot(w / d.parts) + w % d.parts};
      u = end;
      return true;
    }
    const uint32_t k = u / (uint32_t)d.tiles;
    r->i = d.whole + (int)k;
    r->t0 = (int)(u - k * d.tiles);
    r->t1 = min(d.tiles, r->t0 + (int)(end - u));
    r->slot = d.slot(r->i) + (r->t0 == 0 ? 0 : w - d.owner(k * d.tiles));
    u += r->t1 - r->t0;
    return true;
  }
};

constexpr int kVocBufs = 3;
__device__ __forceinline__ int next_buf(int b) { return b == kVocBufs - 1 ? 0 : b + 1; }
// Bytes from the buffer before `b` to buffer b.
template <uint32_t BYTES>
__device__ __forceinline__ uint32_t buf_step(int b) {
  return b == 0 ? 0u - (kVocBufs - 1) * BYTES : BYTES;
}

// One row's (m, l, best) from its shares, held by L neighbouring lanes (q: the
// lane's place); share s lies at at0 + s * stride.
template <int L, bool BEST>
__device__ __forceinline__ void join_shares(int n, size_t at0, size_t stride, int q, const float* __restrict__ pm,
                                            const float* __restrict__ pl, const RowBest* __restrict__ pb, float& M,
                                            float& sum, RowBest& best) {
  M = kNoMax;
  sum = 0.f;
  best = RowBest{-INFINITY, INT_MAX};
  constexpr int U = 4;   // shares in flight per lane
  for (int s0 = q; s0 < n; s0 += L * U) {
    float m[U], l[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u * L;
      const size_t at = at0 + (size_t)(s < n ? s : s0) * stride;
      m[u] = s < n ? pm[at] : kNoMax;
      l[u] = s < n ? pl[at] : 0.f;
      if (BEST && s < n) take_best(best, pb[at].z, pb[at].v);
    }
    float top = M;
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, m[u]);
    sum *= __builtin_amdgcn_exp2f(M - top);
#pragma unroll
    for (int u = 0; u < U; ++u) sum += l[u] * __builtin_amdgcn_exp2f(m[u] - top);
    M = top;
  }
#pragma unroll
  for (int o = L / 2; o >= 1; o /= 2) {
    const float m2 = __shfl_xor(M, o), s2 = __shfl_xor(sum, o), top = fmaxf(M, m2);
    sum = sum * __builtin_amdgcn_exp2f(M - top) + s2 * __builtin_amdgcn_exp2f(m2 - top);
    M = top;
    if (BEST) take_best(best, __shfl_xor(best.z, o), __shfl_xor(best.v, o));
  }
}
// lse of a row: -inf where every entry is masked.
__device__ __forceinline__ float row_lse(float M, float sum, const Temper& te) {
  return sum == 0.f ? -INFINITY : log_of(M, sum, te);
}
__device__ __forceinline__ float row_loss(float lse, float zt, int t, bool bad) {
  return bad ? NAN : t < 0 ? 0.f : lse == -INFINITY ? INFINITY : lse - zt;
}

}  // namespace dev

namespace {
inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
inline int cdiv(long a, long b) { return (int)((a + b - 1) / b); }

inline dev::Deal make_deal(int tiles128, int tiles, int workers) {
  dev::Deal d{};
  d.tiles = tiles;
  // Four tiles a worker pay for its start and its share; fewer where that
  // would leave compute units empty.
  const long all = (long)tiles128 * tiles, few = all < 256 ? all : 256, want = all / 4 > few ? all / 4 : few;
  d.workers = want < workers ? (int)want : workers;
  d.parts = d.workers / tiles128 >= 4 ? d.workers / tiles128 : 0;
  if (d.parts > 0) {
    d.workers = d.parts * tiles128;
    d.rest = tiles128;
    d.each = (uint32_t)tiles / d.parts;
    d.more = (uint32_t)tiles % d.parts;
    d.slots = d.parts;
    return d;
  }
  d.whole = tiles128 / d.workers * d.workers;
  d.rest = tiles128 - d.whole;
  const uint32_t units = (uint32_t)d.rest * (uint32_t)tiles;   // fewer than workers * tiles
  d.each = units / d.workers;
  d.more = units % d.workers;
  d.slots = 1;
  for (int i = d.whole; i < tiles128; ++i) {
    const int n = d.shares(i);
    if (n > d.slots) d.slots = n;
  }
  return d;
}
}  // namespace

}  // namespace ggnn
