// Cross entropy of chosen nodes over a vocabulary, and its gradients, without
// the logits in memory.
//
//   z_iv = x_i . w_v + b_v;  lse_i = log sum_v exp z_iv;  loss_i = lse_i - z_it
//   dz_iv = g_i (exp(z_iv - lse_i) - [v = t_i])
//   dX_i = sum_v dz_iv w_v;  dW_v += sum_i dz_iv x_i;  db_v += sum_i dz_iv
//
// Rows pass: a workgroup holds 128 rows of X as matrix-core fragments and
// walks a share of the vocabulary in tiles staged in LDS.  Logits are formed
// transposed (S^T = W X^T), so that a lane holds one row's logits: running
// maximum, sum and the weighted sum of vocabulary rows O_i = sum_v p_iv w_v
// need no exchange between lanes, and the probabilities are already in the
// fragment order of the second product.  The shares (m, l, O) of the
// vocabulary's splits are joined per row, which gives loss, lse and dX.
// Columns pass: the same with the roles of X and W exchanged, p from the known
// lse, which gives dW and db.
//
// Operations: the logits are formed twice, 2 RVH each (kept in memory they would
// be 6 GB at 60,001 rows over 50,021 entries in bf16, written once and read
// twice), and the two other products cost 4 RVH each in bf16: 12 RVH on the
// matrix cores.  In float32 every product is six bf16 ones: 48 RVH.
//
// Precision: dX and dW are float32, so in bf16 a probability enters the
// products as a bf16 pair (hi + lo, 16 bits); one bf16 would put the rounding
// of every probability, 2^-8, into both gradients.  In float32 states, entries
// and probabilities are three bf16 each.  Logits, maxima, sums and accumulators
// are float32.
//
// What bounds them: at H = 256 the matrix cores.  60,001 rows over 50,021 entries
// in bf16: rows pass 3,740 us, columns pass 3,900, 1.23 and 1.18 PFLOP/s, where a
// plain 8,192^3 product of the library runs at 1.32.  At H = 64 a step has a
// quarter of the products for the same 16 exponentials a lane, and no unit is full
// (vector issue 53% and 46%, matrix cores 32% and 30%, waiting 37% and 34%): 3,001 rows over
// 10,007 entries 22.8 and 23.2 us (0.51 PFLOP/s), then 8.5 and 6.9 us to add up the
// shares (25 and 23 MB, at memory speed).  Loss alone at H = 128, 2,999 rows over
// 50,021 entries: 53 us, 0.72 PFLOP/s (vector issue 57%, matrix cores 40%, waiting
// 44%); with the best entry 70.  float32 at H = 128, 1,229 rows over 4,999 entries:
// 28.7 and 27.9 us (0.65 PFLOP/s of bf16 products, matrix cores 40% busy: 250
// workgroups of 4 waves, one per SIMD, a wait for the copies every 32 entries).
#include <type_traits>

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
// multiply-add: k = log2 e, and the rounding of m is one factor of all terms, which
// the log sum takes out again.  From 2^29 on that rounding would pass the range of
// an exponential.  There k = 2, which makes m exact: logits of this size are equal
// or at least 32 apart, so that any k gives the terms 1 and (to 2^-46) 0.  Maxima of
// both sizes keep their order, and differences that vanish, when compared as m.
constexpr float kFarLogit = 536870912.f;
__device__ __forceinline__ float exponent_factor(float z) { return fabsf(z) >= kFarLogit ? 2.f : kLog2e; }
// The log sum of a row from its m and the sum of its terms.
__device__ __forceinline__ float log_of(float m, float sum) {
  const float s = __log2f(sum);
  return fabsf(m) >= 2.f * kFarLogit ? 0.5f * m + s * kLn2 : (m + s) * kLn2;
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

// ---- the two products of a 32 x 32 tile -----------------------------------
//
// One wave alone must keep its matrix core busy at H = 256, where a SIMD holds
// one, and an LDS read takes the time of several products.  So a step is laid
// out by hand: fragments are read kAhead before their product, and every
// product is followed by a share of the step's vector work, with the
// compiler's scheduler kept from moving anything between these slots (its own
// order read one fragment ahead and left the rest of the latency open).
//
// A step on tile rows r0 .. r0 + 31: logits of the next tile (fragments along
// H), then the second product of this one (fragments across rows, times the
// parts of p).  Of NP planes, products a, b with a + b >= 3 are left out.

typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;

template <int H, int NP, int T>
struct VocStep {
  static constexpr int NS = H / 16, NF = NS * NP;              // k steps; fragments of either product
  static constexpr int kAhead = NF < 8 ? NF : 8;
  static constexpr uint32_t ROW = H * 2, PLANE = T * ROW;      // bytes of a tile row and of a plane
  static constexpr int VS = NS < 8 ? NS : 8, VO = H / 32 < 4 ? H / 32 : 4;
  uint32_t as[VS], ao[2][VO];   // LDS addresses of the fragments; the other ones lie 256 bytes, rows or planes on
  bf16x8 f[2 * NF];             // at most kAhead are alive

  __device__ __forceinline__ void init(uint32_t lds, int lane) {
    const int r = lane % 32, g = lane / 32, p = lane % 16;
#pragma unroll
    for (int k = 0; k < VS; ++k) as[k] = lds + (uint32_t)r * ROW + 16u * ((2 * k + g) ^ swz<H>(r));
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int ht = 0; ht < VO; ++ht) {
        const int row = 8 * i + 4 * g + p / 4, c = 4 * ht + 2 * ((lane / 16) & 1) + (p % 4) / 2;
        ao[i][ht] = lds + (uint32_t)row * ROW + 16u * (c ^ swz<H>(row)) + 8u * (p % 2);
      }
  }
  __device__ __forceinline__ void move_s(uint32_t by) {
#pragma unroll
    for (int k = 0; k < VS; ++k) as[k] += by;
  }
  __device__ __forceinline__ void move_o(uint32_t by) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int ht = 0; ht < VO; ++ht) ao[i][ht] += by;
  }
  // Fragment n of a step.  n < NF: along H of the next tile, row rs + lane % 32,
  // elements 16 kk + 8 (lane / 32) .. + 7 of plane n % NP.  Else across the rows
  // of this one: column 32 ht + lane % 32, rows ro + 16 ks + {0, 8} + 4 (lane /
  // 32) + 0 .. 3, the order in which a lane holds the accumulators of a 32 x 32
  // tile.
  __device__ __forceinline__ void read(int n, int rs, int ro) {
    if (n < NF) {
      const int kk = n / NP;
      f[n] = __builtin_bit_cast(bf16x8, *(lds_u32x4*)(as[kk % VS] + 256u * (kk / VS) + (uint32_t)rs * ROW +
                                                      (uint32_t)(n % NP) * PLANE));
    } else {
      const int q = (n - NF) / NP, ks = q / (H / 32), ht = q % (H / 32);
      typedef short v8i16 __attribute__((ext_vector_type(8)));
      const uint32_t off = 256u * (ht / VO) + (uint32_t)(ro + 16 * ks) * ROW + (uint32_t)((n - NF) % NP) * PLANE;
      const tr_v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(ao[0][ht % VO] + off));
      const tr_v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(ao[1][ht % VO] + off));
      f[n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
  // The step's first reads.  LAST: number of the last fragment that it uses.
  template <int LAST>
  __device__ __forceinline__ void begin(int rs, int ro) {
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if (n <= LAST) read(n, rs, ro);
  }
  // s += logits of the next tile; work(i), i < 16, is done alongside.
  template <int LAST, typename Work>
  __device__ __forceinline__ void logits(f32x16& s, const bf16x8 (&x)[NP][NS], int rs, int ro, Work work) {
#pragma unroll
    for (int n = 0; n < NF; ++n) {
      if (n + kAhead <= LAST) read(n + kAhead, rs, ro);
#pragma unroll
      for (int b = 0; b + n % NP < NP; ++b) mma32(s, f[n], x[b][n / NP]);
#pragma unroll
      for (int i = n * 16 / NF; i < (n + 1) * 16 / NF; ++i) work(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // acc[ht] += (tile rows)^T p (lane's column, rows in accumulator order), p as
  // PARTS bf16 each; work(i), i < 4, is done alongside the first half, which
  // needs part[.][0] only, and late(i), i < 4, alongside the second.  NEXT: the
  // next step's first fragments, from rows rs, are read towards the end.
  template <int PARTS, bool NEXT, typename Work, typename Late>
  __device__ __forceinline__ void product(f32x16 (&acc)[H / 32], const u32x4 (&part)[PARTS][2], int rs, int ro,
                                          Work work, Late late) {
    constexpr int TOP = NP == 1 ? PARTS : NP;
#pragma unroll
    for (int n = 0; n < NF; ++n) {
      const int a = n % NP, ks = n / NP / (H / 32), ht = n / NP % (H / 32);
      if (n + kAhead < NF) read(NF + n + kAhead, rs, ro);
      else if (NEXT) read(n + kAhead - NF, rs, ro);
      mma32(acc[ht], f[NF + n], __builtin_bit_cast(bf16x8, part[0][ks]));
      if (ks == 0 && a == 0) {
#pragma unroll
        for (int i = ht * 4 / (H / 32); i < (ht + 1) * 4 / (H / 32); ++i) work(i);
      }
      if (ks == 1 && a == 0) {
#pragma unroll
        for (int i = ht * 4 / (H / 32); i < (ht + 1) * 4 / (H / 32); ++i) late(i);
      }
#pragma unroll
      for (int b = 1; b < PARTS && a + b < TOP; ++b) mma32(acc[ht], f[NF + n], __builtin_bit_cast(bf16x8, part[b][ks]));
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Two values as the i-th words of PARTS bf16 each, the next part the rest of the
// one before.  (Forming the rest with a bf16 dot product, which needs no
// unpacking, took 2% longer: its results may be read late only.)
template <int PARTS>
__device__ __forceinline__ void split2(float a, float b, u32x4 (&part)[PARTS][2], int ks, int i) {
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    const uint32_t h = pk2(a, b);
    part[q][ks][i] = h;
    a -= lo_f(h);
    b -= hi_f(h);
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

// The planes of a float32 matrix, `count` (a multiple of 4) elements: once a
// call, so that no workgroup splits the rows that it stages.  3.1 us for 4,999 x
// 128.
template <typename S>
__global__ __launch_bounds__(kVocThreads) void vocab_planes_kernel(size_t count, const S* __restrict__ W,
                                                                   bf16s* __restrict__ out) {
  const size_t i = 4 * ((size_t)blockIdx.x * kVocThreads + threadIdx.x);
  if (i < count) store_planes(out + i, count, load4f(W + i), S{});
}

// The tiles of a workgroup's share pass through three LDS buffers: while one
// is used, the next one has landed or is landing, and the copies of the one
// after it go to the buffer that every wave left before the last barrier.
// Within a wave the logits of the next 32 entries are formed before the
// current ones are turned into probabilities, so that the matrix cores have
// work during the exponentials.  With two steps to a tile (bf16) the next tile is
// waited for between the two products of the first step, so that either step's
// first fragments are read during the products before it (against reading them at
// the step's start: rows pass 3,775 -> 3,713 us, columns pass 4,090 -> 3,980, 60,001
// rows, in turn on one card).
//
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

// Workgroups of a pass that a compute unit holds (waves per SIMD): by the
// accumulators and fragments that a wave keeps, and at H = 256 by the buffers.
template <typename S>
constexpr int voc_waves(int H, bool sum) {
  if (sizeof(S) == 4) return H >= 256 ? 1 : H == 128 ? (sum ? 1 : 2) : H == 64 ? 2 : 3;
  return H >= 256 ? 1 : H == 128 ? (sum ? 2 : 3) : H == 64 ? 3 : 4;
}

constexpr int kVocBufs = 3;
__device__ __forceinline__ int next_buf(int b) { return b == kVocBufs - 1 ? 0 : b + 1; }
// Bytes from the buffer before `b` to buffer b.
template <uint32_t BYTES>
__device__ __forceinline__ uint32_t buf_step(int b) {
  return b == 0 ? 0u - (kVocBufs - 1) * BYTES : BYTES;
}

// Rows pass.  Writes each row's (m in units of log 2, l) of a share to pm, pl
// [slot][128]; SUM: O too; BEST: the largest logit's entry too; BIAS: there is
// one (without, the logits' products start from zero, 16 registers less to set
// a step).  A small dX is cleared here, `clear` 16-byte pieces per thread (0:
// elsewhere).
template <typename S, int H, bool SUM, bool BEST, bool BIAS>
__global__ __launch_bounds__(kVocThreads, voc_waves<S>(H, SUM)) void vocab_rows_kernel(int n_nodes, int R, int V, Deal deal,
                                                                 const S* __restrict__ X,
                                                                 const bf16s* __restrict__ W,
                                                                 const float* __restrict__ bias,
                                                                 const int32_t* __restrict__ node,
                                                                 float* __restrict__ pm, float* __restrict__ pl,
                                                                 float* __restrict__ po, RowBest* __restrict__ pb,
                                                                 float* __restrict__ dX, int clear) {
  constexpr int T = voc_tile<S>(), NP = voc_planes<S>(), P = voc_parts<S>();
  using Step = VocStep<H, NP, T>;
  __shared__ __attribute__((aligned(1024))) bf16s tile[kVocBufs][NP * T * H];
  __shared__ __attribute__((aligned(16))) float tb[BIAS ? kVocBufs : 1][T];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = lane / 32;
  const uint32_t lds0 = (uint32_t)(uintptr_t)tile[0];

  if constexpr (SUM) {
    const size_t all = (size_t)n_nodes * (H / 4), each = (size_t)clear * kVocThreads;
    for (int k = 0; k < clear; ++k) {
      const size_t at = blockIdx.x * each + (size_t)k * kVocThreads + threadIdx.x;
      if (at < all) reinterpret_cast<f32x4*>(dX)[at] = f32x4{};
    }
  }
  float nb = 0.f;
  Run run;
  Dealt dealt(deal, blockIdx.x);
  for (int round = 0; dealt.next(deal, blockIdx.x, &run); ++round) {
    const int t0 = run.t0, t1 = run.t1;
    bf16x8 xf[NP][H / 16];
    f32x16 o[H / 32];
    if constexpr (SUM) {
#pragma unroll
      for (int ht = 0; ht < H / 32; ++ht) o[ht] = f32x16{};
    }
    float m = kNoMax, k = kLog2e, l = 0.f;   // k: the row's exponent_factor
    RowBest best{-INFINITY, INT_MAX};
    auto fetch = [&](int t, int buf) {   // start the copies of tile t < t1
      stage_tile<H, NP, T>(W, (size_t)V * H, (long)t * T, V - 1, lds0 + (uint32_t)buf * NP * Step::PLANE, wave,
                           lane);
      // (the raw value: a use here would wait for the copies too)
      if (BIAS && threadIdx.x < T) nb = bias[min(t * T + (int)threadIdx.x, V - 1)];
    };
    auto land = [&](int t, int buf) {   // and wait for those started last, of tile t
      if (BIAS && threadIdx.x < T)
        tb[buf][threadIdx.x] = t * T + (int)threadIdx.x >= V || nb <= kMaskedBias ? -INFINITY : nb;
      wait_copies<0>();
      __syncthreads();
    };
    auto start = [&](f32x16& s, int buf, int r0) {   // biases of a tile's entries
      if constexpr (BIAS) start32(s, tb[buf] + r0, lane);
      else s = f32x16{};
    };
    if (round > 0) __syncthreads();   // every wave has left the buffers of the run before
    Step step;
    step.init(lds0, lane);
    f32x16 s;
    int buf = 0;
    fetch(t0, 0);
    load_planes<S, H>(xf, X, row_node(node, run.i * kVocRows + wave * 32 + lane % 32, R, n_nodes), lane);
    land(t0, 0);
    if (t0 + 1 < t1) fetch(t0 + 1, 1);
    start(s, 0, 0);
    step.template begin<Step::NF - 1>(0, 0);
    step.template logits<Step::NF - 1>(s, xf, 0, 0, [](int) {});
    auto mask = [&](f32x16& z, int first) {   // the last tile: entries beyond V (with a bias, the bias is -inf there)
      if (!BIAS && first + 32 > V) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (first + 8 * (j / 4) + 4 * g + j % 4 >= V) z[j] = -INFINITY;
      }
    };
    mask(s, t0 * T);
    float top = s[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) top = fmaxf(top, s[j]);
    constexpr bool kPipe = SUM && T == 64;   // the next tile is waited for within the first step, fragments read a step ahead
    constexpr int LAST = (SUM ? 2 : 1) * Step::NF - 1;
    if constexpr (kPipe) step.template begin<LAST>(32, 0);
    for (int t = t0; t < t1; ++t) {
      const int nbuf = next_buf(buf);
#pragma unroll
      for (int r0 = 0; r0 < T; r0 += 32) {
        const bool last = r0 + 32 >= T;
        const int rs = last ? 0 : r0 + 32;   // of the next tile (after the last one: of what the buffer holds, not used)
        auto turn = [&]() {
          land(t + 1, nbuf);
          if (t + 2 < t1) fetch(t + 2, next_buf(nbuf));
          step.move_s(buf_step<NP * Step::PLANE>(nbuf));
        };
        if constexpr (!kPipe) {
          if (last) turn();
          step.template begin<LAST>(rs, r0);
        }
        f32x16 sn;
        start(sn, last ? nbuf : buf, rs);
        // The maximum follows only where it would grow by more than 2^8: until
        // then the terms stay below 2^8 and the sums lose nothing.
        if (__ballot(top * k > m + 8.f)) {
          const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
          const float z = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])), kn = exponent_factor(z);
          const float mn = fmaxf(m, z * kn);
          if (mn > m) k = kn;
          const float f = __builtin_amdgcn_exp2f(m - mn);
          m = mn;
          l *= f;
          if constexpr (SUM) {
#pragma unroll
            for (int ht = 0; ht < H / 32; ++ht)
#pragma unroll
              for (int j = 0; j < 16; ++j) o[ht][j] *= f;
          }
        }
        float p[16];
        auto prob = [&](int j) {
          if constexpr (BEST) {
            if (s[j] > best.z) best = RowBest{s[j], t * T + r0 + 8 * (j / 4) + 4 * g + j % 4};
          }
          p[j] = __builtin_amdgcn_exp2f(fmaf(s[j], k, -m));
          l += p[j];
        };
        u32x4 part[P][2];
        __builtin_amdgcn_sched_barrier(0);
        step.template logits<LAST>(sn, xf, rs, r0, [&](int j) {
          prob(j);
          if (SUM && j >= 8 && j % 2 == 1) split2(p[j - 9], p[j - 8], part, 0, (j - 9) / 2);
        });
        if (kPipe && !last) turn();
        mask(sn, (last ? (t + 1) * T : t * T) + rs);
        float topn = sn[0];
        auto grow = [&](int i) {
#pragma unroll
          for (int j = 4 * i; j < 4 * i + 4; ++j) topn = fmaxf(topn, sn[j]);
        };
        if constexpr (SUM) {
          step.template product<P, kPipe>(o, part, last ? 32 : 0, r0,
                                          [&](int i) { split2(p[8 + 2 * i], p[9 + 2 * i], part, 1, i); }, grow);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) grow(i);
        }
        s = sn;
        top = topn;
      }
      if constexpr (SUM) step.move_o(buf_step<NP * Step::PLANE>(nbuf));
      buf = nbuf;
    }
    l += __shfl_xor(l, 32);
    const size_t at = (size_t)run.slot * kVocRows + wave * 32 + lane % 32;
    if constexpr (BEST) {
      take_best(best, __shfl_xor(best.z, 32), __shfl_xor(best.v, 32));
      if (g == 0) pb[at] = best;
    }
    if (g == 0) {
      pm[at] = m;
      pl[at] = l;
    }
    if constexpr (SUM) {
#pragma unroll
      for (int ht = 0; ht < H / 32; ++ht)
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4)
          *reinterpret_cast<f32x4*>(po + at * H + 32 * ht + 8 * j4 + 4 * g) =
              f32x4{o[ht][4 * j4], o[ht][4 * j4 + 1], o[ht][4 * j4 + 2], o[ht][4 * j4 + 3]};
    }
  }
}

// Rows pass for at most 32 rows (loss only): every wave holds the same rows
// and takes `per` tiles of 32 entries, read straight from memory, since no
// other wave needs them.  Bound by memory's latency and the launch: 4.8 us for
// one row over 10,007 entries at H = 64 (1.3 MB).
template <typename S, int H, bool BEST>
__global__ __launch_bounds__(kVocThreads) void vocab_few_kernel(int n_nodes, int R, int V, int per,
                                                                const S* __restrict__ X, const S* __restrict__ W,
                                                                const float* __restrict__ bias,
                                                                const int32_t* __restrict__ node,
                                                                float* __restrict__ pm, float* __restrict__ pl,
                                                                RowBest* __restrict__ pb) {
  const int lane = threadIdx.x % kWave, g = lane / 32, r = lane % 32;
  const int split = blockIdx.x * kVocWaves + threadIdx.x / kWave;
  const int tiles = (V + 31) / 32, t0 = split * per, t1 = min(tiles, t0 + per);
  frag_t<S> xf[H / 16];
  load_row<S, H>(xf, X, row_node(node, r, R, n_nodes), lane);
  float m = kNoMax, k = kLog2e, l = 0.f;
  RowBest best{-INFINITY, INT_MAX};
  for (int t = t0; t < t1; ++t) {
    frag_t<S> wf[H / 16];
    load_row<S, H>(wf, W, min(t * 32 + r, V - 1), lane);
    f32x16 s;
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] = entry_bias(bias, t * 32 + 8 * (j / 4) + 4 * g + j % 4, V);
#pragma unroll
    for (int kk = 0; kk < H / 16; ++kk) mma32(s, wf[kk], xf[kk]);
    float top = s[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) top = fmaxf(top, s[j]);
    const float kn = exponent_factor(top), mn = fmaxf(m, top * kn);
    if (mn > m) k = kn;
    l *= __builtin_amdgcn_exp2f(m - mn);
    m = mn;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if constexpr (BEST) {
        if (s[j] > best.z) best = RowBest{s[j], t * 32 + 8 * (j / 4) + 4 * g + j % 4};
      }
      l += __builtin_amdgcn_exp2f(fmaf(s[j], k, -m));
    }
  }
  const float m2 = __shfl_xor(m, 32), l2 = __shfl_xor(l, 32), mn = fmaxf(m, m2);
  l = l * __builtin_amdgcn_exp2f(m - mn) + l2 * __builtin_amdgcn_exp2f(m2 - mn);
  const size_t at = (size_t)split * 32 + r;
  if constexpr (BEST) {
    take_best(best, __shfl_xor(best.z, 32), __shfl_xor(best.v, 32));
    if (g == 0) pb[at] = best;
  }
  if (g == 0) {
    pm[at] = mn;
    pl[at] = l;
  }
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
__device__ __forceinline__ float row_lse(float M, float sum) {
  return sum == 0.f ? -INFINITY : log_of(M, sum);
}
__device__ __forceinline__ float row_loss(float lse, float zt, int t, bool bad) {
  return bad ? NAN : t < 0 ? 0.f : lse == -INFINITY ? INFINITY : lse - zt;
}

// The loss of at most 32 rows from the many shares of vocab_few_kernel: one
// workgroup per row.  3.0 us, latency.
template <typename S, int H, bool BEST>
__global__ __launch_bounds__(kVocThreads) void vocab_few_join_kernel(
    int n_nodes, int R, int V, int splits, const S* __restrict__ X, const S* __restrict__ W,
    const float* __restrict__ bias, const int32_t* __restrict__ node, const int32_t* __restrict__ target,
    const float* __restrict__ pm, const float* __restrict__ pl, const RowBest* __restrict__ pb,
    float* __restrict__ loss, float* __restrict__ lse, int32_t* __restrict__ best) {
  __shared__ float wm[kVocWaves], wl[kVocWaves], wz[kVocWaves];
  __shared__ RowBest wb[kVocWaves];
  const int r = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int n = row_node(node, r, R, n_nodes);
  int t = n >= 0 && target != nullptr ? target[r] : -1;
  const bool bad = t >= V;
  if (bad) t = -1;
  float z = 0.f;
  if (t >= 0 && threadIdx.x < H) z = to_f<S>(X[(size_t)n * H + threadIdx.x]) * to_f<S>(W[(size_t)t * H + threadIdx.x]);
  // each wave takes every fourth share
  float M, sum;
  RowBest b;
  join_shares<kWave, BEST>((splits - wave + kVocWaves - 1) / kVocWaves, (size_t)wave * 32 + r, (size_t)kVocWaves * 32,
                           lane, pm, pl, pb, M, sum, b);
#pragma unroll
  for (int o = kWave / 2; o >= 1; o /= 2) z += __shfl_xor(z, o);
  if (lane == 0) {
    wm[wave] = M;
    wl[wave] = sum;
    wz[wave] = z;
    wb[wave] = b;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kVocWaves; ++w) {
    const float top = fmaxf(M, wm[w]);
    sum = sum * __builtin_amdgcn_exp2f(M - top) + wl[w] * __builtin_amdgcn_exp2f(wm[w] - top);
    M = top;
    z += wz[w];
    if (BEST) take_best(b, wb[w].z, wb[w].v);
  }
  const float v = row_lse(M, sum);
  lse[r] = v;
  if (loss != nullptr) loss[r] = row_loss(v, t >= 0 ? z + entry_bias(bias, t, V) : 0.f, t, bad);
  if (BEST) best[r] = b.v == INT_MAX ? -1 : b.v;
}

// Joins the shares of a row: H / 4 lanes per row, four features each.  GRAD:
// writes dX's row, and what the columns pass reads: the row's state, its lse,
// target and factor.  A row without a gradient, and those that fill the last
// 128-tile, has a zero state, an infinite lse (its probabilities vanish), target
// -1 and factor 0.  Bound by the shares' bytes: 8.4 us for 3,001 rows of 32 shares
// at H = 64 (25 MB), 54 us for 60,001 rows at H = 256.
template <typename S, int H, bool GRAD, bool BEST>
__global__ __launch_bounds__(kVocThreads) void vocab_join_kernel(
    int n_nodes, int R, int V, int Rp, Deal deal, const S* __restrict__ X, const S* __restrict__ W,
    const float* __restrict__ bias, const int32_t* __restrict__ node, const int32_t* __restrict__ target,
    const float* __restrict__ weight, float scale, const float* __restrict__ pm, const float* __restrict__ pl,
    const float* __restrict__ po, const RowBest* __restrict__ pb, float* __restrict__ loss, float* __restrict__ lse,
    int32_t* __restrict__ best, float* __restrict__ dX, bf16s* __restrict__ xg, float* __restrict__ lse_w,
    int32_t* __restrict__ tgt_w, float* __restrict__ fac_w) {
  constexpr int L = H / 4;
  const int r = (int)(((long)blockIdx.x * kVocThreads + threadIdx.x) / L);
  const int q = threadIdx.x % L, h = 4 * q;
  if (r >= (GRAD ? Rp : R)) return;   // whole groups of L lanes leave together
  const int n = row_node(node, r, R, n_nodes);
  const f32x4 x = n >= 0 ? load4f(X + (size_t)n * H + h) : f32x4{};
  const int shares = r < R ? deal.shares(r / kVocRows) : 0;
  const size_t at0 = (size_t)deal.slot(r / kVocRows) * kVocRows + r % kVocRows;
  int t = n >= 0 && target != nullptr ? target[r] : -1;
  const bool bad = t >= V;
  if (bad) t = -1;
  const f32x4 w = t >= 0 ? load4f(W + (size_t)t * H + h) : f32x4{};
  float M, sum;
  RowBest b;
  join_shares<L, BEST>(shares, at0, kVocRows, q, pm, pl, pb, M, sum, b);
  float zt = x[0] * w[0] + x[1] * w[1] + x[2] * w[2] + x[3] * w[3];
#pragma unroll
  for (int o = L / 2; o >= 1; o /= 2) zt += __shfl_xor(zt, o);
  const float v = row_lse(M, sum);
  if (r < R && q == 0) {
    lse[r] = v;
    if (loss != nullptr) loss[r] = row_loss(v, t >= 0 ? zt + entry_bias(bias, t, V) : 0.f, t, bad);
    if (BEST) best[r] = b.v == INT_MAX ? -1 : b.v;
  }
  if constexpr (GRAD) {
    const float f = (weight != nullptr && r < R ? weight[r] : 1.f) * scale;
    const bool live = t >= 0 && sum != 0.f;
    store_planes(xg + (size_t)r * H + h, (size_t)Rp * H, live ? x : f32x4{}, S{});
    if (q == 0) {
      lse_w[r] = live ? v : INFINITY;
      tgt_w[r] = live ? t : -1;
      fac_w[r] = live ? f : 0.f;   // (whatever an ignored row holds: a product with its zero probability)
    }
    if (live) {
      f32x4 o = {};
#pragma unroll 8
      for (int s = 0; s < shares; ++s) {
        const size_t at = at0 + (size_t)s * kVocRows;
        o += *reinterpret_cast<const f32x4*>(po + at * H + h) * __builtin_amdgcn_exp2f(pm[at] - M);
      }
      *reinterpret_cast<f32x4*>(dX + (size_t)n * H + h) = (o * (1.f / sum) - w) * f;
    }
  }
}

// Columns pass: 128 entries of a workgroup (32 per wave) against the gathered
// states.  Adds to dW [V][H] and db [V] (dbias NULL: none) where the 128-tile is
// one share, else writes its share to pw [slot][128][H] and pdb [slot][128], slots
// from the first tile of the rest on.
// WEIGHT: each row has a factor of its own; otherwise all have `scale`.  TARGETS:
// see below.
template <typename S, int H, bool WEIGHT, bool TARGETS>
__global__ __launch_bounds__(kVocThreads, voc_waves<S>(H, true)) void vocab_cols_kernel(int V, int Rp, Deal deal, float scale,
                                                                 const bf16s* __restrict__ xg,
                                                                 const S* __restrict__ W,
                                                                 const float* __restrict__ bias,
                                                                 const float* __restrict__ lse_w,
                                                                 const int32_t* __restrict__ tgt_w,
                                                                 const float* __restrict__ fac_w,
                                                                 float* __restrict__ dW, float* __restrict__ dbias,
                                                                 float* __restrict__ pw, float* __restrict__ pdb) {
  constexpr int T = voc_tile<S>(), NP = voc_planes<S>(), P = voc_parts<S>();
  using Step = VocStep<H, NP, T>;
  __shared__ __attribute__((aligned(1024))) bf16s tile[kVocBufs][NP * T * H];
  __shared__ __attribute__((aligned(16))) float tl[kVocBufs][T], tf[kVocBufs][T];
  __shared__ __attribute__((aligned(16))) int tt[kVocBufs][T];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = lane / 32;
  const uint32_t lds0 = (uint32_t)(uintptr_t)tile[0];

  float nl = 0.f, nf = 0.f;
  int nt = -1;
  Run run;
  Dealt dealt(deal, blockIdx.x);
  for (int round = 0; dealt.next(deal, blockIdx.x, &run); ++round) {
    const int t0 = run.t0, t1 = run.t1, vw = run.i * kVocRows + wave * 32, v = vw + lane % 32;
    bf16x8 wf[NP][H / 16];
    f32x16 a[H / 32];
#pragma unroll
    for (int ht = 0; ht < H / 32; ++ht) a[ht] = f32x16{};
    float db = 0.f;
    auto fetch = [&](int t, int buf) {   // start the copies of tile t < t1
      stage_tile<H, NP, T>(xg, (size_t)Rp * H, (long)t * T, Rp - 1, lds0 + (uint32_t)buf * NP * Step::PLANE, wave,
                           lane);
      if (threadIdx.x < T) {
        nl = lse_w[t * T + threadIdx.x];
        nt = tgt_w[t * T + threadIdx.x];
        if constexpr (WEIGHT) nf = fac_w[t * T + threadIdx.x];
      }
    };
    auto land = [&](int buf) {   // and wait for those started last
      if (threadIdx.x < T) {
        tl[buf][threadIdx.x] = -nl;
        tt[buf][threadIdx.x] = nt;
        if constexpr (WEIGHT) tf[buf][threadIdx.x] = nf;
      }
      wait_copies<0>();
      __syncthreads();
    };
    if (round > 0) __syncthreads();   // every wave has left the buffers of the run before
    Step step;
    step.init(lds0, lane);
    f32x16 s;
    int buf = 0;
    fetch(t0, 0);
    load_planes<S, H>(wf, W, min(v, V - 1), lane);
    const float b2 = entry_bias(bias, v, V) * kLog2e;
    land(0);
    if (t0 + 1 < t1) fetch(t0 + 1, 1);
    start32(s, tl[0], lane);
    step.template begin<Step::NF - 1>(0, 0);
    step.template logits<Step::NF - 1>(s, wf, 0, 0, [](int) {});
    constexpr bool kPipe = T == 64;   // as in the rows pass
    constexpr int LAST = 2 * Step::NF - 1;
    if constexpr (kPipe) step.template begin<LAST>(32, 0);
    for (int t = t0; t < t1; ++t) {
      const int nbuf = next_buf(buf);
#pragma unroll
      for (int r0 = 0; r0 < T; r0 += 32) {
        const bool last = r0 + 32 >= T;
        const int rs = last ? 0 : r0 + 32;   // of the next tile (after the last one: of what the buffer holds, not used)
        auto turn = [&]() {
          land(nbuf);
          if (t + 2 < t1) fetch(t + 2, next_buf(nbuf));
          step.move_s(buf_step<NP * Step::PLANE>(nbuf));
        };
        if constexpr (!kPipe) {
          if (last) turn();
          step.template begin<LAST>(rs, r0);
        }
        f32x16 sn;
        start32(sn, tl[last ? nbuf : buf] + rs, lane);
        const int tj = tt[buf][r0 + lane % 32];
        float p[16];
        u32x4 part[P][2];
        constexpr bool kFinal = sizeof(S) == 2 && !WEIGHT;   // what follows leaves p as it is
        auto prob = [&](int j) {
          p[j] = __builtin_amdgcn_exp2f(fmaf(s[j], kLog2e, b2));
          keep_here(p[j]);
          if (kFinal && j >= 8 && j % 2 == 1) {
            split2(p[j - 9], p[j - 8], part, 0, (j - 9) / 2);
#pragma unroll
            for (int q = 0; q < P; ++q) {
              uint32_t w = part[q][0][(j - 9) / 2];
              keep_here(w);
              part[q][0][(j - 9) / 2] = w;
            }
          }
        };
        __builtin_amdgcn_sched_barrier(0);
        step.template logits<LAST>(sn, wf, rs, r0, prob);
        // Whether a row's target falls on this wave's entries; its share of db.  (The
        // branch also keeps the compiler from moving the exponentials away from
        // the logits' products.)
        const bool hit = __ballot((unsigned)(tj - vw) < 32u) != 0;
        if (hit) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int i = r0 + 8 * (j / 4) + 4 * g + j % 4;
            if (tt[buf][i] == v) {
              if (sizeof(S) == 4 && TARGETS) p[j] -= 1.f;   // float32 loses nothing
              else db -= WEIGHT ? tf[buf][i] : 1.f;
            }
          }
        }
        if constexpr (WEIGHT) {
#pragma unroll
          for (int j = 0; j < 16; ++j) p[j] *= tf[buf][r0 + 8 * (j / 4) + 4 * g + j % 4];
        }
        if constexpr (!kFinal) {
#pragma unroll
          for (int i = 0; i < 4; ++i) split2(p[2 * i], p[2 * i + 1], part, 0, i);
        }
        if (kPipe && !last) turn();
        const int rn = last ? 32 : 0;   // of the next step's logits
        step.template product<P, kPipe>(
            a, part, rn, r0,
            [&](int i) {
              split2(p[8 + 2 * i], p[9 + 2 * i], part, 1, i);
              db += (p[4 * i] + p[4 * i + 1]) + (p[4 * i + 2] + p[4 * i + 3]);
            },
            [](int) {});
        // In bf16 the target's share of dW is a product of its own, since a pair of
        // p - 1 would lose low bits of p to the 1.  (Without TARGETS it comes from
        // launch_target_rows.)
        if (sizeof(S) == 2 && TARGETS && hit) {
          float q[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int i = r0 + 8 * (j / 4) + 4 * g + j % 4;
            q[j] = tt[buf][i] != v ? 0.f : WEIGHT ? -tf[buf][i] : -1.f;
          }
#pragma unroll
          for (int n = 0; n < (WEIGHT ? 3 : 1); ++n) {   // -1 is one bf16, any float32 three
            u32x4 e[1][2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t h = pk2(q[2 * i], q[2 * i + 1]);
              e[0][i / 4][i % 4] = h;
              q[2 * i] -= lo_f(h);
              q[2 * i + 1] -= hi_f(h);
            }
#pragma unroll
            for (int k = 0; k < step.kAhead; ++k) step.read(Step::NF + k, 0, r0);
            step.template product<1, false>(a, e, 0, r0, [](int) {}, [](int) {});
          }
          if constexpr (kPipe) step.template begin<Step::NF - 1>(rn, r0);   // (rather than kept during these products)
        }
        s = sn;
      }
      step.move_o(buf_step<NP * Step::PLANE>(nbuf));
      buf = nbuf;
    }
    const float f = WEIGHT ? 1.f : scale;
    db = (db + __shfl_xor(db, 32)) * f;
    if (v < V) {
      const bool only = deal.shares(run.i) == 1;   // no one else adds to these rows
      const size_t at = only ? 0 : (size_t)(run.slot - deal.whole) * kVocRows + wave * 32 + lane % 32;
      if (dbias != nullptr && g == 0) {
        if (only) dbias[v] += db;
        else pdb[at] = db;
      }
      float* out = only ? dW + (size_t)v * H : pw + at * H;
#pragma unroll
      for (int ht = 0; ht < H / 32; ++ht)
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4) {
          f32x4* q = reinterpret_cast<f32x4*>(out + 32 * ht + 8 * j4 + 4 * g);
          f32x4 w = f32x4{a[ht][4 * j4], a[ht][4 * j4 + 1], a[ht][4 * j4 + 2], a[ht][4 * j4 + 3]} * f;
          if (only) w += *q;
          *q = w;
        }
    }
  }
}

// dW and db of the 128-tiles that several shares make up: += their sum, in
// share order.  H / 4 lanes per entry, four features each.  Bound by the shares'
// bytes: 6.9 us for 79 tiles of 9 shares at H = 64 (23 MB).
template <int H>
__global__ __launch_bounds__(kVocThreads) void vocab_wsum_kernel(int V, Deal deal, const float* __restrict__ pw,
                                                                 const float* __restrict__ pdb,
                                                                 float* __restrict__ dW, float* __restrict__ dbias) {
  constexpr int L = H / 4;
  const long v = (long)deal.whole * kVocRows + ((long)blockIdx.x * kVocThreads + threadIdx.x) / L;
  const int q = threadIdx.x % L;
  if (v >= V) return;
  const int i = (int)(v / kVocRows), n = deal.shares(i);
  if (n == 1) return;
  const size_t at = (size_t)(i - deal.whole) * deal.slots * kVocRows + v % kVocRows;
  f32x4 w = {};
#pragma unroll 8
  for (int s = 0; s < n; ++s) w += *reinterpret_cast<const f32x4*>(pw + (at + (size_t)s * kVocRows) * H + 4 * q);
  *reinterpret_cast<f32x4*>(dW + v * H + 4 * q) += w;
  if (dbias != nullptr && q == 0) {
    float b = 0.f;
#pragma unroll 8
    for (int s = 0; s < n; ++s) b += pdb[at + (size_t)s * kVocRows];
    dbias[v] += b;
  }
}

}  // namespace dev

namespace {
inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
inline int cdiv(long a, long b) { return (int)((a + b - 1) / b); }

// Workgroups that the chip's 256 compute units hold at once.
template <typename S>
int voc_workers(int H, bool sum) {
  return 256 * dev::voc_waves<S>(H, sum);
}

dev::Deal make_deal(int tiles128, int tiles, int workers) {
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

// Where the targets' share of dW, -g x of each row on its target's row, comes
// from: a product beside the probabilities in the columns pass, or the sum over
// rows sorted by target (csrc/embed.hip).  The first makes the workgroups with
// the most frequent targets late, the more the wider the rows; the second takes
// six launches (42 us at 60,001 rows, H = 256).  The whole call, first against
// second: H = 64, 12,001 x 20,011 259 / 272 us, 30,001 x 50,021 1,262 / 1,251; H =
// 128, 8,001 x 30,011 376 / 392, 16,001 x 30,011 701 / 707; H = 256, 3,001 x 10,007
// 143 / 159, 6,001 x 20,011 414 / 401, 16,001 x 50,021 2,267 / 2,102.
// The rule puts all of these on their faster side but 30,001 x 50,021 at H = 64 and
// 16,001 x 30,011 at H = 128, where both forms are within 1%.
// In float32 all parts of p - 1 are kept, without a product more.
bool targets_sorted(int es, int H, int R, int V) { return es == 2 && (double)R * V * H * H > 6.5e12; }

// How a call is cut, and where its shares lie in the workspace.
struct VocabPlan {
  bool few;
  int splits, per;     // few rows
  int row_tiles, Rp, col_tiles;
  dev::Deal rows, cols;
  size_t pm, pl, pb, po, wp, xg, lse, tgt, fac, pw, pdb, sort, bytes;
};
template <typename S>
VocabPlan vocab_plan(int H, int R, int V, bool grad) {
  constexpr int T = dev::voc_tile<S>();
  VocabPlan p{};
  p.few = !grad && R <= 32;
  size_t shares;
  if (p.few) {
    const int tiles = cdiv(V, 32);
    p.per = cdiv(tiles, 1024);
    p.splits = cdiv(cdiv(tiles, p.per), dev::kVocWaves) * dev::kVocWaves;
    shares = (size_t)p.splits * 32;
  } else {
    p.row_tiles = cdiv(R, dev::kVocRows);
    p.Rp = p.row_tiles * dev::kVocRows;
    p.rows = make_deal(p.row_tiles, cdiv(V, T), voc_workers<S>(H, grad));
    shares = (size_t)p.rows.all_slots() * dev::kVocRows;
  }
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at = up256(at + bytes);
    return here;
  };
  p.pm = take(shares * 4);
  p.pl = take(shares * 4);
  if (!grad) p.pb = take(shares * sizeof(dev::RowBest));
  if (sizeof(S) == 4 && !p.few) p.wp = take((size_t)V * H * 6);
  if (grad) {
    p.col_tiles = cdiv(V, dev::kVocRows);
    p.cols = make_deal(p.col_tiles, p.Rp / T, voc_workers<S>(H, true));
    const size_t cshares = p.cols.slots > 1 ? (size_t)p.cols.rest * p.cols.slots * dev::kVocRows : 0;
    p.po = take(shares * H * 4);
    p.xg = take((size_t)p.Rp * H * 2 * dev::voc_planes<S>());
    p.lse = take((size_t)p.Rp * 4);
    p.tgt = take((size_t)p.Rp * 4);
    p.fac = take((size_t)p.Rp * 4);
    p.pw = take(cshares * H * 4);
    p.pdb = take(cshares * 4);
    if (targets_sorted(sizeof(S), H, R, V)) p.sort = take(target_rows_workspace(H, p.Rp));
  }
  p.bytes = at;
  return p;
}

// The rows that the passes stage: W itself, or its planes.
template <typename S>
const dev::bf16s* staged_rows(const VocabArgs& c, int H, void* planes, hipStream_t st) {
  if constexpr (sizeof(S) == 2) {
    return static_cast<const dev::bf16s*>(c.W);
  } else {
    const size_t count = (size_t)c.V * H;
    hipLaunchKernelGGL(dev::vocab_planes_kernel<S>, dim3((unsigned)((count / 4 + dev::kVocThreads - 1) / dev::kVocThreads)),
                       dim3(dev::kVocThreads), 0, st, count, static_cast<const S*>(c.W),
                       static_cast<dev::bf16s*>(planes));
    return static_cast<const dev::bf16s*>(planes);
  }
}

template <typename S, int H, bool BEST>
hipError_t vocab_loss_h(const VocabArgs& c, hipStream_t st) {
  using namespace dev;
  const VocabPlan p = vocab_plan<S>(H, c.R, c.V, false);
  char* ws = static_cast<char*>(c.ws);
  float *pm = reinterpret_cast<float*>(ws + p.pm), *pl = reinterpret_cast<float*>(ws + p.pl);
  RowBest* pb = reinterpret_cast<RowBest*>(ws + p.pb);
  const S *X = static_cast<const S*>(c.X), *W = static_cast<const S*>(c.W);
  if (p.few) {
    hipLaunchKernelGGL((vocab_few_kernel<S, H, BEST>), dim3(p.splits / kVocWaves), dim3(kVocThreads), 0, st,
                       c.n_nodes, c.R, c.V, p.per, X, W, c.bias, c.node, pm, pl, pb);
    hipLaunchKernelGGL((vocab_few_join_kernel<S, H, BEST>), dim3(c.R), dim3(kVocThreads), 0, st, c.n_nodes, c.R, c.V,
                       p.splits, X, W, c.bias, c.node, c.target, pm, pl, pb, c.loss, c.lse, c.best);
    return hipGetLastError();
  }
  const bf16s* Ws = staged_rows<S>(c, H, ws + p.wp, st);
  if (c.bias != nullptr)
    hipLaunchKernelGGL((vocab_rows_kernel<S, H, false, BEST, true>), dim3(p.rows.workers), dim3(kVocThreads), 0, st,
                       c.n_nodes, c.R, c.V, p.rows, X, Ws, c.bias, c.node, pm, pl, nullptr, pb, nullptr, 0);
  else
    hipLaunchKernelGGL((vocab_rows_kernel<S, H, false, BEST, false>), dim3(p.rows.workers), dim3(kVocThreads), 0, st,
                       c.n_nodes, c.R, c.V, p.rows, X, Ws, nullptr, c.node, pm, pl, nullptr, pb, nullptr, 0);
  hipLaunchKernelGGL((vocab_join_kernel<S, H, false, BEST>), dim3(cdiv((long)c.R * (H / 4), kVocThreads)),
                     dim3(kVocThreads), 0, st, c.n_nodes, c.R, c.V, p.Rp, p.rows, X, W, c.bias, c.node, c.target,
                     nullptr, 1.f, pm, pl, nullptr, pb, c.loss, c.lse, c.best, nullptr, nullptr, nullptr, nullptr,
                     nullptr);
  return hipGetLastError();
}

template <typename S, int H>
hipError_t vocab_grad_h(const VocabArgs& c, hipStream_t st) {
  using namespace dev;
  const VocabPlan p = vocab_plan<S>(H, c.R, c.V, true);
  char* ws = static_cast<char*>(c.ws);
  float *pm = reinterpret_cast<float*>(ws + p.pm), *pl = reinterpret_cast<float*>(ws + p.pl);
  float *po = reinterpret_cast<float*>(ws + p.po), *lse_w = reinterpret_cast<float*>(ws + p.lse);
  float *fac_w = reinterpret_cast<float*>(ws + p.fac), *pw = reinterpret_cast<float*>(ws + p.pw);
  float* pdb = reinterpret_cast<float*>(ws + p.pdb);
  int32_t* tgt_w = reinterpret_cast<int32_t*>(ws + p.tgt);
  bf16s* xg = reinterpret_cast<bf16s*>(ws + p.xg);
  const bf16s* Ws = staged_rows<S>(c, H, ws + p.wp, st);
  const S *X = static_cast<const S*>(c.X), *W = static_cast<const S*>(c.W);
  // A small dX is cleared by the rows pass, one launch less (5 us of the 70 at
  // 3,001 rows); a large one, which would hold its products up, by its own.
  const long pieces = (long)c.n_nodes * (H / 4), each = (long)p.rows.workers * kVocThreads;
  const int clear = pieces <= 8 * each ? (int)((pieces + each - 1) / each) : 0;
  if (clear == 0) {
    const hipError_t err = launch_fill_zero(c.dX, (size_t)c.n_nodes * H, st);
    if (err != hipSuccess) return err;
  }
  if (c.bias != nullptr)
    hipLaunchKernelGGL((vocab_rows_kernel<S, H, true, false, true>), dim3(p.rows.workers), dim3(kVocThreads), 0, st,
                       c.n_nodes, c.R, c.V, p.rows, X, Ws, c.bias, c.node, pm, pl, po, nullptr, c.dX, clear);
  else
    hipLaunchKernelGGL((vocab_rows_kernel<S, H, true, false, false>), dim3(p.rows.workers), dim3(kVocThreads), 0, st,
                       c.n_nodes, c.R, c.V, p.rows, X, Ws, nullptr, c.node, pm, pl, po, nullptr, c.dX, clear);
  hipLaunchKernelGGL((vocab_join_kernel<S, H, true, false>), dim3(cdiv((long)p.Rp * (H / 4), kVocThreads)),
                     dim3(kVocThreads), 0, st, c.n_nodes, c.R, c.V, p.Rp, p.rows, X, W, c.bias, c.node, c.target,
                     c.weight, c.scale, pm, pl, po, nullptr, c.loss, c.lse, nullptr, c.dX, xg, lse_w, tgt_w, fac_w);
  const bool sorted = targets_sorted(sizeof(S), H, c.R, c.V);
#define COLS(WEIGHT, TARGETS)                                                                                       \
  hipLaunchKernelGGL((vocab_cols_kernel<S, H, WEIGHT, TARGETS>), dim3(p.cols.workers), dim3(kVocThreads), 0, st, c.V, \
                     p.Rp, p.cols, c.scale, xg, W, c.bias, lse_w, tgt_w, fac_w, c.dW, c.dbias, pw, pdb)
  if (c.weight != nullptr) {
    if (sorted) COLS(true, false); else COLS(true, true);
  } else {
    if (sorted) COLS(false, false); else COLS(false, true);
  }
#undef COLS
  const long left = (long)c.V - (long)p.cols.whole * kVocRows;
  if (left > 0 && p.cols.slots > 1)
    hipLaunchKernelGGL((vocab_wsum_kernel<H>), dim3(cdiv(left * (H / 4), kVocThreads)), dim3(kVocThreads), 0, st, c.V,
                       p.cols, pw, pdb, c.dW, c.dbias);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || !sorted) return err;
  return launch_target_rows(p.Rp, H, c.V, tgt_w, xg, -c.scale,
                            c.weight != nullptr ? fac_w : nullptr, c.dW, ws + p.sort, st);
}

template <typename S, int H>
hipError_t vocab_h(const VocabArgs& c, bool grad, hipStream_t st) {
  if (grad) return vocab_grad_h<S, H>(c, st);
  return c.best != nullptr ? vocab_loss_h<S, H, true>(c, st) : vocab_loss_h<S, H, false>(c, st);
}
}  // namespace

namespace GGNN_IMPL_NS {
size_t vocab_workspace(int H, int R, int V, bool grad) { return vocab_plan<dev::dt_t>(H, R, V, grad).bytes; }

hipError_t launch_vocab(int H, const VocabArgs& c, bool grad, hipStream_t st) {
  using S = dev::dt_t;
  switch (H) {
    case 32: return vocab_h<S, 32>(c, grad, st);
    case 64: return vocab_h<S, 64>(c, grad, st);
    case 128: return vocab_h<S, 128>(c, grad, st);
    case 256: return vocab_h<S, 256>(c, grad, st);
  }
  return hipErrorInvalidValue;
}
}  // namespace GGNN_IMPL_NS

}  // namespace ggnn
