// Dropout from a counter-based generator: the mask is a function of the
// element's number, so it is recomputed where it is needed and never stored.
//
// Generator: Philox4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw, "Parallel
// random numbers: as easy as 1, 2, 3", SC 2011; 7 rounds is the least count
// that passes the paper's statistical tests).  The block at counter
// (e / 8, offset) under the key `seed` gives eight 16-bit words; element e
// takes word e % 8 and stays where the word is at least p * 2^16 (rounded), so
// one block serves a lane's eight consecutive elements.  16 bits per element:
// the generator's products bound a pass over bfloat16 states, and p is met to
// 2^-17; the scale of the kept elements is exact for the rounded p.
#pragma once

#include "device_common.h"
#include "kernels.h"

namespace ggnn {
namespace dev {

__device__ __forceinline__ u32x4 philox7(uint64_t block, const Dropout& d) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = d.offset_lo, c3 = d.offset_hi;
  uint32_t k0 = d.seed_lo, k1 = d.seed_hi;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

// Eight elements numbered 8 block .. 8 block + 7: dropped ones become 0
// whatever they held (infinities and NaN too), kept ones are scaled.
__device__ __forceinline__ void drop8(float (&v)[8], uint64_t block, const Dropout& d) {
  const u32x4 w = philox7(block, d);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = (w[i] & 0xFFFFu) >= d.cut ? v[2 * i] * d.scale : 0.f;
    v[2 * i + 1] = (w[i] >> 16) >= d.cut ? v[2 * i + 1] * d.scale : 0.f;
  }
}

// Eight consecutive elements as floats, and back (16-byte aligned).
template <typename S>
__device__ __forceinline__ void load8f(const S* p, float (&v)[8]) {
  const f32x4 a = load4f(p), b = load4f(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
template <>
__device__ __forceinline__ void load8f<bf16s>(const bf16s* p, float (&v)[8]) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = lo_f(w[i]);
    v[2 * i + 1] = hi_f(w[i]);
  }
}
__device__ __forceinline__ void store8f(bf16s* p, const float (&v)[8]) {
  *reinterpret_cast<u32x4*>(p) = u32x4{pk2(v[0], v[1]), pk2(v[2], v[3]), pk2(v[4], v[5]), pk2(v[6], v[7])};
}
__device__ __forceinline__ void store8f(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

// The same for results that this kernel does not read again: past the caches
// that hold what it does.
__device__ __forceinline__ void store8f_once(bf16s* p, const float (&v)[8]) {
  __builtin_nontemporal_store(u32x4{pk2(v[0], v[1]), pk2(v[2], v[3]), pk2(v[4], v[5]), pk2(v[6], v[7])},
                              reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ void store8f_once(float* p, const float (&v)[8]) {
  __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4*>(p));
  __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4*>(p + 4));
}

}  // namespace dev
}  // namespace ggnn
