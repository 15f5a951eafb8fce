// mlproj: the counter-based generator of dropout, whose mask is computed where it is needed and never stored.
#ifndef MLPROJ_DROPOUT_H
#define MLPROJ_DROPOUT_H

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/mlproj.h"

namespace mlproj {

// Entry (t, c) is kept if word c % 4 of Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011) at counter (c / 4, t, offset) and key seed is at least `threshold`.  So four neighbouring columns take one
// evaluation wherever they are computed: in a pass of its own, in a product's epilogue, or in the gradient.  An evaluation is
// 20 products of 32 x 32 bits and as many exclusive ors of three for four entries.  64M entries: beside HBM's time it is hidden in fp32 (92
// us with and without), and in bf16 where there is a residual (74 and 72); bf16 without one takes 65 us instead of 52.
struct Dropout {
  unsigned threshold;          // 0: every entry is kept
  float scale;                 // of those kept
  unsigned long long seed, offset;
  const unsigned long long* step;   // device: added to offset; or null
};

// (p was checked)
inline Dropout dropout_start(const mlproj_dropout* d) {
  Dropout r{};
  if (!d || d->p == 0.0) return r;
  const double t = std::nearbyint(d->p * 4294967296.0);
  r.threshold = t > 4294967295.0 ? 0xffffffffu : (unsigned)t;
  r.scale = (float)(1.0 / (1.0 - d->p));
  r.seed = d->seed; r.offset = d->offset; r.step = d->step;
  return r;
}
inline int dropout_check(const mlproj_dropout* d) {
  if (!d) return MLPROJ_OK;
  if (!(d->p >= 0.0 && d->p < 1.0)) return MLPROJ_ERR_BAD_VALUE;
  return reinterpret_cast<uintptr_t>(d->step) % 8 == 0 ? MLPROJ_OK : MLPROJ_ERR_ALIGNMENT;
}

// Where a kernel begins: the offset of this run of it.
__device__ __forceinline__ void dropout_at_step(Dropout& d) {
  if (d.threshold && d.step) d.offset += *d.step;
}

typedef unsigned philox_t __attribute__((ext_vector_type(4)));
// a ^ b ^ c in one instruction (0x96 is the truth table)
__device__ __forceinline__ unsigned philox_xor(unsigned a, unsigned b, unsigned c) { return (unsigned)__builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
__device__ __forceinline__ philox_t dropout_words(const Dropout& d, unsigned row, unsigned quad) {
  philox_t c = {quad, row, (unsigned)d.offset, (unsigned)(d.offset >> 32)};
  unsigned k0 = (unsigned)d.seed, k1 = (unsigned)(d.seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; i++) {
    const unsigned long long a = (unsigned long long)c[0] * 0xD2511F53u, b = (unsigned long long)c[2] * 0xCD9E8D57u;
    c = philox_t{philox_xor((unsigned)(b >> 32), c[1], k0), (unsigned)b, philox_xor((unsigned)(a >> 32), c[3], k1), (unsigned)a};
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}
// Four entries of row `row`, columns 4 quad .. 4 quad + 3.  What is dropped is zero whatever it was, NaN included.
template <typename V>
__device__ __forceinline__ V dropout4(const Dropout& d, long long row, long long quad, V v) {
  const philox_t w = dropout_words(d, (unsigned)row, (unsigned)quad);
#pragma unroll
  for (int i = 0; i < 4; i++) v[i] = w[i] >= d.threshold ? v[i] * d.scale : 0.0f;
  return v;
}
// Of a gradient, and what it is to be multiplied by: a slope at a NaN that was dropped is none.
template <typename V>
__device__ __forceinline__ V dropout4(const Dropout& d, long long row, long long quad, V v, V& slope) {
  const philox_t w = dropout_words(d, (unsigned)row, (unsigned)quad);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const bool kept = w[i] >= d.threshold;
    v[i] = kept ? v[i] * d.scale : 0.0f;
    slope[i] = kept ? slope[i] : 0.0f;
  }
  return v;
}

}  // namespace mlproj
#endif
