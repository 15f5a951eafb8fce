// mlproj: what the operators with 8-bit operands share: the format, rounding to it, checks of its arrays.
#ifndef MLPROJ_Q8_H
#define MLPROJ_Q8_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/mlproj.h"
#include "host.h"

namespace mlproj {

// Rows of e4m3 codes in whole blocks of 128, zeros past the row's end, and a byte per 32 of them: scale 2^(byte - 127), the
// form that the matrix cores take operands in.
constexpr int Q8_GROUP = 32, Q8_BLOCK = 128;
constexpr long long Q8_MAX_DIM = 1LL << 30;
__host__ __device__ inline long long q8_wide(long long n) { return (n + Q8_BLOCK - 1) / Q8_BLOCK * Q8_BLOCK; }

// A group's scale from the bits of its largest magnitude: the smallest power of two with which that is at most 448 = 1.75 *
// 2^8, so that nothing is clipped (rounding down the exponent would keep one more bit of groups whose largest entry has a
// fraction above 1.75, and lose that entry).  NaN and infinities compare largest as bits.
__device__ __forceinline__ unsigned q8_scale(unsigned top) {
  const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u);
  return e < 0 ? 0u : (unsigned)e;
}
constexpr unsigned Q8_NOT_FINITE = 0x7f800000u;
// 2^(127 - scale)
__device__ __forceinline__ float q8_inverse(unsigned scale) { return __builtin_bit_cast(float, (254u - scale) << 23); }
// Four entries times the inverse as codes, rounded to nearest-even (their magnitudes are at most 448).
__device__ __forceinline__ unsigned q8_codes4(float a, float b, float c, float d, float inverse) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, r, true);
}
__device__ __forceinline__ unsigned q8_magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }

// VEC neighbouring entries of a row as codes; the 32 / VEC lanes that hold a group are neighbours, and all of them are here.  A group
// with a NaN or an infinity has NaN codes throughout (and scale 1).  Returns the group's scale.
template <int VEC>
__device__ __forceinline__ unsigned q8_round(const float (&v)[VEC], unsigned (&codes)[VEC / 4]) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < VEC; i++) top = max(top, q8_magnitude(v[i]));
#pragma unroll
  for (int s = 1; s < Q8_GROUP / VEC; s <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, s));
  const bool finite = top < Q8_NOT_FINITE;
  const unsigned scale = finite ? q8_scale(top) : 127u;
  const float inverse = q8_inverse(scale);
#pragma unroll
  for (int q = 0; q < VEC / 4; q++)
    codes[q] = finite ? q8_codes4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], inverse) : 0x7f7f7f7fu;
  return scale;
}

// `needed`: it has entries to be read or written.
inline int q8_check(const mlproj_q8* q, long long rows, long long n, bool needed) {
  if (!q) return MLPROJ_ERR_NULL_POINTER;
  if (q->rows != rows || q->n != n) return MLPROJ_ERR_BAD_DIMENSION;
  if (!q->codes || !q->scales) return needed ? MLPROJ_ERR_NULL_POINTER : MLPROJ_OK;
  if (q->ld < q8_wide(n) || q->lds < q8_wide(n) / Q8_GROUP) return MLPROJ_ERR_BAD_DIMENSION;
  if (q->ld > Q8_MAX_DIM || q->lds > Q8_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  return aligned(q->codes, 16) && q->ld % 16 == 0 && aligned(q->scales, 4) && q->lds % 4 == 0 ? MLPROJ_OK : MLPROJ_ERR_ALIGNMENT;
}

}  // namespace mlproj
#endif
