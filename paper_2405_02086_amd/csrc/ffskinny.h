// mlproj: fp32 products of few tokens: weights go from memory straight into the matrix cores' operands.
#ifndef MLPROJ_FFSKINNY_H
#define MLPROJ_FFSKINNY_H

#include "ffcommon.h"

namespace mlproj {
namespace {      // (each translation unit that includes this has its own kernels)

// ------------------------------------------------------------------ few tokens in fp32
// G = X Wg and U = X Wu (one product alone: X W) for a few tokens, 16 of them per workgroup: every weight is used for a handful of tokens, so the
// kernel has to keep loads in flight and nothing else.  A wavefront takes 64 columns and 32 rows at a time, a lane
// four columns of eight rows, and feeds them to the fp32 matrix instructions, whose operands are single elements: no
// cutting into bf16 parts, no LDS, no barrier until the wavefronts, which share out the rows, add their sums in a
// tree (in a fixed order).  Loads take any address.  Workgroups of the same columns and other tokens run on one
// XCD next to one another and share the weights in its L2.
// us, staged tiles / this: 16 x 4096 -> 16384 216 / 108 (5 TB/s), 16 x 256 -> 128 24 / 7; at 64 tokens the tiles win, 192
// against 315.  (16-bit pieces turned into operands by byte permutes were no faster than the tiles: one token through
// 4097 x 16383 bf16 110 against 112.)
constexpr int FK_WAVES = 8, FK_COLS = 64;

__device__ __forceinline__ f32x4 fk_mfma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Four neighbouring entries of which the first `valid` exist, the others zeros.
__device__ __forceinline__ f32x4 fk_load(const float* p, long long valid) {
  if (valid >= 4) return ff_load4(p);
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; i++) r[i] = i < valid ? p[i] : 0.0f;
  return r;
}

template <int EPI, bool DUAL>
__global__ __launch_bounds__(FK_WAVES * 64) void ff_skinny_kernel(FfProduct p) {
  constexpr int CW = 4, PRODUCTS = DUAL ? 2 : 1, VALUES = PRODUCTS * CW * 4;
  __shared__ float sums[FK_WAVES / 2][VALUES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  const long long N = p.kept ? *p.kept : p.N;
  const long long tiles_n = (N + FK_COLS - 1) / FK_COLS, tiles_m = (p.M + 15) / 16;
  // workgroup 8 i + x runs on XCD x: columns x, x + 8, ... there, each with all its tokens in turn
  const long long mine = blockIdx.x >> 3, tn = mine / tiles_m * 8 + (blockIdx.x & 7), row0 = mine % tiles_m * 16;
  if (tn >= tiles_n) return;
  p.share = blockIdx.y;
  const long long col0 = tn * FK_COLS, col = col0 + c * CW;
  const float* X = static_cast<const float*>(p.A0);
  const float* B[2] = {static_cast<const float*>(p.B0), static_cast<const float*>(p.B1)};
  const int steps = (int)((p.K + 31) / 32);
  const int first = (int)((long long)steps * blockIdx.y / p.splits), last = (int)((long long)steps * (blockIdx.y + 1) / p.splits);
  f32x4 acc[PRODUCTS][CW] = {};
  for (int step = first + wave; step < last; step += FK_WAVES) {
    const long long k0 = (long long)step * 32 + 8 * g;
    f32x4 w[PRODUCTS][8];
#pragma unroll
    for (int i = 0; i < PRODUCTS; i++)
#pragma unroll
      for (int s = 0; s < 8; s++) w[i][s] = fk_load(B[i] + (k0 + s) * p.ldb + col, k0 + s < p.K ? N - col : 0);
    const FfVec8<float> x = ff_load8(X + (row0 + c) * p.lda + k0, row0 + c < p.M ? p.K - k0 : 0);
#pragma unroll
    for (int i = 0; i < PRODUCTS; i++)
#pragma unroll
      for (int s = 0; s < 8; s++)
#pragma unroll
        for (int j = 0; j < CW; j++) acc[i][j] = fk_mfma(x.v[s], w[i][s][j], acc[i][j]);
  }
  // the tree: the upper half of the wavefronts hands its sums to the lower one
  auto value = [&](int v) -> float& { return reinterpret_cast<float*>(acc)[v]; };
#pragma unroll
  for (int half = FK_WAVES / 2; half >= 1; half /= 2) {
    if (wave >= half && wave < 2 * half)
#pragma unroll
      for (int v = 0; v < VALUES; v++) sums[wave - half][v][lane] = value(v);
    __syncthreads();
    if (wave < half)
#pragma unroll
      for (int v = 0; v < VALUES; v++) value(v) += sums[wave][v][lane];
    __syncthreads();
  }
  if (wave == 0)
#pragma unroll
    for (int v = 0; v < VALUES; v++) sums[0][v][lane] = value(v);
  __syncthreads();
  if constexpr (EPI == FF_LINEAR) dropout_at_step(p.drop);
  // four neighbouring columns of a token per thread
  const int rows = p.M - row0 < 16 ? (int)(p.M - row0) : 16;
  for (int e = threadIdx.x; e < rows * (FK_COLS / 4); e += FK_WAVES * 64) {
    const int t = e / (FK_COLS / 4), in = e % (FK_COLS / 4) * 4;
    const long long at = col0 + in;
    if (at >= N) continue;
    f32x4 v[2] = {};
#pragma unroll
    for (int i = 0; i < PRODUCTS; i++)
#pragma unroll
      for (int q = 0; q < 4; q++) v[i][q] = sums[0][(i * CW + (in + q) % CW) * 4 + t % 4][t / 4 * 16 + (in + q) / CW];
    FfVec4<float> d = {};
    f32x4 bias = {};
    if constexpr (FF_UPSTREAM<EPI>) d = ff_upstream<float>(p, row0 + t, at, N);
    if constexpr (EPI == FF_LINEAR) bias = ff_bias<float>(p, at, N);
    ff_finish<EPI, DUAL, float>(p, row0 + t, at, N, v[0], v[1], d, bias);
  }
}

}  // namespace
}  // namespace mlproj
#endif
