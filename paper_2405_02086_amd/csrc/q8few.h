// mlproj: products of few 8-bit tokens with 8-bit weights: weights go from memory straight into the matrix cores' operands.
#ifndef MLPROJ_Q8FEW_H
#define MLPROJ_Q8FEW_H

#include "q8tile.h"

namespace mlproj {
namespace {

// ------------------------------------------------------------------ few tokens
// A workgroup has 16 columns (DUAL: of both products) and up to 16 MT tokens; its wavefronts share out K, U blocks of 128 at a
// time, and add their sums in LDS in their order.  Loads bring operands as the matrix cores take them: a lane 16 codes of
// each of two groups and the scale of one, so that four neighbouring lanes read 64 neighbouring bytes of a row.  Rows past
// the end are the last one again, and not stored.  Bound by HBM: every weight is read once.
constexpr int Q8F_COLS = 16;

template <typename T, bool DUAL, int EPI, int MT, int U, int WAVES, bool EXACT>
__global__ __launch_bounds__(WAVES * 64) void q8_few_kernel(Q8Product q) {
  constexpr int MATS = DUAL ? 2 : 1, VALUES = MATS * MT;
  __shared__ f32x4 sums[WAVES][VALUES][64];
  FfProduct& p = q.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const long long col0 = (long long)blockIdx.x * Q8F_COLS;
  const int blocks = (int)(p.K / Q8_BLOCK);
  const long long col = col0 + r < p.N ? col0 + r : p.N - 1;
  const unsigned char *w[MATS], *sw[MATS], *x[MT], *sx[MT];
#pragma unroll
  for (int i = 0; i < MATS; i++) {
    w[i] = static_cast<const unsigned char*>(i ? p.B1 : p.B0) + col * p.ldb + 16 * g;
    sw[i] = (i ? q.sB1 : q.sB0) + col * q.ldsb;
  }
#pragma unroll
  for (int t = 0; t < MT; t++) {
    const long long row = t * 16 + r < p.M ? t * 16 + r : p.M - 1;
    x[t] = static_cast<const unsigned char*>(p.A0) + row * p.lda + 16 * g;
    sx[t] = q.sA + row * q.ldsa;
  }
  struct Operand { i32x8 codes; unsigned scale; };
  auto fetch = [&](const unsigned char* codes, const unsigned char* scales, int block) {
    Operand o;
    u32x4 v[2];
    __builtin_memcpy(&v[0], __builtin_assume_aligned(codes + (long long)block * Q8_BLOCK, 16), 16);
    __builtin_memcpy(&v[1], __builtin_assume_aligned(codes + (long long)block * Q8_BLOCK + 64, 16), 16);
    __builtin_memcpy(&o.codes, v, 32);
    o.scale = *reinterpret_cast<const unsigned*>(scales + (long long)block * 4);
    return o;
  };
  f32x4 acc[VALUES] = {};
  auto multiply = [&](const Operand& a, const Operand& b, f32x4 c) {
    if constexpr (EXACT) {
#pragma unroll
      for (int k = 0; k < 4; k++) {
        // a lane's codes are of groups g / 2 and 2 + g / 2
        const int at = 8 * ((g >> 1) + (k >> 1) * 2);
        c = ff_mfma(q8_widen(a.codes[2 * k], a.codes[2 * k + 1], (a.scale >> at) & 255u), q8_widen(b.codes[2 * k], b.codes[2 * k + 1], (b.scale >> at) & 255u), c);
      }
      return c;
    } else {
      return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.codes, b.codes, c, 0, 0, 0, (int)(a.scale >> (8 * g)), 0, (int)(b.scale >> (8 * g)));
    }
  };
  // whole rounds of U blocks, the next round's weights on their way while the present one's are multiplied; then what is left
  int block = wave * U;
  for (; block + U <= blocks; block += WAVES * U) {
    Operand ow[U][MATS], ox[U][MT];
#pragma unroll
    for (int u = 0; u < U; u++) {
#pragma unroll
      for (int i = 0; i < MATS; i++) ow[u][i] = fetch(w[i], sw[i], block + u);
#pragma unroll
      for (int t = 0; t < MT; t++) ox[u][t] = fetch(x[t], sx[t], block + u);
    }
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int i = 0; i < MATS; i++)
#pragma unroll
        for (int t = 0; t < MT; t++) acc[i * MT + t] = multiply(ow[u][i], ox[u][t], acc[i * MT + t]);
  }
  for (; block < blocks; block++) {
#pragma unroll
    for (int i = 0; i < MATS; i++) {
      const Operand ow = fetch(w[i], sw[i], block);
#pragma unroll
      for (int t = 0; t < MT; t++) acc[i * MT + t] = multiply(ow, fetch(x[t], sx[t], block), acc[i * MT + t]);
    }
  }
#pragma unroll
  for (int v = 0; v < VALUES; v++) sums[wave][v][lane] = acc[v];
  __syncthreads();
  // a lane's four sums are neighbouring columns of one token
  dropout_at_step(p.drop);
  for (int at = threadIdx.x; at < MT * 64; at += WAVES * 64) {
    const int t = at >> 6, l = at & 63;
    const long long row = t * 16 + (l & 15), c = col0 + (l >> 4) * 4;
    if (row >= p.M || c >= p.N) continue;
    f32x4 v[2] = {};
#pragma unroll
    for (int i = 0; i < MATS; i++)
      for (int s = 0; s < WAVES; s++) v[i] += sums[s][i * MT + t][l];
    FfVec4<T> d = {};
    f32x4 bias = {};
    if constexpr (EPI == FF_LINEAR) {
      d = ff_upstream<T>(p, row, c, p.N);
      bias = ff_bias<T>(p, c, p.N);
    }
    ff_finish<EPI, DUAL, T>(p, row, c, p.N, v[0], v[1], d, bias);
  }
}

}  // namespace
}  // namespace mlproj
#endif
