// mlproj: products of few 8-bit tokens with 8-bit weights: weights go from memory straight into the matrix cores' operands.
#ifndef MLPROJ_Q8FEW_H
#define MLPROJ_Q8FEW_H

#include "q8tile.h"

namespace mlproj {
namespace {

// ------------------------------------------------------------------ few tokens
// A workgroup has 16 CB columns (DUAL: of both products) and up to 16 tokens; its wavefronts share out K, U blocks of 128 at a
// time, and add their sums in LDS in their order.  Loads bring operands as the matrix cores take them: a lane 16 codes of
// each of two groups and the scale of one, so that four neighbouring lanes read 64 neighbouring bytes of a row.  Rows past
// the end are the last one again, and not stored.  Bound by HBM and by how many loads are under way: every weight is read once, and a
// wavefront waits once a round.  us, U = 2 / 4 / 8 with eight wavefronts, weights that were not read just before: one token 4096 -> 2 x
// 16384 31 / 26 / 40 (32 blocks of 128 are half a round), 16384 -> 4096 17 / 19 / 14, 8 tokens 8192 -> 8192 17 / 16 / 16, one token 4096
// -> 4096 6.2 / 5.6 / 5.4; four or sixteen wavefronts are no faster.
//
// Pairs of products with 16-bit results in 32 columns (CB = 2) read the tokens half as often and have half as many workgroups, two on
// a compute unit where three of 16 columns are.  16 against 32 columns, us, m columns in each product, weights as above:
//   m <= 4096: half the compute units would be idle (16 tokens 4096 -> 2 x 4096 9.7 / 14.2), and as at m = 10240 (24.0 / 27.0) and 12288
//     (25.9 / 27.7) whenever the last 4096 columns are the first half of 8192;
//   m > 12288: a second turn of 16 columns.  5 tokens 1024 -> 2 x 12288 8.0 / 8.9, 2 x 12544 10.9 / 8.9, 2 x 16384 12.0 / 9.2; where n is
//     longer HBM covers it for few tokens (2048 -> 2 x 16384 3 tokens 16.9 / 14.6; 4096 -> 2 x 16384 3, 8 and 16 tokens 27.2 / 29.1, 29.0 /
//     29.3, 33.2 / 30.9);
//   4096 < m <= 8192: the tokens' share of the reads decides.  16 tokens 1024, 2048, 4096 -> 2 x 6144 7.2 / 7.6, 9.1 / 9.3, 17.1 / 15.0,
//     5 tokens 4096 -> 2 x 5120 14.0 / 13.5; 16 tokens 4096 and 8192 -> 2 x 8192 18.2 / 16.2 and 32.7 / 39.1.
// Over 320 shapes the rule (q8_few_wide) takes 0.4 % more than the better of both, 15 % at most.  With fp32 results 32 columns lose
// throughout (16 tokens 4096 -> 2 x 8192 18.7 / 20.4, 1024 -> 2 x 16384 12.2 / 21.7), and so does one product (16384 -> 4096 19 / 26).
constexpr int Q8F_COLS = 16;

template <typename T, bool DUAL, int EPI, int CB, int U, int WAVES, bool EXACT>
__global__ __launch_bounds__(WAVES * 64) void q8_few_kernel(Q8Product q) {
  constexpr int MATS = DUAL ? 2 : 1, VALUES = MATS * CB;
  __shared__ f32x4 sums[WAVES][VALUES][64];
  FfProduct& p = q.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const long long col0 = (long long)blockIdx.x * (Q8F_COLS * CB);
  const int blocks = (int)(p.K / Q8_BLOCK);
  const unsigned char *w[VALUES], *sw[VALUES];
#pragma unroll
  for (int i = 0; i < VALUES; i++) {
    const long long at = col0 + i % CB * 16 + r, col = at < p.N ? at : p.N - 1;
    w[i] = static_cast<const unsigned char*>(i >= CB ? p.B1 : p.B0) + col * p.ldb + 16 * g;
    sw[i] = (i >= CB ? q.sB1 : q.sB0) + col * q.ldsb;
  }
  const long long row = r < p.M ? r : p.M - 1;
  const unsigned char *x = static_cast<const unsigned char*>(p.A0) + row * p.lda + 16 * g, *sx = q.sA + row * q.ldsa;
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
  int block = wave * U;
  for (; block + U <= blocks; block += WAVES * U) {
    Operand ow[U][VALUES], ox[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
#pragma unroll
      for (int i = 0; i < VALUES; i++) ow[u][i] = fetch(w[i], sw[i], block + u);
      ox[u] = fetch(x, sx, block + u);
    }
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int i = 0; i < VALUES; i++) acc[i] = multiply(ow[u][i], ox[u], acc[i]);
  }
  if (block < blocks) {
    // a round that is not whole: its last block again in the place of those that are not there, and not multiplied
    Operand ow[U][VALUES], ox[U];
#pragma unroll
    for (int u = 0; u < U - 1; u++) {
      const int at = block + u < blocks ? block + u : blocks - 1;
#pragma unroll
      for (int i = 0; i < VALUES; i++) ow[u][i] = fetch(w[i], sw[i], at);
      ox[u] = fetch(x, sx, at);
    }
#pragma unroll
    for (int u = 0; u < U - 1; u++)
      if (block + u < blocks)
#pragma unroll
        for (int i = 0; i < VALUES; i++) acc[i] = multiply(ow[u][i], ox[u], acc[i]);
  }
#pragma unroll
  for (int v = 0; v < VALUES; v++) sums[wave][v][lane] = acc[v];
  __syncthreads();
  // a lane's four sums are neighbouring columns of one token
  for (int at = threadIdx.x; at < CB * 64; at += WAVES * 64) {
    const int b = at >> 6, l = at & 63;
    const long long t = l & 15, c = col0 + b * 16 + (l >> 4) * 4;
    if (t >= p.M || c >= p.N) continue;
    f32x4 v[2] = {};
#pragma unroll
    for (int i = 0; i < MATS; i++)
      for (int s = 0; s < WAVES; s++) v[i] += sums[s][i * CB + b][l];
    FfVec4<T> d = {};
    f32x4 bias = {};
    if constexpr (EPI == FF_PLAIN) {
      d = ff_upstream<T>(p, t, c, p.N);
      bias = ff_bias<T>(p, c, p.N);
    }
    ff_finish<EPI, DUAL, T>(p, t, c, p.N, v[0], v[1], d, bias);
  }
}

}  // namespace
}  // namespace mlproj
#endif
