// mlproj: what the kernels of the gated feed-forward block share: the arguments of one product, element
// access, the activation and the epilogues.
#ifndef MLPROJ_FFCOMMON_H
#define MLPROJ_FFCOMMON_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "../../include/mlproj.h"
#include "dropout.h"

namespace mlproj {

using bf16_t = __bf16;
using f16_t = _Float16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));

// What a product leaves behind.
//   STORE    C0 (and C1, where the tile holds two products side by side)
//   FWD      C0 = keep * act(G) * U; G and U too where the caller wants them
//   GRAD     C0 = keep * act'(G) * U * dH, C1 = keep * act(G) * dH, rounded to the storage type: they are operands of the matrix
//            cores in the products that follow.  With 16 bits that is a second rounding behind the one of the results, and errors of
//            dX, dWg and dWu grow by the root of two (bf16 1.7e-3 -> 2.4e-3 of a result's norm, fp16 2.1e-4 -> 2.9e-4); without it
//            these products would be in fp32, six times their operations
//   LINEAR   Z = v + bias, C0 = residual + D(act(Z)) with D the dropout; Z too where the caller wants it
//   PLAIN    C0 = residual + act(v + bias): LINEAR where there is neither dropout nor Z (8 bits)
//   SCALED   C0 = scale * v: the gradients of LINEAR, whose operand dY is exact in 16 bits and dY / (1 - p) is not
//   PARTIAL  the sums over this workgroup's share of K, in fp32, for the join kernel
enum : int { FF_WHOLE = 0, FF_TURNS = 1, FF_REST = 2 };
enum : int { FF_STORE = 0, FF_FWD = 1, FF_GRAD = 2, FF_PARTIAL = 3, FF_LINEAR = 4, FF_SCALED = 5, FF_PLAIN = 6 };

// One product C = A B (M x N, summed over K), or two that share A: C0 = A B0, C1 = A B1.
// A: `a_kc` its rows run along K (row-major M x K); otherwise its rows are the K index (K x M).
// B: `b_kc` row-major N x K; otherwise K x N.
// With segs = 2 the sum runs over two pairs of operands: C = A0 B0 + A1 B1.
struct FfProduct {
  const void *A0, *A1, *B0, *B1;
  long long lda, ldb;          // elements between rows
  long long M, N, K;           // N: columns of each of the two products
  int segs;
  bool a_filled, b_filled;     // the workspace's: rows may be read up to their whole 16-byte pieces, past K they hold zeros
  int act;
  void *C0, *C1;
  long long ldc;
  void *G, *U;                 // FWD: optional outputs; LINEAR: Z in G
  const void* dH;              // GRAD; LINEAR, PLAIN: the residual, or null
  const void* bias;            // LINEAR, PLAIN, or null
  Dropout drop;                // LINEAR
  float scale;                 // SCALED
  long long ldg, ldh;
  const unsigned char* keep;   // one byte per column of the result, or null
  const int* kept;             // packed channels, on the device: how many there are, instead of N (dX: of K); or null
  float* partial;              // PARTIAL: [splits][products][M][N in whole quads]
  int splits;                  // shares of the sum, and the one a workgroup has (set in the kernels)
  int share;
  int part;                    // direct tiles: FF_WHOLE, or a product shared between two launches (ffdirect.h)
};

// ------------------------------------------------------------------ elements
template <typename T> __device__ __forceinline__ T ff_round(float x) { return (T)x; }

template <typename T> struct alignas(sizeof(T)) FfVec4 { T v[4]; };
template <typename T> struct alignas(sizeof(T)) FfVec8 { T v[8]; };

// Four neighbouring elements at any element-aligned address; the compiler makes one wide access of it.
template <typename T>
__device__ __forceinline__ f32x4 ff_load4(const T* p) {
  FfVec4<T> t;
  __builtin_memcpy(&t, p, sizeof(t));
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; i++) r[i] = (float)t.v[i];
  return r;
}
template <typename T>
__device__ __forceinline__ void ff_store4(T* p, f32x4 x) {
  FfVec4<T> t;
#pragma unroll
  for (int i = 0; i < 4; i++) t.v[i] = ff_round<T>(x[i]);
  __builtin_memcpy(p, &t, sizeof(t));
}

// Eight neighbouring elements of which the first `valid` exist, the others zeros.
template <typename T>
__device__ __forceinline__ FfVec8<T> ff_load8(const T* p, long long valid) {
  FfVec8<T> r;
  if (valid >= 8) {
    __builtin_memcpy(&r, p, sizeof(r));
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) r.v[i] = i < valid ? p[i] : (T)0.0f;
  }
  return r;
}

// ------------------------------------------------------------------ tiles
// The tile of a workgroup.  Workgroups are dealt to the 8 XCDs in turn; each XCD takes a run of consecutive tiles, and
// tiles are numbered down FF_BAND tile rows before the next column, so that what runs on an XCD at one time shares rows of A
// and columns of B in its L2.  Shares of a sum go to different XCDs (with fewer than 8 shares, several XCDs divide a
// share's tiles), so that each of them reads a part of K only.
//
// A product of 3.25 turns of 256 x 256 tiles on 256 compute units takes as long as one of 4.  It can go out in two launches:
// FF_TURNS takes the whole turns, FF_REST the remaining tiles cut into four of 128 x 128, which a quarter of the units
// would have taken whole.  More than FF_LEFT remaining tiles would be more than one turn of small ones: then they stay
// whole.  (The number of tiles may be known on the device only, where channels are packed.)
constexpr int FF_BAND = 4, FF_TURN = 256, FF_LEFT = 128;
__host__ __device__ inline long long ff_in_turns(long long tiles) {
  const long long rest = tiles % FF_TURN;
  return rest > FF_LEFT ? tiles : tiles - rest;
}
__device__ __forceinline__ void ff_place(long long v, long long tiles_m, long long tiles_n, long long* tm, long long* tn) {
  const long long band = v / (FF_BAND * tiles_n), in = v % (FF_BAND * tiles_n);
  const long long rows = tiles_m - band * FF_BAND < FF_BAND ? tiles_m - band * FF_BAND : FF_BAND;
  *tm = band * FF_BAND + in % rows;
  *tn = in / rows;
}
// First row and column of the workgroup's tile of BM x COLS, and its share of the sum (p.share); false: there is none.
template <int BM, int COLS>
__device__ __forceinline__ bool ff_tile(FfProduct& p, long long N, long long* row0, long long* col0) {
  long long tm, tn;
  p.share = 0;
  if (p.part == FF_REST) {        // a quarter of a tile of twice the size
    const long long tiles_m = (p.M + 2 * BM - 1) / (2 * BM), tiles_n = (N + 2 * COLS - 1) / (2 * COLS);
    const long long v = ff_in_turns(tiles_m * tiles_n) + (blockIdx.x >> 2);
    if (v >= tiles_m * tiles_n) return false;
    ff_place(v, tiles_m, tiles_n, &tm, &tn);
    *row0 = (2 * tm + (blockIdx.x >> 1 & 1)) * BM;
    *col0 = (2 * tn + (blockIdx.x & 1)) * COLS;
    return *row0 < p.M && *col0 < N;
  }
  const long long tiles_m = (p.M + BM - 1) / BM, tiles_n = (N + COLS - 1) / COLS;
  const long long all = p.part == FF_TURNS ? ff_in_turns(tiles_m * tiles_n) : tiles_m * tiles_n;
  p.share = blockIdx.x % p.splits;
  const long long id = blockIdx.x / p.splits;
  if (id >= all) return false;
  const long long xcds = p.splits < 8 ? 8 / p.splits : 1;         // that divide the share's tiles (splits: a power of two)
  const long long xcd = id % xcds, each = all / xcds, more = all % xcds;
  ff_place(xcd * each + (xcd < more ? xcd : more) + id / xcds, tiles_m, tiles_n, &tm, &tn);
  *row0 = tm * BM;
  *col0 = tn * COLS;
  return true;
}

// ------------------------------------------------------------------ activation
// act(g) and its slope in fp32.  silu: g s with s = 1/(1 + e^-g), slope s (1 + g (1 - s)).  gelu: g Phi(g),
// slope Phi(g) + g phi(g).  relu: max(g, 0), slope 1 where g > 0 (NaN stays NaN in the product).
//
// EXACT (fp32 storage) takes the library's functions.  Results that are rounded to 16 bits take the hardware's exponential and
// reciprocal (an ulp of fp32 each) and, for Phi, Abramowitz and Stegun 7.1.26: in the epilogue of a 256 x 256 tile the
// library's forms cost a tenth of the whole tile's time.  Phi is taken from the side on which it is small, Phi(-|g|) = erfc(|g| /
// sqrt 2) / 2: 1 + erf would cancel there.  Largest relative error of the 16-bit form: 5e-5 above -3, 0.1 % above -4.5, 0.4 % above -6
// (1 + erf: 5 % above -5, nothing right below).
// Slopes are 0 and 1 from |g| = 128 on, and are taken there past it, as a gradient's act(g) is below -128: a g that is infinite, which
// finite sums are once they are stored in fp16, would give infinity times zero.
template <bool EXACT> __device__ __forceinline__ float ff_exp(float x) {
  return EXACT ? expf(x) : __builtin_amdgcn_exp2f(x * 1.44269504f);
}
template <bool EXACT> __device__ __forceinline__ float ff_reciprocal(float x) {
  return EXACT ? 1.0f / x : __builtin_amdgcn_rcpf(x);
}
// Phi(g) given e = exp(-g^2 / 2); the polynomial has half the coefficients of 7.1.26, which is a form of erfc
template <bool EXACT> __device__ __forceinline__ float ff_normal(float g, float e) {
  const float x = fabsf(g) * 0.70710678f;
  float below;                                   // Phi(-|g|)
  if constexpr (EXACT) {
    below = 0.5f * erfcf(x);
  } else {
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
    below = ((((0.530702715f * t - 0.726576014f) * t + 0.710706871f) * t - 0.142248368f) * t + 0.127414796f) * t * e;
  }
  return g < 0.0f ? below : 1.0f - below;
}
__device__ __forceinline__ float ff_near(float g) { return __builtin_amdgcn_fmed3f(g, -128.0f, 128.0f); }   // (a NaN is in s or e as well)
template <bool LIMITS> __device__ __forceinline__ float ff_above(float g) { return LIMITS ? __builtin_amdgcn_fmed3f(g, -128.0f, __builtin_inff()) : g; }
template <bool EXACT, bool LIMITS = false> __device__ __forceinline__ void ff_gate4(int act, f32x4 g, f32x4& value, f32x4& slope) {
  if (act == MLPROJ_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float s = ff_reciprocal<EXACT>(1.0f + ff_exp<EXACT>(-g[i]));
      value[i] = ff_above<LIMITS>(g[i]) * s;
      slope[i] = s * (1.0f + ff_near(g[i]) * (1.0f - s));
    }
  } else if (act == MLPROJ_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float e = ff_exp<EXACT>(-0.5f * g[i] * g[i]);
      const float phi = ff_normal<EXACT>(g[i], e);
      value[i] = ff_above<LIMITS>(g[i]) * phi;
      slope[i] = phi + ff_near(g[i]) * 0.39894228f * e;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      value[i] = g[i] > 0.0f ? g[i] : (g[i] == g[i] ? 0.0f : g[i]);
      slope[i] = g[i] > 0.0f ? 1.0f : (g[i] == g[i] ? 0.0f : g[i]);
    }
  }
}

// With no activation as well; the value alone.
template <bool EXACT> __device__ __forceinline__ f32x4 ff_value4(int act, f32x4 z) {
  if (act == MLPROJ_ACT_NONE) return z;
  f32x4 value, slope;
  ff_gate4<EXACT>(act, z, value, slope);
  return value;
}

// ------------------------------------------------------------------ epilogue
// Columns col .. col+3 of row `row`, of which those below N exist; v0, v1: their sums in the two products.
// A pruned channel's outputs are zeros whatever its sums are, NaN included.
// ff_upstream: GRAD's four entries of dH, LINEAR's and PLAIN's of the residual; all of a thread's are fetched before its first store,
// which the compiler could not move them across.  ff_bias: LINEAR's and PLAIN's of the bias.
template <typename T>
__device__ __forceinline__ FfVec4<T> ff_upstream(const FfProduct& p, long long row, long long col, long long N) {
  FfVec4<T> d;
  const T* at = static_cast<const T*>(p.dH) + row * p.ldh + col;
  if (!p.dH) {
#pragma unroll
    for (int i = 0; i < 4; i++) d.v[i] = (T)0.0f;
  } else if (col + 4 <= N) {
    __builtin_memcpy(&d, at, sizeof(d));
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) d.v[i] = col + i < N ? at[i] : (T)0.0f;
  }
  return d;
}
template <int EPI> constexpr bool FF_BIAS = EPI == FF_LINEAR || EPI == FF_PLAIN;
template <int EPI> constexpr bool FF_UPSTREAM = EPI == FF_GRAD || FF_BIAS<EPI>;
template <typename T>
__device__ __forceinline__ f32x4 ff_bias(const FfProduct& p, long long col, long long N) {
  f32x4 b = {};
  if (!p.bias) return b;
  const T* at = static_cast<const T*>(p.bias) + col;
  if (col + 4 <= N) return ff_load4(at);
#pragma unroll
  for (int i = 0; i < 4; i++) b[i] = col + i < N ? (float)at[i] : 0.0f;
  return b;
}
template <int EPI, bool DUAL, typename T>
__device__ __forceinline__ void ff_finish(const FfProduct& p, long long row, long long col, long long N, f32x4 v0, f32x4 v1, FfVec4<T> d,
                                          f32x4 bias = {}) {
  const bool whole = col + 4 <= N;
  const int count = whole ? 4 : (int)(N - col);
  if constexpr (EPI == FF_PARTIAL) {
    // (rows of whole quads: what lies past N is written and never read)
    const long long ld = (p.N + 3) / 4 * 4, plane = p.M * ld;
    float* at = p.partial + (long long)p.share * (DUAL ? 2 : 1) * plane + row * ld + col;
    ff_store4(at, v0);
    if constexpr (DUAL) ff_store4(at + plane, v1);
    return;
  }
  f32x4 o0 = v0, o1 = v1;
  if constexpr (EPI == FF_SCALED) o0 *= p.scale;
  if constexpr (FF_BIAS<EPI>) {
    v0 += bias;
    o0 = ff_value4<sizeof(T) == 4>(p.act, v0);
    if constexpr (EPI == FF_LINEAR)
      if (p.drop.threshold) o0 = dropout4(p.drop, row, col >> 2, o0);
#pragma unroll
    for (int i = 0; i < 4; i++) o0[i] += (float)d.v[i];
  }
  if constexpr (EPI == FF_FWD || EPI == FF_GRAD) {
    f32x4 value, slope;
    ff_gate4<sizeof(T) == 4, EPI == FF_GRAD>(p.act, v0, value, slope);
    if constexpr (EPI == FF_FWD) {
      o0 = value * v1;
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        o0[i] = (float)d.v[i] * v1[i] * slope[i];
        o1[i] = (float)d.v[i] * value[i];
      }
    }
  }
  if (p.keep) {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < count && !p.keep[col + i]) o0[i] = o1[i] = v0[i] = v1[i] = 0.0f;
  }
  T* c0 = static_cast<T*>(p.C0) + row * p.ldc + col;
  if constexpr (EPI == FF_LINEAR) {
    if (p.G) {
      T* z = static_cast<T*>(p.G) + row * p.ldg + col;
      if (whole) ff_store4(z, v0);
      else
        for (int i = 0; i < count; i++) z[i] = ff_round<T>(v0[i]);
    }
  }
  T* c1 = (DUAL && EPI != FF_FWD) ? static_cast<T*>(p.C1) + row * p.ldc + col : nullptr;
  if (whole) {
    ff_store4(c0, o0);
    if constexpr (DUAL && EPI != FF_FWD) ff_store4(c1, o1);
  } else {
    for (int i = 0; i < count; i++) {
      c0[i] = ff_round<T>(o0[i]);
      if constexpr (DUAL && EPI != FF_FWD) c1[i] = ff_round<T>(o1[i]);
    }
  }
  if constexpr (EPI == FF_FWD) {
    if (p.G) {
      T* g = static_cast<T*>(p.G) + row * p.ldg + col;
      T* u = static_cast<T*>(p.U) + row * p.ldg + col;
      if (whole) {
        ff_store4(g, v0);
        ff_store4(u, v1);
      } else {
        for (int i = 0; i < count; i++) { g[i] = ff_round<T>(v0[i]); u[i] = ff_round<T>(v1[i]); }
      }
    }
  }
}

}  // namespace mlproj
#endif
