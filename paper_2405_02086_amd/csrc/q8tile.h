// mlproj: products of 8-bit operands in tiles that go from memory straight into LDS.
#ifndef MLPROJ_Q8TILE_H
#define MLPROJ_Q8TILE_H

#include "ffcommon.h"
#include "ffdirect.h"
#include "q8.h"

namespace mlproj {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// C = A B^T, both operands rows of codes along K with their scales: p.A0 (M rows), p.B0 (N rows) and, for two products that
// share A, p.B1; strides in bytes, K in whole blocks.
struct Q8Product {
  FfProduct p;
  const unsigned char *sA, *sB0, *sB1;
  long long ldsa, ldsb;
};

// ------------------------------------------------------------------ operands
// EXACT: codes times scales as bf16, which holds them exactly (entries below 2^-126 are lost), for results in fp32: the matrix cores'
// own 8-bit products align the eight of a group to the largest of them and keep 16 bits, 1.5e-5 of a result's norm whatever K
// is.  That is lost in the rounding of 16-bit results, not in fp32 ones.  Eight codes (two dwords) with one scale, a byte:
__device__ __forceinline__ bf16x8 q8_widen(int lo, int hi, unsigned scale) {
  typedef bf16_t pair_t __attribute__((ext_vector_type(2)));
  const float s = __builtin_bit_cast(float, scale << 23);
  pair_t v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true),
                 __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true)};
  bf16x8 r;
  __builtin_memcpy(&r, v, 16);
  return r;
}

// ------------------------------------------------------------------ tiles
// The ring of ffdirect.h with rows of 64 codes: a step is one 32 x 32 x 64 matrix instruction per operand pair, whose lane holds 16 codes
// of each of two groups of a row and the scale of one of them.  The scales of two steps (a block of 128) are one dword per
// row, which comes with the even step's tile into one of two places.
constexpr int Q8_STEP = 64;

// Loads of `W` rows.
template <int W, int THREADS>
struct Q8Part {
  static constexpr int LOADS = W * Q8_STEP / 16 / THREADS;
  unsigned offset[LOADS];
  __device__ __forceinline__ void plan(int tid, long long ld, long long there) {
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const int q = tid + i * THREADS, row = q >> 2, piece = (q & 3) ^ fd_row_turn(row);
      offset[i] = row < there ? (unsigned)(row * ld + piece * 16) : FD_OUT;
    }
  }
  __device__ __forceinline__ void load(const unsigned char* base, bool there, unsigned char* lds, int wave) const {
    __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, there ? 0x7ffffff0u : 0u, 0x00020000);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const unsigned at = offset[i];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (fd_lds_t*)(lds + (wave * 64 + i * THREADS) * 16), 16, at, 0, 0, 0);
    }
  }
};

// A step's operands of a wavefront, the scales of two steps, and their products; ODD: the second of the two.
template <int RT, int CT> struct Q8Operands { i32x8 a[RT], b[CT]; };
template <int RT, int CT> struct Q8Scales { unsigned a[RT], b[CT]; };
template <bool EXACT, int ODD, int RT, int CT>
__device__ __forceinline__ void q8_multiply(const Q8Operands<RT, CT>& o, const Q8Scales<RT, CT>& s, f32x16 (&acc)[RT][CT]) {
  if constexpr (EXACT) {
#pragma unroll
    for (int k = 0; k < 4; k++) {
      bf16x8 b[CT];
#pragma unroll
      for (int j = 0; j < CT; j++) b[j] = q8_widen(o.b[j][2 * k], o.b[j][2 * k + 1], (s.b[j] >> (16 * ODD + 8 * (k >> 1))) & 255u);
#pragma unroll
      for (int i = 0; i < RT; i++) {
        const bf16x8 a = q8_widen(o.a[i][2 * k], o.a[i][2 * k + 1], (s.a[i] >> (16 * ODD + 8 * (k >> 1))) & 255u);
#pragma unroll
        for (int j = 0; j < CT; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j], a, acc[i][j], 0, 0, 0);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
      for (int j = 0; j < CT; j++)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(o.b[j], o.a[i], acc[i][j], 0, 0, 2 * ODD, (int)s.b[j], 2 * ODD, (int)s.a[i]);
  }
}

template <typename T, bool DUAL, int EPI, int BM, int BN, int WM, int WN, bool EXACT>
__global__ __launch_bounds__(WM * WN * 64) void q8_tile_kernel(Q8Product q) {
  constexpr int WAVES = WM * WN, THREADS = WAVES * 64, BW = BN / 2;
  constexpr int RT = BM / WM / 32, CJ = BN / WN / 64;          // 32 x 32 tiles of a wavefront: down, across in each half
  constexpr int STAGE = (BM + BN) * Q8_STEP;
  constexpr int CHUNKS = (BM + BN) / 64, SLOADS = (CHUNKS + WAVES - 1) / WAVES;
  __shared__ __align__(16) unsigned char lds0[STAGE], lds1[STAGE], lds2[STAGE], lds3[STAGE];
  __shared__ __align__(16) unsigned char scales0[SLOADS * WAVES * 256], scales1[SLOADS * WAVES * 256];
  FfProduct& p = q.p;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const long long N = p.N;
  constexpr int COLS = DUAL ? BW : BN;
  long long row0, col0;
  if (!ff_tile<BM, COLS>(p, N, &row0, &col0)) return;
  const int blocks = (int)(p.K / Q8_BLOCK);
  const int first = (int)((long long)blocks * p.share / p.splits) * 2, last = (int)((long long)blocks * (p.share + 1) / p.splits) * 2;

  Q8Part<BM, THREADS> pa;
  Q8Part<BW, THREADS> pb[2];
  pa.plan(tid, p.lda, p.M - row0);
#pragma unroll
  for (int i = 0; i < 2; i++) pb[i].plan(tid, p.ldb, N - (col0 + (DUAL ? 0 : i * BW)));
  const unsigned char *A = static_cast<const unsigned char*>(p.A0) + row0 * p.lda;
  const unsigned char* B[2] = {static_cast<const unsigned char*>(p.B0) + col0 * p.ldb,
                               DUAL ? static_cast<const unsigned char*>(p.B1) + col0 * p.ldb : static_cast<const unsigned char*>(p.B0) + (col0 + BW) * p.ldb};
  auto load = [&](int step, unsigned char* lds) {
    const long long k0 = (long long)step * Q8_STEP;
    const bool there = step < last;
    pa.load(A + k0, there, lds, wave);
#pragma unroll
    for (int i = 0; i < 2; i++) pb[i].load(B[i] + k0, there, lds + (BM + i * BW) * Q8_STEP, wave);
  };
  const unsigned char *const sA = q.sA, *const sB0 = q.sB0, *const sB1 = q.sB1;
  const long long ldsa = q.ldsa, ldsb = q.ldsb;
  // 64 rows' scales per wavefront and load: A's, then those of both halves of B
  auto load_scales = [&](int block, unsigned char* to) {
#pragma unroll
    for (int i = 0; i < SLOADS; i++) {
      const int chunk = wave + i * WAVES, of_b = chunk - BM / 64, half = of_b >= BW / 64;
      const long long at = of_b < 0 ? row0 + chunk * 64 : col0 + (DUAL || !half ? 0 : BW) + (of_b - half * (BW / 64)) * 64;
      const long long there = chunk >= CHUNKS ? 0 : (of_b < 0 ? p.M : N) - at, ld = of_b < 0 ? +ldsa : +ldsb;
      const unsigned char* base = sA;
      if (of_b >= 0) base = DUAL && half ? +sB1 : +sB0;
      base += at * ld + (long long)block * 4;
      __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, block * 2 < last ? 0x7ffffff0u : 0u, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (fd_lds_t*)(to + chunk * 256), 4, lane < there ? (unsigned)(lane * ld) : FD_OUT, 0, 0, 0);
    }
  };

  f32x16 acc[RT][2 * CJ] = {};
  const int r = lane & 31, h = lane >> 5;
  using Operands = Q8Operands<RT, 2 * CJ>;
  using Scales = Q8Scales<RT, 2 * CJ>;
  const int turn = fd_row_turn(r), low = r * Q8_STEP + ((h ^ turn) << 4), high = r * Q8_STEP + (((2 + h) ^ turn) << 4);
  auto fragment = [&](const unsigned char* lds, int row) {
    u32x4 v[2] = {*reinterpret_cast<const u32x4*>(lds + (low + row * Q8_STEP)), *reinterpret_cast<const u32x4*>(lds + (high + row * Q8_STEP))};
    i32x8 f;
    __builtin_memcpy(&f, v, 32);
    return f;
  };
  auto read = [&](const unsigned char* lds) {
    Operands o;
#pragma unroll
    for (int j = 0; j < 2 * CJ; j++) o.b[j] = fragment(lds, BM + (j / CJ) * BW + wn * CJ * 32 + j % CJ * 32);
#pragma unroll
    for (int i = 0; i < RT; i++) o.a[i] = fragment(lds, wm * RT * 32 + i * 32);
    return o;
  };
  // the scales a lane gives are those of group h of a step
  auto read_scales = [&](const unsigned char* from) {
    Scales s;
#pragma unroll
    for (int j = 0; j < 2 * CJ; j++) s.b[j] = *reinterpret_cast<const unsigned*>(from + (BM + (j / CJ) * BW + wn * CJ * 32 + j % CJ * 32 + r) * 4);
#pragma unroll
    for (int i = 0; i < RT; i++) s.a[i] = *reinterpret_cast<const unsigned*>(from + (wm * RT * 32 + i * 32 + r) * 4);
    if constexpr (!EXACT) {
#pragma unroll
      for (int j = 0; j < 2 * CJ; j++) s.b[j] >>= 8 * h;
#pragma unroll
      for (int i = 0; i < RT; i++) s.a[i] >>= 8 * h;
    }
    return s;
  };
  // Behind this all loads but those of the last two steps are in LDS (an even step's come with scales), and nobody reads what was read before.
  constexpr int LOADS = (BM + BN) * Q8_STEP / 16 / THREADS;
  auto meet = [&]() {
    asm volatile("" ::: "memory");
    constexpr int v = 2 * LOADS + SLOADS;
    __builtin_amdgcn_s_waitcnt(0x0070 | (v & 15) | ((v >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  constexpr int MFMAS = RT * 2 * CJ, READS = (RT + 2 * CJ) * 2;
  Operands even, odd;
  Scales here, next;
  // An even step makes room in its block's place for the scales of the block after the next one; an odd step reads the next block's.
  auto even_step = [&](int step, unsigned char* at, unsigned char* ahead, unsigned char* scales) {
    meet();
    load_scales(step / 2 + 2, scales);
    load(step + 4, at);
    odd = read(ahead);
    q8_multiply<EXACT, 0>(even, here, acc);
    if constexpr (!EXACT) fd_schedule<0, MFMAS, READS>();
  };
  auto odd_step = [&](int step, unsigned char* at, unsigned char* ahead, const unsigned char* scales) {
    meet();
    load(step + 4, at);
    even = read(ahead);
    next = read_scales(scales);
    q8_multiply<EXACT, 1>(odd, here, acc);
    if constexpr (!EXACT) fd_schedule<0, MFMAS, READS + RT + 2 * CJ>();
    here = next;
  };

  load_scales(first / 2, scales0);
  load(first, lds0);
  load(first + 1, lds1);
  load_scales(first / 2 + 1, scales1);
  load(first + 2, lds2);
  meet();
  even = read(lds0);
  here = read_scales(scales0);
  load(first + 3, lds3);
  int step = first;
  for (; step + 2 < last; step += 4) {
    even_step(step, lds0, lds1, scales0);
    odd_step(step + 1, lds1, lds2, scales1);
    even_step(step + 2, lds2, lds3, scales1);
    odd_step(step + 3, lds3, lds0, scales0);
  }
  if (step < last) {
    even_step(step, lds0, lds1, scales0);
    odd_step(step + 1, lds1, lds2, scales1);
  }
  // no load may be under way where results go, or when the workgroup's LDS is given to another
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);            // vmcnt(0) lgkmcnt(0)
  __syncthreads();

  // Results through LDS, each wavefront's in a share of its own, in whole rows (as in ffdirect.h).
  constexpr int QUADS = 2 * CJ * 8, PITCH = QUADS * 16, TILES = RT < 2 ? RT : 2, CHUNK = 4;
  constexpr int ACROSS = DUAL ? QUADS / 2 : QUADS, DOWN = 64 / ACROSS;      // of a wavefront's lanes
  constexpr int SHARE = TILES * 32 * PITCH, PER = STAGE / SHARE;
  static_assert(PER >= 1 && PER * 4 >= WAVES, "a wavefront's share of the stages");
  typedef __attribute__((address_space(3))) unsigned char byte_t;
  typedef __attribute__((address_space(3))) f32x4 quad_t;
  const int stage = wave / PER;
  byte_t* mine = (stage == 0 ? (byte_t*)lds0 : stage == 1 ? (byte_t*)lds1 : stage == 2 ? (byte_t*)lds2 : (byte_t*)lds3) + wave % PER * SHARE;
  dropout_at_step(p.drop);
  const int quad = lane % ACROSS, down = lane / ACROSS, j = quad >> 3;
  const long long col = col0 + wn * CJ * 32 + (j < CJ ? j * 32 : BW + (j - CJ) * 32) + (quad & 7) * 4;
  const f32x4 bias = EPI == FF_LINEAR && col < N ? ff_bias<T>(p, col, N) : f32x4{};
#pragma unroll
  for (int pass = 0; pass < RT / TILES; pass++) {
#pragma unroll
    for (int i = 0; i < TILES; i++)
#pragma unroll
      for (int jj = 0; jj < 2 * CJ; jj++)
#pragma unroll
        for (int u = 0; u < 4; u++) {
          const f32x16& t = acc[pass * TILES + i][jj];
          *(quad_t*)(mine + (i * 32 + r) * PITCH + (((jj * 8 + 2 * u + h) ^ (r & 15)) << 4)) = f32x4{t[4 * u], t[4 * u + 1], t[4 * u + 2], t[4 * u + 3]};
        }
    const long long first_row = row0 + wm * RT * 32 + pass * TILES * 32 + down;
    FfVec4<T> d[CHUNK], ahead[CHUNK];
    auto fetch = [&](int chunk, FfVec4<T> (&to)[CHUNK]) {
#pragma unroll
      for (int u = 0; u < CHUNK; u++) {
        const long long row = first_row + (chunk * CHUNK + u) * DOWN;
        to[u] = {};
        if (EPI == FF_LINEAR && p.dH && row < p.M && col < N) to[u] = ff_upstream<T>(p, row, col, N);
      }
    };
    constexpr int ROUNDS = TILES * 32 / DOWN / CHUNK;
    static_assert(ROUNDS * DOWN * CHUNK == TILES * 32, "whole chunks");
    fetch(0, d);
#pragma unroll 1
    for (int chunk = 0; chunk < ROUNDS; chunk++) {
      if (chunk + 1 < ROUNDS) fetch(chunk + 1, ahead);
#pragma unroll
      for (int u = 0; u < CHUNK; u++) {
        const int in = (chunk * CHUNK + u) * DOWN + down;
        const f32x4 v0 = *(const quad_t*)(mine + in * PITCH + ((quad ^ (in & 15)) << 4));
        f32x4 v1 = {};
        if constexpr (DUAL) v1 = *(const quad_t*)(mine + in * PITCH + (((quad + ACROSS) ^ (in & 15)) << 4));
        const long long row = first_row + (chunk * CHUNK + u) * DOWN;
        if (row < p.M && col < N) ff_finish<EPI, DUAL, T>(p, row, col, N, v0, v1, d[u], bias);
        d[u] = ahead[u];
      }
    }
  }
}

}  // namespace
}  // namespace mlproj
#endif
