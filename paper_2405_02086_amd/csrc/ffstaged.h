// mlproj: matrix products of the gated feed-forward block on the matrix cores, operands staged through
// registers: any size, stride and alignment, 16-bit elements and fp32.
#ifndef MLPROJ_FFSTAGED_H
#define MLPROJ_FFSTAGED_H

#include "ffcommon.h"

namespace mlproj {

// ------------------------------------------------------------------ tiles staged through registers
// A workgroup of four wavefronts computes 128 rows x 128 columns (two products: 128 x 64 of each, the same
// columns of both), each wavefront 64 x 64 of them, in steps of 32 along K.  The next step's operands are
// loaded into registers while the matrix cores work on the present one in LDS.  Loads take any address, and
// what lies outside the matrix is filled with zeros element by element, so nothing is asked of sizes,
// strides or alignment.  16-bit elements come here only where copying them into aligned rows costs more than it saves
// (ff_pads): a step of a tile takes two to three times the direct tiles' (2047 x 2047 -> 4095 bf16 forward 169 us here, 81 with copies,
// the copies included).
//
// fp32 goes through the bf16 matrix cores: an element is cut into three bf16 parts of 8 significant bits each
// (x = p0 + p1 + p2 exactly, by truncation), and a product of two elements is summed from the six products of
// parts that reach 2^-16 of it.  What is left out is 2^-24 of a product on average (2^-21 at most), and the sums are
// fp32 throughout.  Six bf16 products cost 6/16 of what the chip's fp32 matrix instructions would.  Bound by the vector
// instructions that cut: 2048 x 2048 -> 4096 fp32 runs at 192 TFLOP/s forward and 195 backward, the library's plain products at
// 150 to 154.  Largest error of G over 7467 x 488 -> 1024: 3.3e-7 rms, the library's 4.0e-7.
// (A part past the range of bf16's exponent, below 2^-126, is lost: an absolute error no sum can see.  What remains of an
// infinity is a NaN, and so are the sums that it is part of: fs_again.)
constexpr int FS_M = 128, FS_N = 128, FS_K = 32, FS_THREADS = 256;

template <typename T> struct FfParts { static constexpr int count = 1; using type = T; };
template <> struct FfParts<float> { static constexpr int count = 3; using type = bf16_t; };

__device__ __forceinline__ f32x4 ff_mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 ff_mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

template <typename E> struct FfFrag;
template <> struct FfFrag<bf16_t> { using type = bf16x8; };
template <> struct FfFrag<f16_t> { using type = f16x8; };

// Eight elements as the 16 bytes of each of their parts.  INFINITIES: an infinity is its first part alone; otherwise what
// remains of it is a NaN.
template <typename T, bool INFINITIES = false>
__device__ __forceinline__ void fs_parts(const FfVec8<T>& x, u32x4 (&out)[FfParts<T>::count]) {
  if constexpr (FfParts<T>::count == 1) {
    __builtin_memcpy(&out[0], &x, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      unsigned w[3][2];
#pragma unroll
      for (int j = 0; j < 2; j++) {
        const float a = x.v[2 * i + j];
        const unsigned a0 = __builtin_bit_cast(unsigned, a) & 0xffff0000u;
        const float r1 = INFINITIES && __builtin_isinf(a) ? 0.0f : a - __builtin_bit_cast(float, a0);
        const unsigned a1 = __builtin_bit_cast(unsigned, r1) & 0xffff0000u;
        w[0][j] = a0;
        w[1][j] = a1;
        w[2][j] = __builtin_bit_cast(unsigned, r1 - __builtin_bit_cast(float, a1));
      }
#pragma unroll
      for (int k = 0; k < 3; k++) out[k][i] = __builtin_amdgcn_perm(w[k][1], w[k][0], 0x07060302);
    }
  }
}

// A tile in LDS: 128 rows (columns) x 32 along K.  KC (K runs along the rows of memory): [128][32], so that a
// lane's eight K values are 16 bytes; the 16-byte pieces of a row are permuted by the row's number, which
// spreads eight rows over all banks.  Otherwise [32][128], read with the transposing LDS load: 16 lanes take
// a 4 x 16 block and get its columns; the 32-byte pieces of a row are permuted for the same reason.
__device__ __forceinline__ int fs_put(bool kc, int chunk) {
  if (kc) {
    const int row = chunk >> 2, c = chunk & 3;
    return row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
  }
  const int k = chunk >> 4, c = chunk & 15;
  const int f = (k & 3) | (((k >> 3) & 1) << 2);
  return k * 256 + (((c >> 1) ^ f) << 5) + ((c & 1) << 4);
}
template <bool KC, typename F>
__device__ __forceinline__ F fs_frag(const unsigned char* tile, int idx, int lane) {
  F r;
  const int g = lane >> 4, c = lane & 15;
  if constexpr (KC) {
    const int row = idx * 16 + c;
    r = *reinterpret_cast<const F*>(tile + row * 64 + ((g ^ ((row >> 1) & 3)) << 4));
  } else {
    const int f = (c >> 2) | ((g & 1) << 2);
    const unsigned char* at = tile + (8 * g + (c >> 2)) * 256 + ((idx ^ f) << 5) + ((c & 3) << 3);
    typedef __attribute__((address_space(3))) s16x4 lds_t;
    s16x4 half[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)at), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(at + 4 * 256))};
    __builtin_memcpy(&r, half, 16);
  }
  return r;
}

// Sums in fp32 that came out as NaN, again: with the fp32 matrix instructions, whose infinities are infinities, straight from
// memory.  Each wavefront does that for the 16 columns at a time of its part of the tile in which there are any (and the channel
// is not pruned); the others keep their bits.  Two to four times a tile's time, for
// tiles with infinities or NaN alone (2048 x 2048 -> 4096 forward with one NaN token: 360 -> 1300 us); looking for them costs calls of
// few steps 2 to 7 %, others nothing that was measured.
template <bool A_KC, bool B_KC, bool DUAL>
__device__ __forceinline__ void fs_again(const FfProduct& p, long long row0, long long col0, long long N, long long K, long long ksteps,
                                         long long first, long long last, int lane, f32x4 (&acc)[4][4]) {
  const int g = lane >> 4, c = lane & 15;
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const long long left = col0 + (j & 1) * 16 + (DUAL || j < 2 ? 0 : 64);      // of these sixteen columns; a lane's results: four of them
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int v = 0; v < 4; v++) {
        const long long at = left + g * 4 + v;
        if (acc[i][j][v] != acc[i][j][v] && at < N && row0 + i * 16 + c < p.M) nan = nan || !p.keep || p.keep[at];
      }
    if (!__any(nan)) continue;
    f32x4 sum[4] = {};
    const long long col = left + c;
    for (long long step = first; step < last; step++) {
      const int seg = step >= ksteps;
      const long long k0 = (step - (seg ? ksteps : 0)) * FS_K + 8 * g;
      const float* A = static_cast<const float*>(seg ? p.A1 : p.A0);
      const float* B = static_cast<const float*>((DUAL ? j >= 2 : seg) ? p.B1 : p.B0);
      FfVec8<float> b, a[4];
      if constexpr (B_KC) b = ff_load8(B + col * p.ldb + k0, col < N ? K - k0 : 0);
      else
#pragma unroll
        for (int s = 0; s < 8; s++) b.v[s] = col < N && k0 + s < K ? B[(k0 + s) * p.ldb + col] : 0.0f;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const long long row = row0 + i * 16 + c;
        if constexpr (A_KC) a[i] = ff_load8(A + row * p.lda + k0, row < p.M ? K - k0 : 0);
        else
#pragma unroll
          for (int s = 0; s < 8; s++) a[i].v[s] = row < p.M && k0 + s < K ? A[(k0 + s) * p.lda + row] : 0.0f;
      }
#pragma unroll
      for (int s = 0; s < 8; s++)
#pragma unroll
        for (int i = 0; i < 4; i++) sum[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(b.v[s], a[i].v[s], sum[i], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int v = 0; v < 4; v++) acc[i][j][v] = acc[i][j][v] != acc[i][j][v] ? sum[i][v] : acc[i][j][v];
  }
}

template <typename T, bool A_KC, bool B_KC, bool DUAL, int EPI>
__global__ __launch_bounds__(FS_THREADS) void ff_staged_kernel(FfProduct p) {
  using E = typename FfParts<T>::type;
  using F = typename FfFrag<E>::type;
  constexpr int P = FfParts<T>::count;
  constexpr int TILE = 128 * FS_K * 2;                     // bytes of a tile of one part
  __shared__ __align__(16) unsigned char lds[2 * P * TILE];   // A's parts, then B's
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  constexpr int COLS = DUAL ? 64 : 128;                    // columns of each product in a tile
  const long long N = p.kept && !(B_KC && A_KC) ? *p.kept : p.N;
  const long long K = p.kept && (B_KC && A_KC) ? *p.kept : p.K;
  long long row0, col0;
  if (!ff_tile<FS_M, COLS>(p, N, &row0, &col0)) return;
  const long long ksteps = (K + FS_K - 1) / FS_K, all = ksteps * p.segs;
  const long long first = all * p.share / p.splits, last = all * (p.share + 1) / p.splits;

  FfVec8<T> ra[2], rb[2];
  auto fetch = [&](long long step) {
    const int seg = step >= ksteps;
    const long long k0 = (step - (seg ? ksteps : 0)) * FS_K;
    const T* A = static_cast<const T*>(seg ? p.A1 : p.A0);
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int c = tid + i * FS_THREADS;
      if constexpr (A_KC) {
        const long long r = row0 + (c >> 2), k = k0 + (c & 3) * 8;
        ra[i] = ff_load8(A + r * p.lda + k, r < p.M ? K - k : 0);
      } else {
        const long long k = k0 + (c >> 4), r = row0 + (c & 15) * 8;
        ra[i] = ff_load8(A + k * p.lda + r, k < K ? p.M - r : 0);
      }
      if constexpr (B_KC) {
        const int j = c >> 2;
        const T* B = static_cast<const T*>(DUAL ? (j < 64 ? p.B0 : p.B1) : (seg ? p.B1 : p.B0));
        const long long col = col0 + (DUAL ? j & 63 : j), k = k0 + (c & 3) * 8;
        rb[i] = ff_load8(B + col * p.ldb + k, col < N ? K - k : 0);
      } else {
        const int j = (c & 15) * 8;
        const T* B = static_cast<const T*>(DUAL ? (j < 64 ? p.B0 : p.B1) : (seg ? p.B1 : p.B0));
        const long long col = col0 + (DUAL ? j & 63 : j), k = k0 + (c >> 4);
        rb[i] = ff_load8(B + k * p.ldb + col, k < K ? N - col : 0);
      }
    }
  };
  auto put = [&]() {
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int c = tid + i * FS_THREADS;
      u32x4 parts[P];
      fs_parts(ra[i], parts);
#pragma unroll
      for (int k = 0; k < P; k++) *reinterpret_cast<u32x4*>(lds + k * TILE + fs_put(A_KC, c)) = parts[k];
      fs_parts(rb[i], parts);
#pragma unroll
      for (int k = 0; k < P; k++) *reinterpret_cast<u32x4*>(lds + (P + k) * TILE + fs_put(B_KC, c)) = parts[k];
    }
  };

  // acc[i][j]: rows 16 i of the wavefront's 64; j = 0, 1: columns 32 wn + 16 j of the tile's left half, 2, 3 of
  // the right one.  The operands are given in the order (B, A), so that a lane holds four neighbouring columns.
  f32x4 acc[4][4] = {};
  if (first < last) fetch(first);
  for (long long step = first; step < last; step++) {
    __syncthreads();
    put();
    __syncthreads();
    if (step + 1 < last) fetch(step + 1);
    F a[P][4], b[P][4];
#pragma unroll
    for (int k = 0; k < P; k++) {
#pragma unroll
      for (int i = 0; i < 4; i++) a[k][i] = fs_frag<A_KC, F>(lds + k * TILE, wm * 4 + i, lane);
#pragma unroll
      for (int j = 0; j < 4; j++) b[k][j] = fs_frag<B_KC, F>(lds + (P + k) * TILE, (j >> 1) * 4 + wn * 2 + (j & 1), lane);
    }
    // the smallest parts first
#pragma unroll
    for (int sum = P - 1; sum >= 0; sum--)
#pragma unroll
      for (int ka = 0; ka <= sum; ka++)
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
          for (int j = 0; j < 4; j++) acc[i][j] = ff_mfma(b[sum - ka][j], a[ka][i], acc[i][j]);
  }

  if constexpr (P > 1) {
    // an infinity of A is a row of NaN, one of B a column: one entry of each shows them all
    bool nan = __builtin_isunordered(acc[0][0][0], acc[1][0][0]) || __builtin_isunordered(acc[2][0][0], acc[3][0][0]);
#pragma unroll
    for (int j = 0; j < 4; j++) nan = nan || __builtin_isunordered(acc[0][j][0], acc[0][j][1]) || __builtin_isunordered(acc[0][j][2], acc[0][j][3]);
    if (__any(nan)) fs_again<A_KC, B_KC, DUAL>(p, row0 + wm * 64, col0 + wn * 32, N, K, ksteps, first, last, lane, acc);
  }

  FfVec4<T> d[4][2] = {};
  if constexpr (EPI == FF_GRAD) {
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int j = 0; j < 2; j++) {
        const long long row = row0 + wm * 64 + i * 16 + (lane & 15), col = col0 + wn * 32 + j * 16 + (lane >> 4) * 4;
        if (row < p.M && col < N) d[i][j] = ff_upstream<T>(p, row, col, N);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const long long row = row0 + wm * 64 + i * 16 + (lane & 15);
    if (row >= p.M) continue;
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const long long col = col0 + wn * 32 + j * 16 + (lane >> 4) * 4;
      if constexpr (DUAL) {
        if (col < N) ff_finish<EPI, true, T>(p, row, col, N, acc[i][j], acc[i][2 + j], d[i][j]);
      } else {
        if (col < N) ff_finish<EPI, false, T>(p, row, col, N, acc[i][j], f32x4{}, {});
        if (col + 64 < N) ff_finish<EPI, false, T>(p, row, col + 64, N, acc[i][2 + j], f32x4{}, {});
      }
    }
  }
}

// Joins the shares of K: sums the partial products in their order and finishes them.  GROUPS threads share a quad's sum where
// the shares are many and the quads few, each a run of shares; their sums are added in order.
template <typename T, bool DUAL, int EPI, int GROUPS>
__global__ __launch_bounds__(256) void ff_join_kernel(FfProduct p) {
  constexpr int QUADS = 256 / GROUPS, PLANES = DUAL ? 2 : 1;
  __shared__ f32x4 sums[GROUPS > 1 ? GROUPS : 1][PLANES][QUADS];
  const long long quads = (p.N + 3) / 4, plane = p.M * quads * 4;
  const int in = threadIdx.x % QUADS, group = threadIdx.x / QUADS;
  const long long i = (long long)blockIdx.x * QUADS + in;
  const long long row = i / quads, col = i % quads * 4;
  const long long N = p.kept && DUAL ? *p.kept : p.N;
  const bool there = i < quads * p.M && col < N;
  f32x4 v[2] = {};
  if (there) {
    const float* at = p.partial + i * 4;
    const int last = p.splits * (group + 1) / GROUPS;
#pragma unroll 8
    for (int s = p.splits * group / GROUPS; s < last; s++)
#pragma unroll
      for (int k = 0; k < PLANES; k++) v[k] += ff_load4(at + (s * PLANES + k) * plane);
  }
  if constexpr (GROUPS > 1) {
#pragma unroll
    for (int k = 0; k < PLANES; k++) sums[group][k][in] = v[k];
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 1; g < GROUPS; g++)
#pragma unroll
      for (int k = 0; k < PLANES; k++) v[k] += sums[g][k][in];
  }
  if (!there) return;
  FfVec4<T> d = {};
  if constexpr (EPI == FF_GRAD) d = ff_upstream<T>(p, row, col, N);
  ff_finish<EPI, DUAL, T>(p, row, col, N, v[0], v[1], d);
}

}  // namespace mlproj
#endif
