// mlproj: the kept channels of a masked block, packed side by side, so that pruned ones cost no products.
#ifndef MLPROJ_FFCOMPACT_H
#define MLPROJ_FFCOMPACT_H

#include "ffcommon.h"

namespace mlproj {

// ------------------------------------------------------------------ kept channels
// What the projection leaves of a weight matrix is a set of whole columns, scattered over its rows.  They are packed
// side by side in their order; their number is known on the device only, so kernels are launched for m columns and
// workgroups past the kept ones leave at once.  The number is filled up to a multiple of 8 with columns of zeros,
// which keeps packed rows in whole 16-byte pieces.  Bound by HBM and, where a wavefront's lanes scatter, by its
// requests: 4096 x 4096 -> 16384 bf16 backward with 40 % kept spends 11 + 88 + 48 + 124 us of 1420 here (index; weights and
// dH packed; gradients out, zeros included); without a mask it takes 2840.
// position[c], c = 0 .. m: where the caller's column c went, p, or ~p if it was pruned, with p the number of
// kept columns before it either way.
constexpr int FC_THREADS = 1024, FC_OWN = 16;
__global__ __launch_bounds__(FC_THREADS) void ff_index_kernel(const unsigned char* mask, long long m, int* position, int* kept) {
  __shared__ int wave_sum[FC_THREADS / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0;
  for (long long at = 0; at < m; at += FC_THREADS * FC_OWN) {
    const long long c0 = at + (long long)threadIdx.x * FC_OWN;
    unsigned char own[FC_OWN];
    if (c0 + FC_OWN <= m) {
      __builtin_memcpy(own, mask + c0, FC_OWN);
    } else {
#pragma unroll
      for (int i = 0; i < FC_OWN; i++) own[i] = c0 + i < m ? mask[c0 + i] : 0;
    }
    int count = 0;
#pragma unroll
    for (int i = 0; i < FC_OWN; i++) count += own[i] != 0;
    int upto = count;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int below = __shfl_up(upto, s);
      if (lane >= s) upto += below;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int p = base + upto - count;
    for (int w = 0; w < FC_THREADS / 64; w++) {
      if (w < wave) p += wave_sum[w];
      base += wave_sum[w];
    }
#pragma unroll
    for (int i = 0; i < FC_OWN; i++) {
      if (c0 + i < m) position[c0 + i] = own[i] ? p : ~p;
      p += own[i] != 0;
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    position[m] = ~base;
    *kept = (base + 7) / 8 * 8;
  }
}

struct FcArrays {
  const void* from[4];
  void* to[4];
  long long ld_from[4], ld_to[4], rows[4];
  long long cols;                         // of the caller's matrices
  const int *position, *kept;
  int count, groups[4];                   // matrices; workgroups along each one's rows
};

// A workgroup moves FC_COLS columns of the caller's matrix, FC_ROWS rows at a time, through LDS: packed ones out of the
// caller's (PACK), or the caller's out of packed ones with zeros where a channel was pruned.  Both sides of memory see
// whole 16-byte pieces of consecutive columns; the single elements are picked from LDS.  Bound by HBM: 4096 x 16384 bf16
// at 40 % kept, two matrices, 375 MB.
constexpr int FC_COLS = 2048, FC_ROWS = 4, FC_GROUPS = 1024;
template <typename T, bool PACK>
__global__ __launch_bounds__(256) void ff_move_kernel(FcArrays a) {
  __shared__ T held[FC_ROWS][FC_COLS + 8];
  __shared__ short source[PACK ? FC_COLS : 1];
  int which = 0, group = blockIdx.y;
  while (which + 1 < a.count && group >= a.groups[which]) group -= a.groups[which++];
  const T* from = static_cast<const T*>(a.from[which]);
  T* to = static_cast<T*>(a.to[which]);
  const long long ld_from = a.ld_from[which], ld_to = a.ld_to[which], rows = a.rows[which];
  const long long c0 = (long long)blockIdx.x * FC_COLS, c1 = c0 + FC_COLS < a.cols ? c0 + FC_COLS : a.cols;
  auto before = [&](long long c) { const int p = a.position[c]; return p < 0 ? ~p : p; };
  const int p0 = before(c0), p1 = before(c1);
  const int wide = (int)(c1 - c0), packed = p1 - p0;
  const int t8 = threadIdx.x * 8;
  int place[8];                                   // my eight columns in the packed segment, or -1
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const int p = t8 + i < wide ? a.position[c0 + t8 + i] : -1;
    place[i] = p < 0 ? -1 : p - p0;
    if (PACK && p >= 0) source[p - p0] = (short)(t8 + i);
  }
  if (PACK) __syncthreads();
  // the last segment also writes the columns of zeros that fill the packed rows up: behind a segment that was kept whole
  // up to seven of them lie past the eight columns per thread and are written on their own (`past`)
  const int filled = PACK ? (c1 == a.cols ? *a.kept - p0 : packed) : wide;
  const int in = PACK ? wide : packed, out = filled;
  const int past_row = threadIdx.x / 8, past = FC_COLS + threadIdx.x % 8;
  const bool writes_past = PACK && past_row < FC_ROWS && past < out;
  from += PACK ? c0 : p0;
  to += PACK ? p0 : c0;
  int pick[8];
#pragma unroll
  for (int i = 0; i < 8; i++) pick[i] = PACK ? (t8 + i < packed ? source[t8 + i] : -1) : place[i];
  FfVec8<T> v[FC_ROWS];
  auto fetch = [&](long long r0) {
#pragma unroll
    for (int r = 0; r < FC_ROWS; r++) v[r] = ff_load8(from + (r0 + r) * ld_from + t8, r0 + r < rows ? in - t8 : 0);
  };
  const long long stride = (long long)a.groups[which] * FC_ROWS;
  fetch((long long)group * FC_ROWS);
  for (long long r0 = (long long)group * FC_ROWS; r0 < rows; r0 += stride) {
    __syncthreads();
#pragma unroll
    for (int r = 0; r < FC_ROWS; r++) *reinterpret_cast<FfVec8<T>*>(&held[r][t8]) = v[r];
    if (r0 + stride < rows) fetch(r0 + stride);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < FC_ROWS; r++) {
      if (r0 + r >= rows || t8 >= out) continue;
      T* at = to + (r0 + r) * ld_to + t8;
      FfVec8<T> w;
#pragma unroll
      for (int i = 0; i < 8; i++) w.v[i] = pick[i] >= 0 ? held[r][pick[i]] : (T)0.0f;
      if (t8 + 8 <= out) {
        __builtin_memcpy(at, &w, sizeof(w));
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
          if (t8 + i < out) at[i] = w.v[i];
      }
    }
    if (writes_past && r0 + past_row < rows) to[(r0 + past_row) * ld_to + past] = (T)0.0f;
  }
}

}  // namespace mlproj
#endif
