// mlproj: the kept channels of a masked block, packed side by side, so that pruned ones cost no products.
#ifndef MLPROJ_FFCOMPACT_H
#define MLPROJ_FFCOMPACT_H

#include "ffcommon.h"

namespace mlproj {

// ------------------------------------------------------------------ kept channels
// What the projection leaves of a weight matrix is a set of whole columns, scattered over its rows.  Column j of
// the packed matrices is column index[j] of the caller's; their number is known on the device only, so kernels are
// launched for m columns and workgroups past the kept ones leave at once.  The number is filled up to a
// multiple of 8 with columns of zeros (index -1), which keeps packed rows in whole 16-byte pieces.
// position[c] is where the caller's column c went, or -1.
constexpr int FC_THREADS = 1024;
__global__ __launch_bounds__(FC_THREADS) void ff_index_kernel(const unsigned char* mask, long long m, int* index, int* position, int* kept) {
  __shared__ int wave_sum[FC_THREADS / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0;
  for (long long at = 0; at < m; at += FC_THREADS) {
    const long long c = at + threadIdx.x;
    const bool there = c < m && mask[c];
    const unsigned long long votes = __ballot(there);
    if (lane == 0) wave_sum[wave] = __popcll(votes);
    __syncthreads();
    int before = base, all = 0;
    for (int w = 0; w < FC_THREADS / 64; w++) {
      if (w < wave) before += wave_sum[w];
      all += wave_sum[w];
    }
    const int mine = before + __popcll(votes & ((1ull << lane) - 1));
    if (c < m) position[c] = there ? mine : -1;
    if (there) index[mine] = (int)c;
    base += all;
    __syncthreads();
  }
  const int whole = (base + 7) / 8 * 8;
  if (threadIdx.x < whole - base) index[base + threadIdx.x] = -1;
  if (threadIdx.x == 0) *kept = whole;
}

struct FcArrays {
  const void* from[3];
  void* to[3];
  long long ld_from, ld_to, rows, cols;   // cols: of the caller's matrices
  const int* map;                         // index or position
  const int* kept;
};

// Eight columns x FC_ROWS rows per thread; the map's eight entries are read once for all of them.  GATHER: packed
// columns from the caller's, else the caller's from packed ones, with zeros where a channel was pruned.
constexpr int FC_ROWS = 8;
template <typename T, bool GATHER>
__global__ __launch_bounds__(256) void ff_move_kernel(FcArrays a) {
  const long long limit = GATHER ? *a.kept : a.cols;
  const long long col = ((long long)blockIdx.x * 256 + threadIdx.x) * 8;
  if (col >= limit) return;
  const T* from = static_cast<const T*>(a.from[blockIdx.z]);
  T* to = static_cast<T*>(a.to[blockIdx.z]);
  const int count = limit - col < 8 ? (int)(limit - col) : 8;
  int map[8];
#pragma unroll
  for (int i = 0; i < 8; i++) map[i] = i < count ? a.map[col + i] : -1;
  for (long long r0 = (long long)blockIdx.y * FC_ROWS; r0 < a.rows; r0 += (long long)gridDim.y * FC_ROWS) {
    FfVec8<T> v[FC_ROWS];
#pragma unroll
    for (int r = 0; r < FC_ROWS; r++)
#pragma unroll
      for (int i = 0; i < 8; i++) v[r].v[i] = map[i] >= 0 && r0 + r < a.rows ? from[(r0 + r) * a.ld_from + map[i]] : (T)0.0f;
#pragma unroll
    for (int r = 0; r < FC_ROWS; r++) {
      if (r0 + r >= a.rows) break;
      T* at = to + (r0 + r) * a.ld_to + col;
      if (count == 8) {
        __builtin_memcpy(at, &v[r], sizeof(v[r]));
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
          if (i < count) at[i] = v[r].v[i];
      }
    }
  }
}

}  // namespace mlproj
#endif
