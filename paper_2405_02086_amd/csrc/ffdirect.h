// mlproj: matrix products of the gated feed-forward block for 16-bit elements in aligned rows: tiles go from memory
// to LDS without passing through registers.
#ifndef MLPROJ_FFDIRECT_H
#define MLPROJ_FFDIRECT_H

#include "ffcommon.h"
#include "ffstaged.h"

namespace mlproj {

// ------------------------------------------------------------------ tiles straight into LDS
// A tile is 32 deep.  FD_STAGES of them lie in LDS as a ring: while the matrix cores work on the operands of one, which are in
// registers, the next one's are read from LDS and the loads of the ones behind it, 16 bytes per lane and straight into
// LDS, are under way.  One barrier per tile: behind it the next tile is complete and everybody has left the present one's
// place, which the loads of the tile FD_STAGES further on then take.
//
// The tile is cut into parts of 64 or 128 rows (of A), columns (of B).  A part whose K runs along memory rows is [row][32]:
// 64 bytes per row, its 16-byte pieces permuted by the row's number so that eight rows spread over all banks.  A part
// whose memory rows are the K index is read with the transposing load, whose half wavefront reads 32 bytes (16 columns) of
// eight rows k = 16 G + 8 g + 4 h + r (one G and h; g < 2, r < 4); so those eight rows x 64 columns are a block of 1 KiB,
// [32 columns: 2][row 4 g + r][64 bytes], in which rows with g = 1 have their two halves exchanged: the half wavefront meets
// every bank once, the four lanes that load a row's 64 bytes stay within one cache line, and operand after
// operand lies at constant distances.  Lanes write LDS in order, so all permutations are applied to the addresses they load from.
//
// Bound by the matrix cores where tiles are many: 4096 x 4096 -> 16384 bf16 forward takes 850 us, 1.29 PFLOP/s (the library's
// plain products of this size reach 1.2 to 1.4); by memory with few tokens: 1 x 4096 -> 16384 takes 47 us, 5.7 TB/s.  Tiles of 256
// x 256, 128 x 128 and 64 x 128 (32, 16 and 11 operations per byte brought to LDS; one, two and three workgroups per
// compute unit, by their 128, 64 and 48 KiB of LDS); ff_plan chooses.  Results leave as 8 bytes per lane: through LDS and in whole
// rows they were no faster (dX, dW 0 to 3 % slower), L2 joins them.
//
// Requires (checked by ff_direct): 16-byte aligned operands, rows and K (or the row length) in whole 16-byte pieces.
// Outside the matrix a lane's offset lies past the end of the buffer resource and the load returns zeros.
constexpr int FD_K = 32, FD_STAGES = 4;
constexpr unsigned FD_OUT = 0xfffffff0u;         // past any buffer

typedef __attribute__((address_space(3))) void fd_lds_t;

// What the 16-byte pieces of a row [row][32] are permuted by.
__device__ __forceinline__ int fd_row_turn(int row) { return (row >> 1) & 3; }

// Loads of one part.  offset[i]: where lane's i-th piece lies from the part's first element of the step.
template <bool KC, int W, int THREADS>
struct FdPart {
  static constexpr int LOADS = W * FD_K / 8 / THREADS;
  unsigned offset[LOADS];
  unsigned k_of[LOADS];                          // KC: first K index of the piece within the step

  // `there`: rows (KC) or columns that exist from the part's first one on
  __device__ __forceinline__ void plan(int tid, long long ld, long long there) {
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const int p = tid + i * THREADS;
      if constexpr (KC) {
        const int row = p / (FD_K / 8), piece = (p % (FD_K / 8)) ^ fd_row_turn(row);
        offset[i] = row < there ? (unsigned)(row * ld * 2 + piece * 16) : FD_OUT;
        k_of[i] = piece * 8;
      } else {
        const int block = p >> 6, in = p & 63, row = (in >> 2) & 7;
        const int k = (block >> 1 & 1) * 16 + (row >> 2) * 8 + (block & 1) * 4 + (row & 3);
        const int col = (block >> 2) * 64 + (in >> 5) * 32 + (((in >> 1) & 1) ^ (row >> 2)) * 16 + (in & 1) * 8;
        offset[i] = col < there ? (unsigned)(k * ld * 2 + col * 2) : FD_OUT;
      }
    }
  }
  // base: the part's first element of the step; left: K indices from the step's first one to the end
  __device__ __forceinline__ void load(const void* base, long long ld, long long left, unsigned char* lds, int wave) const {
    const int k_here = left < FD_K ? (int)left : FD_K;
    const unsigned bytes = KC ? 0x7ffffff0u : (unsigned)(k_here * ld * 2);
    __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const unsigned at = KC && (int)k_of[i] >= k_here ? FD_OUT : offset[i];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (fd_lds_t*)(lds + (wave * 64 + i * THREADS) * 16), 16, at, 0, 0, 0);
    }
  }
};

// Where a lane finds its operands in a part, from the part's sixteen rows (columns) number `first` on: the place of the
// first one and of the second one.
struct FdFrom { int at[2]; };
template <bool KC>
__device__ __forceinline__ FdFrom fd_from(int part, int first, int lane) {
  const int g = lane >> 4, c = lane & 15;
  if (KC) {
    const int at = part + (first * 16 + c) * (FD_K * 2) + ((g ^ fd_row_turn(c)) << 4);
    return {{at, at + 16 * FD_K * 2}};
  }
  const int at = part + (first >> 2) * 4096 + ((first >> 1) & 1) * 512 + (g >> 1) * 2048 + ((g & 1) * 4 + (c >> 2)) * 64 + (c & 3) * 8;
  return {{at + ((g & 1) << 5), at + ((~g & 1) << 5)}};
}
// Operand number idx from there on, `part` bytes further.  (Every address is one step from the array it lies in: the
// compiler then still sees which stage it reads, and does not wait for loads into the others.)
template <bool KC, typename F>
__device__ __forceinline__ F fd_frag(const unsigned char* lds, const FdFrom& from, int part, int idx) {
  F r;
  if constexpr (KC) {
    r = *reinterpret_cast<const F*>(lds + (from.at[0] + (part + idx * 16 * FD_K * 2)));
  } else {
    const int at = from.at[idx & 1] + (part + (idx >> 2) * 4096 + ((idx >> 1) & 1) * 512);
    typedef __attribute__((address_space(3))) s16x4 lds_t;
    s16x4 half[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(lds + at)), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(lds + (at + 1024)))};
    __builtin_memcpy(&r, half, 16);
  }
  return r;
}

// The order of a step's instructions: its LDS reads spread evenly between its matrix instructions.
template <int DONE, int MFMAS, int READS>
__device__ __forceinline__ void fd_schedule() {
  if constexpr (DONE < READS) {
    constexpr int upto = (DONE + 1) * MFMAS / READS, from = DONE * MFMAS / READS;
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    if constexpr (upto > from) __builtin_amdgcn_sched_group_barrier(0x8, upto - from, 0);
    fd_schedule<DONE + 1, MFMAS, READS>();
  }
}

// BM x BN of the result (two products: BM x BN/2 of each) per workgroup of WM x WN wavefronts.
template <typename T, bool A_KC, bool B_KC, bool DUAL, int EPI, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64, 2) void ff_direct_kernel(FfProduct p) {
  using F = typename FfFrag<T>::type;
  constexpr int THREADS = WM * WN * 64;
  constexpr int AW = BM < 128 ? BM : 128, AP = BM / AW;        // A's parts: rows in one, how many
  constexpr int BW = BN / 2;                                   // B: two parts
  constexpr int RI = BM / WM / 16, CJ = BN / WN / 32;          // 16 x 16 tiles of a wavefront: down, across in each half
  constexpr int STAGE = (BM + BN) * FD_K * 2;
  __shared__ __align__(16) unsigned char lds0[STAGE], lds1[STAGE], lds2[STAGE], lds3[STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  constexpr bool SUMS_CHANNELS = A_KC && B_KC;                 // dX: K runs over the hidden channels
  const long long N = p.kept && !SUMS_CHANNELS ? *p.kept : p.N;
  const long long K = p.kept && SUMS_CHANNELS ? *p.kept : p.K;
  constexpr int COLS = DUAL ? BW : BN;
  long long row0, col0;
  if (!ff_tile<BM, COLS>(p, N, &row0, &col0)) return;
  const int ksteps = (int)((K + FD_K - 1) / FD_K), all = ksteps * p.segs;
  const int first = (int)((long long)all * p.share / p.splits), last = (int)((long long)all * (p.share + 1) / p.splits);

  FdPart<A_KC, AW, THREADS> pa[AP];
  FdPart<B_KC, BW, THREADS> pb[2];
#pragma unroll
  for (int i = 0; i < AP; i++) pa[i].plan(tid, p.lda, p.M - (row0 + i * AW));
#pragma unroll
  for (int i = 0; i < 2; i++) pb[i].plan(tid, p.ldb, N - (col0 + (DUAL ? 0 : i * BW)));

  auto load = [&](int step, unsigned char* lds) {
    const int seg = step >= ksteps;
    const long long k0 = (long long)(step - (seg ? ksteps : 0)) * FD_K, left = step < last ? K - k0 : 0;
    const T* A = static_cast<const T*>(seg ? p.A1 : p.A0);
#pragma unroll
    for (int i = 0; i < AP; i++) {
      const long long r = row0 + i * AW;
      pa[i].load(A + (A_KC ? r * p.lda + k0 : k0 * p.lda + r), p.lda, left, lds + i * AW * FD_K * 2, wave);
    }
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const T* B = static_cast<const T*>((DUAL ? i : seg) ? p.B1 : p.B0);
      const long long c = col0 + (DUAL ? 0 : i * BW);
      pb[i].load(B + (B_KC ? c * p.ldb + k0 : k0 * p.ldb + c), p.ldb, left, lds + (BM + i * BW) * FD_K * 2, wave);
    }
  };

  f32x4 acc[RI][2 * CJ] = {};
  struct Operands { F a[RI], b[2 * CJ]; };
  const FdFrom from_a = fd_from<A_KC>((wm * RI / (AW / 16)) * AW * FD_K * 2, wm * RI % (AW / 16), lane);
  const FdFrom from_b = fd_from<B_KC>(BM * FD_K * 2, wn * CJ, lane);
  auto read = [&](const unsigned char* lds) {
    Operands o;
    // (B's operands, which live until the tile's last instruction, in the middle of A's, which free their registers in turn)
#pragma unroll
    for (int i = 0; i < RI / 2; i++) o.a[i] = fd_frag<A_KC, F>(lds, from_a, 0, i);
#pragma unroll
    for (int j = 0; j < 2 * CJ; j++) o.b[j] = fd_frag<B_KC, F>(lds, from_b, (j / CJ) * BW * FD_K * 2, j % CJ);
#pragma unroll
    for (int i = RI / 2; i < RI; i++) o.a[i] = fd_frag<A_KC, F>(lds, from_a, 0, i);
    return o;
  };
  auto multiply = [&](const Operands& o) {
#pragma unroll
    for (int i = 0; i < RI; i++)
#pragma unroll
      for (int j = 0; j < 2 * CJ; j++) acc[i][j] = ff_mfma(o.b[j], o.a[i], acc[i][j]);
  };
  // Behind this all loads but those of the last `tiles` tiles are in LDS, and nobody reads what was read before.
  constexpr int LOADS = (AW * AP + BN) * FD_K / 8 / THREADS;
  auto meet = [&]() {
    asm volatile("" ::: "memory");
    // vmcnt((FD_STAGES - 2) LOADS) lgkmcnt(0)
    constexpr int v = (FD_STAGES - 2) * LOADS;
    __builtin_amdgcn_s_waitcnt(0x0070 | (v & 15) | ((v >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  constexpr int READS = RI * (A_KC ? 1 : 2) + 2 * CJ * (B_KC ? 1 : 2);
  Operands even, odd;
  auto step_of = [&](int step, unsigned char* here, unsigned char* next, const Operands& now, Operands& then) {
    meet();
    load(step + FD_STAGES, here);
    then = read(next);
    multiply(now);
    fd_schedule<0, RI * 2 * CJ, READS>();
  };

  // (a load past the last step asks for nothing and brings zeros)
  load(first, lds0);
  load(first + 1, lds1);
  load(first + 2, lds2);
  meet();
  even = read(lds0);
  load(first + 3, lds3);
  int step = first;
  for (; step + 3 < last; step += 4) {
    step_of(step, lds0, lds1, even, odd);
    step_of(step + 1, lds1, lds2, odd, even);
    step_of(step + 2, lds2, lds3, even, odd);
    step_of(step + 3, lds3, lds0, odd, even);
  }
  if (step < last) step_of(step, lds0, lds1, even, odd);
  if (step + 1 < last) step_of(step + 1, lds1, lds2, odd, even);
  if (step + 2 < last) step_of(step + 2, lds2, lds3, even, odd);
  // no load may be under way when the workgroup's LDS is given to another
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);            // vmcnt(0) lgkmcnt(0)

  const long long my_row = row0 + wm * RI * 16 + (lane & 15), my_col = col0 + wn * CJ * 16 + (lane >> 4) * 4;
  FfVec4<T> d[RI][CJ] = {};
  if constexpr (EPI == FF_GRAD) {
#pragma unroll
    for (int i = 0; i < RI; i++)
#pragma unroll
      for (int j = 0; j < CJ; j++)
        if (my_row + i * 16 < p.M && my_col + j * 16 < N) d[i][j] = ff_upstream<T>(p, my_row + i * 16, my_col + j * 16, N);
  }
#pragma unroll
  for (int i = 0; i < RI; i++) {
    const long long row = my_row + i * 16;
    if (row >= p.M) continue;
#pragma unroll
    for (int j = 0; j < CJ; j++) {
      const long long col = my_col + j * 16;
      if constexpr (DUAL) {
        if (col < N) ff_finish<EPI, true, T>(p, row, col, N, acc[i][j], acc[i][CJ + j], d[i][j]);
      } else {
        if (col < N) ff_finish<EPI, false, T>(p, row, col, N, acc[i][j], f32x4{}, {});
        if (col + BW < N) ff_finish<EPI, false, T>(p, row, col + BW, N, acc[i][CJ + j], f32x4{}, {});
      }
    }
  }
}

}  // namespace mlproj
#endif
