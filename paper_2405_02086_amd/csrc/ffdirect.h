// mlproj: matrix products of the gated feed-forward block for 16-bit elements in aligned rows: tiles go from memory
// to LDS without passing through registers.
#ifndef MLPROJ_FFDIRECT_H
#define MLPROJ_FFDIRECT_H

#include "ffcommon.h"
#include "ffstaged.h"

namespace mlproj {

// ------------------------------------------------------------------ tiles straight into LDS
// A tile is FD_K = 64 deep; two of them lie in LDS, one being computed while the loads of the next one, 16 bytes
// per lane and straight into LDS, are under way.  One barrier per step: behind it the step's tile is complete
// and everybody has left the other one.
//
// The tile is cut into parts of 64 or 128 rows (of A), columns (of B).  A part whose K runs along memory rows is [row][64]:
// 128 bytes per row, the 16-byte pieces permuted by row % 8.  A part whose memory rows are the K index is
// [64][columns], read with the transposing load, the 32-byte pieces permuted so that the eight rows a half
// wavefront reads lie in different banks.  Lanes write LDS in order, so the permutation is applied to the
// addresses they load from.
//
// Requires (checked by ff_direct): 16-byte aligned operands, rows and K (or the row length) in whole 16-byte pieces.
// Outside the matrix a lane's offset lies past the end of the buffer resource and the load returns zeros.
constexpr int FD_K = 64;
constexpr unsigned FD_OUT = 0xfffffff0u;         // past any buffer

typedef __attribute__((address_space(3))) void fd_lds_t;

// The swizzle of a part read with the transposing load: which 32-byte piece holds piece 0 of memory row k.
template <int W>
__device__ __forceinline__ int fd_turn(int k) {
  return W == 128 ? (k & 3) | (((k >> 3) & 1) << 2) : ((k >> 1) & 1) | (((k >> 3) & 1) << 1);
}

// Loads of one part.  offset[i]: where lane's i-th piece lies from the part's first element of the step.
template <bool KC, int W, int THREADS>
struct FdPart {
  static constexpr int LOADS = W * 8 / THREADS;
  unsigned offset[LOADS];
  unsigned k_of[LOADS];                          // KC: first K index of the piece within the step

  // `there`: rows (KC) or columns that exist from the part's first one on
  __device__ __forceinline__ void plan(int tid, long long ld, long long there) {
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const int p = tid + i * THREADS;
      if constexpr (KC) {
        const int row = p >> 3, piece = (p & 7) ^ (row & 7);
        offset[i] = row < there ? (unsigned)(row * ld * 2 + piece * 16) : FD_OUT;
        k_of[i] = piece * 8;
      } else {
        constexpr int PIECES = W / 8;
        const int k = p / PIECES, pos = p % PIECES;
        const int col = (((pos >> 1) ^ fd_turn<W>(k)) * 2 + (pos & 1)) * 8;
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

// Sixteen rows (columns) x 32 along K of the part at lds + part, as a lane's operand.  (Every address is one step
// from the array it lies in: the compiler then still sees which of the two halves of the buffer it reads, and does not wait for
// loads into the other one.)
template <bool KC, int W, typename F>
__device__ __forceinline__ F fd_frag(const unsigned char* lds, int part, int idx, int kk, int lane) {
  F r;
  const int g = lane >> 4, c = lane & 15;
  if constexpr (KC) {
    const int at = part + (idx * 16 + c) * 128 + (((kk * 4 + g) ^ (c & 7)) << 4);
    r = *reinterpret_cast<const F*>(lds + at);
  } else {
    const int k = kk * 32 + 8 * g + (c >> 2);
    const int at = part + k * (W * 2) + ((idx ^ fd_turn<W>(8 * g + (c >> 2))) << 5) + ((c & 3) << 3);
    typedef __attribute__((address_space(3))) s16x4 lds_t;
    // (four rows further down the turn is the same: it does not look at bit 2)
    s16x4 half[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(lds + at)), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(lds + (at + 4 * W * 2)))};
    __builtin_memcpy(&r, half, 16);
  }
  return r;
}

// The tile of a workgroup.  Workgroups are dealt to the 8 XCDs in turn; each XCD takes a run of consecutive tiles, and
// tiles are numbered down FD_BAND tile rows before the next column, so that what runs on an XCD at one time shares rows of A
// and columns of B in its L2.
constexpr int FD_BAND = 4;
__device__ __forceinline__ bool fd_tile(long long tiles_m, long long tiles_n, long long* tm, long long* tn) {
  const long long all = tiles_m * tiles_n, id = blockIdx.x;
  if (id >= all) return false;
  const long long xcd = id & 7, each = all >> 3, more = all & 7;
  const long long v = xcd * each + (xcd < more ? xcd : more) + (id >> 3);
  const long long band = v / (FD_BAND * tiles_n), in = v % (FD_BAND * tiles_n);
  const long long rows = tiles_m - band * FD_BAND < FD_BAND ? tiles_m - band * FD_BAND : FD_BAND;
  *tm = band * FD_BAND + in % rows;
  *tn = in / rows;
  return true;
}

// The order of a step's instructions from group G on (see compute): the group's matrix instructions, then the reads
// of the group two further on, and, in the last groups of the first half, one of B's operands of the second half.
template <int G, int GROUPS, int PER, int READ_A, int READ_B, int LATE, int HALF>
__device__ __forceinline__ void fd_schedule() {
  if constexpr (G < GROUPS) {
    __builtin_amdgcn_sched_group_barrier(0x8, PER, 0);
    constexpr int reads = (G + 2 < GROUPS ? READ_A : 0) + (G >= LATE && G < HALF ? READ_B * ((PER + HALF - LATE - 1) / (HALF - LATE)) : 0);
    if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
    fd_schedule<G + 1, GROUPS, PER, READ_A, READ_B, LATE, HALF>();
  }
}

// BM x BN of the result (two products: BM x BN/2 of each) per workgroup of WM x WN wavefronts.
template <typename T, bool A_KC, bool B_KC, bool DUAL, int EPI, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void ff_direct_kernel(FfProduct p) {
  using F = typename FfFrag<T>::type;
  constexpr int THREADS = WM * WN * 64;
  constexpr int AW = BM < 128 ? BM : 128, AP = BM / AW;        // A's parts: rows in one, how many
  constexpr int BW = BN / 2;                                   // B: two parts
  constexpr int RI = BM / WM / 16, CJ = BN / WN / 32;          // 16 x 16 tiles of a wavefront: down, across in each half
  constexpr int STAGE = (BM + BN) * FD_K * 2;
  __shared__ __align__(16) unsigned char lds0[STAGE], lds1[STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  constexpr bool SUMS_CHANNELS = A_KC && B_KC;                 // dX: K runs over the hidden channels
  const long long N = p.kept && !SUMS_CHANNELS ? *p.kept : p.N;
  const long long K = p.kept && SUMS_CHANNELS ? *p.kept : p.K;
  constexpr int COLS = DUAL ? BW : BN;
  long long tm, tn;
  if (!fd_tile((p.M + BM - 1) / BM, (N + COLS - 1) / COLS, &tm, &tn)) return;
  const long long row0 = tm * BM, col0 = tn * COLS;
  const int ksteps = (int)((K + FD_K - 1) / FD_K), all = ksteps * p.segs;
  const int first = (int)((long long)all * blockIdx.y / p.splits), last = (int)((long long)all * (blockIdx.y + 1) / p.splits);

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
  // A step: 2 RI groups of 2 CJ matrix instructions, one per 16 rows and half of K.  The operands of a group are
  // read two groups ahead, and those of B's second half during the first one; left to itself the compiler reads everything
  // at once and spills (KS operands: 102 to 164 registers).
  auto compute = [&](const unsigned char* lds) {
    constexpr int READ_A = A_KC ? 1 : 2, READ_B = B_KC ? 1 : 2;
    F a[FD_K / 32][RI], b[FD_K / 32][2 * CJ];
#pragma unroll
    for (int kk = 0; kk < FD_K / 32; kk++) {
#pragma unroll
      for (int j = 0; j < 2 * CJ; j++)
        b[kk][j] = fd_frag<B_KC, BW, F>(lds, (BM + (j / CJ) * BW) * FD_K * 2, wn * CJ + j % CJ, kk, lane);
#pragma unroll
      for (int i = 0; i < RI; i++) {
        const int r = wm * RI + i;
        a[kk][i] = fd_frag<A_KC, AW, F>(lds, (r / (AW / 16)) * AW * FD_K * 2, r % (AW / 16), kk, lane);
      }
#pragma unroll
      for (int i = 0; i < RI; i++)
#pragma unroll
        for (int j = 0; j < 2 * CJ; j++) acc[i][j] = ff_mfma(b[kk][j], a[kk][i], acc[i][j]);
    }
    constexpr int LATE = RI >= 2 * CJ ? RI - 2 * CJ : 0;
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * CJ * READ_B + 2 * READ_A, 0);
    fd_schedule<0, 2 * RI, 2 * CJ, READ_A, READ_B, LATE, RI>();
  };
  // behind this: the loads of the step are in LDS, and nobody reads the other half any more
  auto meet = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);          // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // (a load past the last step asks for nothing and brings zeros)
  load(first, lds0);
  int step = first;
  for (; step + 1 < last; step += 2) {
    meet();
    load(step + 1, lds1);
    compute(lds0);
    meet();
    load(step + 2, lds0);
    compute(lds1);
  }
  if (step < last) {
    meet();
    compute(lds0);
  }
  // no load may be under way when the workgroup's LDS is given to another
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);

#pragma unroll
  for (int i = 0; i < RI; i++) {
    const long long row = row0 + (wm * RI + i) * 16 + (lane & 15);
    if (row >= p.M) continue;
#pragma unroll
    for (int j = 0; j < CJ; j++) {
      const long long col = col0 + (wn * CJ + j) * 16 + (lane >> 4) * 4;
      if constexpr (DUAL) {
        if (col < N) ff_finish<EPI, true, T>(p, row, col, N, acc[i][j], acc[i][CJ + j]);
      } else {
        if (col < N) ff_finish<EPI, false, T>(p, row, col, N, acc[i][j], f32x4{});
        if (col + BW < N) ff_finish<EPI, false, T>(p, row, col + BW, N, acc[i][CJ + j], f32x4{});
      }
    }
  }
}

}  // namespace mlproj
#endif
