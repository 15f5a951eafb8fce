// mlproj: how a matrix product of the block's operators is planned and launched (tiles, shares of the sum), copies of operands
// in aligned rows, checks of arrays.  Included by one translation unit per operator, which has kernels of its own.
#ifndef MLPROJ_FFPLAN_H
#define MLPROJ_FFPLAN_H

#include "ffcommon.h"
#include "ffdirect.h"
#include "ffskinny.h"
#include "ffstaged.h"
#include "host.h"

namespace mlproj {
namespace {

constexpr long long FF_MAX_DIM = 1LL << 30;
// fp32 forward products of at most this many tokens go without tiles (ffskinny.h).
constexpr long long FK_TOKENS = 32;

static long long ff_cdiv(long long a, long long b) { return (a + b - 1) / b; }
static size_t ff_up(size_t x) { return (x + 255) / 256 * 256; }

// ------------------------------------------------------------------ plan of a product
// Which tiles a product takes and into how many shares its sum is cut: the cheapest by what was measured, which is a
// 32-deep step of a tile by how many workgroups the compute unit holds, a tile beside its steps (more where others
// on the unit want the same), and joining shares.  Fitted to the four products of 59 blocks, 1 x 440 -> 2048 to 8192 x
// 2048 -> 8192, each in every tile and with every number of shares: the plan's choice takes 0.6 % more than the best
// one on average, 14 % at most.  256 x 256 tiles (one workgroup per compute unit) have the fastest steps, 64 x 128 (three)
// fill the chip where there are few tiles: 303 x 256 -> 1272 backward products take 7, 10 and 6 us in them, in 128 x 128
// (two) 10, 12 and 8, in 256 x 256 18, 20 and 16; 4096 x 4096 -> 4096 forward takes 359, 269 and 215 us.
struct FfPlan {
  int kind;      // 0: direct 256 x 256, 1: direct 128 x 128, 2: staged, 3: few tokens, 4: direct 64 x 128
  int splits;
  double us;
  bool parts;    // direct 256: whole turns, and the rest in smaller tiles
};
struct FfKind {
  int rows, cols, places;      // of the tile; workgroups per compute unit
  double step[2][3];           // us; one product or two, workgroups on the unit
  double tile[5], crowd;       // by epilogue; more by this share for each further workgroup
  double turn(bool dual, int epi, long long steps, long long on_unit) const {
    return steps * step[dual][on_unit - 1] + tile[epi] * (1.0 + crowd * (on_unit - 1));
  }
};
static FfPlan ff_plan(long long M, long long N, long long steps, bool dual, int epi, bool direct, int es) {
  static const FfKind tile256 = {256, 256, 1, {{0.66}, {0.66}}, {8.2, 8.5, 18.6, 2.3, 10.0}, 0.0};
  static const FfKind tile128 = {128, 128, 2, {{0.30, 0.59}, {0.24, 0.50}}, {1.9, 1.7, 4.1, 0.5, 2.5}, 1.9};
  static const FfKind tile64 = {64, 128, 3, {{0.18, 0.42, 0.70}, {0.16, 0.44, 0.57}}, {1.1, 0.9, 1.7, 0.5, 1.2}, 1.4};
  static const FfKind staged = {128, 128, 3, {{0.81, 1.27, 0.85}, {1.46, 1.40, 1.33}}, {3.0, 0.5, 1.7, 0.1, 3.0}, 1.9};
  static const FfKind staged32 = {128, 128, 2, {{3.1, 3.1}, {3.1, 3.1}}, {2.0, 3.0, 5.0, 2.0, 3.0}, 0.0};
  constexpr double LAUNCH = 3.6;
  if (es == 4 && (epi == FF_FWD || epi == FF_GRAD || epi == FF_LINEAR) && M <= FK_TOKENS) {
    // shares until there are two workgroups per compute unit or a wavefront has one step left
    int splits = 1;
    const long long groups = ff_cdiv(N, FK_COLS) * ff_cdiv(M, 16);
    while (groups * splits < 512 && steps > FK_WAVES * splits && splits < 64) splits *= 2;
    return {3, splits, LAUNCH + 32.0 * steps * N * (dual ? 2 : 1) * 4 / 4.9e6, false};      // the weights, once
  }
  FfPlan best{2, 1, 1e30, false};
  const double planes = 4.0 * M * N * (dual ? 2 : 1);
  auto consider = [&](int kind, const FfKind& k) {
    const long long tiles = ff_cdiv(M, k.rows) * ff_cdiv(N, dual ? k.cols / 2 : k.cols);
    for (int splits = 1; splits <= 64; splits *= 2) {
      if (splits > 1 && (steps / splits < 2 || planes * splits > 512e6)) break;
      const long long groups = tiles * splits, units = 256 * k.places, rest = groups % units, each = ff_cdiv(steps, splits);
      const int out = splits > 1 ? FF_PARTIAL : epi;
      double us = LAUNCH + (double)(groups / units) * k.turn(dual, out, each, k.places);
      if (rest) us += k.turn(dual, out, each, ff_cdiv(rest, 256));
      if (splits > 1) us += 3.0 + planes * 2 * splits / 5.7e6;
      if (us < best.us) best = {kind, splits, us, false};
    }
    if (kind == 0 && tiles > 256 && ff_in_turns(tiles) < tiles) {
      const long long left = tiles % 256 * 4;
      const double us = 2 * LAUNCH + (double)(tiles / 256) * k.turn(dual, epi, steps, 1) + tile128.turn(dual, epi, steps, ff_cdiv(left, 256));
      if (us < best.us) best = {0, 1, us, true};
    }
  };
  if (direct) {
    consider(0, tile256);
    consider(1, tile128);
    consider(4, tile64);
  } else {
    consider(2, es == 4 ? staged32 : staged);
  }
  return best;
}
static long long ff_steps(long long K, int segs) { return ff_cdiv(K, 32) * segs; }
// Workgroups (along x) of a product's launch and their threads.
struct FfGrid { long long groups; int threads; };
static FfGrid ff_grid(int kind, long long M, long long N, bool dual, int splits) {
  const int half = dual ? 2 : 1;
  switch (kind) {
    case 0: return {ff_cdiv(M, 256) * ff_cdiv(N, 256 / half) * splits, 512};
    case 3: return {ff_cdiv(ff_cdiv(N, FK_COLS), 8) * 8 * ff_cdiv(M, 16), FK_WAVES * 64};      // (shares along y)
    case 4: return {ff_cdiv(M, 64) * ff_cdiv(N, 128 / half) * splits, 256};
    default: return {ff_cdiv(M, 128) * ff_cdiv(N, 128 / half) * splits, 256};                  // 1: direct, 2: staged
  }
}
// A launch has less than 2^32 threads along an axis.
constexpr long long FF_MOST_THREADS = (1LL << 32) - 1;
static size_t ff_partial_bytes(long long M, long long N, long long K, int segs, bool dual, int epi, int es, bool* fits) {
  size_t most = 0;
  for (int direct = 0; direct < 2; direct++) {
    const FfPlan plan = ff_plan(M, N, ff_steps(K, segs), dual, epi, direct, es);
    const FfGrid grid = ff_grid(plan.kind, M, N, dual, plan.splits);
    if ((es == 2 || !direct) && grid.groups > FF_MOST_THREADS / grid.threads) *fits = false;
    const size_t bytes = plan.splits > 1 ? (size_t)plan.splits * (dual ? 2 : 1) * M * (ff_cdiv(N, 4) * 4) * 4 : 0;
    if (bytes > most) most = bytes;
  }
  return most;
}

// ------------------------------------------------------------------ launches
// Whether a product's operands can go straight into LDS: 16-bit elements, rows, starts and row lengths in whole
// 16-byte pieces, and a tile's rows within a buffer resource's 2 GiB.
// (The last piece of a row may reach past the matrix where the rows are the workspace's.  Past K there are zeros.)
template <bool A_KC, bool B_KC, typename T>
bool ff_direct(const FfProduct& p) {
  if (sizeof(T) != 2) return false;
  const long long a_row = p.a_filled ? 0 : A_KC ? p.K : p.M, b_row = p.b_filled ? 0 : B_KC ? p.K : p.N;
  for (const void* q : {p.A0, p.A1, p.B0, p.B1})
    if (!aligned(q, 16)) return false;
  return a_row % 8 == 0 && b_row % 8 == 0 && p.lda % 8 == 0 && p.ldb % 8 == 0 && p.lda < (1 << 22) && p.ldb < (1 << 22) &&
         p.K < (1LL << 31) - 64;
}

template <typename T, bool A_KC, bool B_KC, bool DUAL, int EPI>
void ff_launch(const FfProduct& p, int kind, hipStream_t stream) {
  mark(stream);
  const FfGrid g = ff_grid(kind, p.M, p.N, DUAL, p.splits);
  const dim3 grid(p.part == FF_REST ? 4 * FF_LEFT : (unsigned)g.groups, kind == 3 ? p.splits : 1), block(g.threads);
  if constexpr (sizeof(T) == 4 && A_KC && !B_KC) {
    if (kind == 3) {
      launch(ff_skinny_kernel<EPI, DUAL>, grid, block, stream, p);
      return;
    }
  }
  if constexpr (sizeof(T) == 2) {
    if (kind == 0) {
      launch(ff_direct_kernel<T, A_KC, B_KC, DUAL, EPI, 256, 256, 2, 4>, grid, block, stream, p);
      return;
    }
    if (kind == 4) {
      launch(ff_direct_kernel<T, A_KC, B_KC, DUAL, EPI, 64, 128, 2, 2>, grid, block, stream, p);
      return;
    }
    if (kind == 1) {
      launch(ff_direct_kernel<T, A_KC, B_KC, DUAL, EPI, 128, 128, 2, 2>, grid, block, stream, p);
      return;
    }
  }
  launch(ff_staged_kernel<T, A_KC, B_KC, DUAL, EPI>, grid, block, stream, p);
}
template <typename T, bool A_KC, bool B_KC, bool DUAL, int EPI>
void ff_product(FfProduct p, void* partial, hipStream_t stream) {
  if (p.M == 0) return;
  const FfPlan plan = ff_plan(p.M, p.N, ff_steps(p.K, p.segs), DUAL, EPI == FF_SCALED ? FF_STORE : EPI, ff_direct<A_KC, B_KC, T>(p), sizeof(T));
  p.splits = plan.splits;
  p.partial = static_cast<float*>(partial);
  // (packed channels: how many tiles there will be is not known here, so both launches go out wherever they are many)
  if (plan.kind == 0 && p.splits == 1 && (plan.parts || (p.kept && DUAL && ff_cdiv(p.M, 256) * ff_cdiv(p.N, 128) > 256))) {
    p.part = FF_TURNS;
    ff_launch<T, A_KC, B_KC, DUAL, EPI>(p, 0, stream);
    p.part = FF_REST;
    ff_launch<T, A_KC, B_KC, DUAL, EPI>(p, 1, stream);
    return;
  }
  if (p.splits == 1) {
    ff_launch<T, A_KC, B_KC, DUAL, EPI>(p, plan.kind, stream);
    return;
  }
  ff_launch<T, A_KC, B_KC, DUAL, FF_PARTIAL>(p, plan.kind, stream);
  mark(stream);
  const long long quads = ff_cdiv(p.N, 4) * p.M;
  if (p.splits >= 16) launch(ff_join_kernel<T, DUAL, EPI, 8>, dim3((unsigned)ff_cdiv(quads, 32)), dim3(256), stream, p);
  else launch(ff_join_kernel<T, DUAL, EPI, 1>, dim3((unsigned)ff_cdiv(quads, 256)), dim3(256), stream, p);
}

// Elementwise kernels: at most this many workgroups, which go on in strides of the grid where there is more to do than one
// launch may have threads.
constexpr long long FF_MOST_GROUPS = 1 << 16;
static dim3 ff_strided_grid(long long threads) {
  const long long groups = ff_cdiv(threads, 256);
  return dim3((unsigned)(groups < FF_MOST_GROUPS ? groups : FF_MOST_GROUPS));
}

// An operand or result: present where it has entries, aligned to its elements, rows no longer than their stride.
int ff_check_array(const void* p, bool needed, long long row, long long ld, int es) {
  if (!p) return needed ? MLPROJ_ERR_NULL_POINTER : MLPROJ_OK;
  if (ld < row) return MLPROJ_ERR_BAD_DIMENSION;
  if (ld > FF_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  return aligned(p, es) ? MLPROJ_OK : MLPROJ_ERR_ALIGNMENT;
}
#define FF_TRY(x)                          \
  do {                                     \
    const int st_ = (x);                   \
    if (st_ != MLPROJ_OK) return st_;      \
  } while (0)

int ff_check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws) return MLPROJ_ERR_NULL_POINTER;
  return have >= need && aligned(ws, 256) ? MLPROJ_OK : MLPROJ_ERR_WORKSPACE;
}

// Copies of matrices in rows of whole 16-byte pieces, filled up with zeros; without `from` only the filling: the pieces
// from the last whole one on.
struct FfPad {
  const void* from[5];
  void* to[5];
  long long ld_from[5], ld_to[5], cols[5];
  long long pieces[5], all[5];  // to be written: of a row, of a matrix
  const unsigned char* mask[5];  // columns to be replaced by zeros, or null
  int count;
};
// Bound by HBM where matrices are large, by latency where they are small.  Workgroups along y are the matrices, so that what
// belongs to one is in scalars (looked up by each thread, one piece at a time: 43 us instead of 26 for 4096 x 4099 and 4099 x 4099
// fp16, 12 instead of 9 for 777 x 2731 and 2731 x 1001), and a thread has FF_PAD pieces in flight (four: 28 and 10.6).
constexpr int FF_PAD = 2;
template <typename T>
__global__ __launch_bounds__(256) void ff_pad_kernel(FfPad a) {
  const int i = blockIdx.y;
  const T* from = static_cast<const T*>(a.from[i]);
  const unsigned char* mask = a.mask[i];
  T* to = static_cast<T*>(a.to[i]);
  const long long pieces = a.pieces[i], all = a.all[i], cols = a.cols[i], ld_from = a.ld_from[i], ld_to = a.ld_to[i];
  for (long long first = (long long)blockIdx.x * (256 * FF_PAD); first < all; first += (long long)gridDim.x * (256 * FF_PAD)) {
    FfVec8<T> v[FF_PAD];
    T* out[FF_PAD];
#pragma unroll
    for (int u = 0; u < FF_PAD; u++) {
      const long long at = first + u * 256 + threadIdx.x;
      const long long row = at >> 32 ? at / pieces : (unsigned)at / (unsigned)pieces;
      const long long col = from ? (at - row * pieces) * 8 : ld_to - 8;
      out[u] = at < all ? to + row * ld_to + col : nullptr;
      v[u] = {};
      if (from && at < all) v[u] = ff_load8(from + row * ld_from + col, cols - col);
      if (mask && at < all)
#pragma unroll
        for (int j = 0; j < 8; j++)
          if (col + j < cols && !mask[col + j]) v[u].v[j] = (T)0.0f;
    }
#pragma unroll
    for (int u = 0; u < FF_PAD; u++)
      if (out[u]) __builtin_memcpy(out[u], &v[u], sizeof(v[u]));
  }
}
struct FfPadder {
  FfPad a{};
  long long most = 0;
  void add(const void* from, long long ld_from, void* to, long long ld_to, long long rows, long long cols, const unsigned char* mask = nullptr) {
    const int i = a.count++;
    a.from[i] = from; a.ld_from[i] = ld_from; a.to[i] = to; a.ld_to[i] = ld_to; a.cols[i] = cols;
    a.mask[i] = mask;
    a.pieces[i] = from ? ld_to / 8 : 1;
    a.all[i] = rows * a.pieces[i];
    most = a.all[i] > most ? a.all[i] : most;
  }
  template <typename T>
  void go(hipStream_t stream) {
    if (most == 0) return;
    mark(stream);
    dim3 grid = ff_strided_grid(ff_cdiv(most, FF_PAD));
    grid.y = a.count;
    launch(ff_pad_kernel<T>, grid, dim3(256), stream, a);
  }
};

}  // namespace
}  // namespace mlproj
#endif
