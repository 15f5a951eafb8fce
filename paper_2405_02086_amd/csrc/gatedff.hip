// mlproj: the gated feed-forward block whose hidden channels the projection prunes, forward and backward:
// argument checks, plans, copies of operands and the C ABI.  The products' kernels: ffdirect.h (16-bit elements, tiles straight
// into LDS), ffstaged.h (fp32 and other alignments; joins), ffskinny.h (few fp32 tokens), what they share: ffcommon.h;
// moving kept channels: ffcompact.h.
#include "ffcommon.h"
#include "ffcompact.h"
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
  double tile[4], crowd;       // by epilogue; more by this share for each further workgroup
  double turn(bool dual, int epi, long long steps, long long on_unit) const {
    return steps * step[dual][on_unit - 1] + tile[epi] * (1.0 + crowd * (on_unit - 1));
  }
};
static FfPlan ff_plan(long long M, long long N, long long steps, bool dual, int epi, bool direct, int es) {
  static const FfKind tile256 = {256, 256, 1, {{0.66}, {0.66}}, {8.2, 8.5, 18.6, 2.3}, 0.0};
  static const FfKind tile128 = {128, 128, 2, {{0.30, 0.59}, {0.24, 0.50}}, {1.9, 1.7, 4.1, 0.5}, 1.9};
  static const FfKind tile64 = {64, 128, 3, {{0.18, 0.42, 0.70}, {0.16, 0.44, 0.57}}, {1.1, 0.9, 1.7, 0.5}, 1.4};
  static const FfKind staged = {128, 128, 3, {{0.81, 1.27, 0.85}, {1.46, 1.40, 1.33}}, {3.0, 0.5, 1.7, 0.1}, 1.9};
  static const FfKind staged32 = {128, 128, 2, {{3.1, 3.1}, {3.1, 3.1}}, {2.0, 3.0, 5.0, 2.0}, 0.0};
  constexpr double LAUNCH = 3.6;
  if (es == 4 && (epi == FF_FWD || epi == FF_GRAD) && M <= FK_TOKENS) {
    // shares until there are two workgroups per compute unit or a wavefront has one step left
    int splits = 1;
    const long long groups = ff_cdiv(N, FK_COLS) * ff_cdiv(M, 16);
    while (groups * splits < 512 && steps > FK_WAVES * splits && splits < 64) splits *= 2;
    return {3, splits, LAUNCH + 32.0 * steps * N * 2 * 4 / 4.9e6, false};      // the weights, once
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

// What a call's products take, all of them, by the plan.
static double ff_products_us(int es, long long tokens, long long n, long long m, bool backward, bool direct) {
  double us = ff_plan(tokens, m, ff_steps(n, 1), true, backward ? FF_GRAD : FF_FWD, direct, es).us;
  if (backward) us += ff_plan(tokens, n, ff_steps(m, 2), false, FF_STORE, direct, es).us + ff_plan(n, m, ff_steps(tokens, 1), true, FF_STORE, direct, es).us;
  return us;
}
// Whether 16-bit operands whose rows are not in whole 16-byte pieces are copied into rows that are (ff_pad_kernel), for
// the direct tiles: where that is cheaper than the staged tiles by the plan.  Copies go at 4 TB/s, read and written.
static bool ff_pads(int es, long long tokens, long long n, long long m, bool backward, bool masked) {
  if (es != 2 || (n % 8 == 0 && (m % 8 == 0 || masked))) return false;
  const double elements = (double)tokens * n + (masked ? 0.0 : 2.0 * n * m);
  return ff_products_us(es, tokens, n, m, backward, true) + 5.0 + elements * 2 * es / 4.0e6 < ff_products_us(es, tokens, n, m, backward, false);
}
// Whether a masked call packs its kept channels: where half of its products (the host does not know how many were kept) take
// longer than moving weights, planes and results, and the launches that does.  Otherwise pruned channels are computed
// and replaced by zeros (backward: the weights' too, in a copy).
static bool ff_packs(int es, long long tokens, long long n, long long m, bool backward) {
  const double weights = 2.0 * n * m * es, plane = (double)tokens * m * es;
  const double moves = backward ? 45.0 + (1.5 * weights + 1.5 * plane + 1.5 * weights) / 4.0e6 - (5.0 + 2.0 * weights / 4.0e6)
                                : 28.0 + (1.5 * weights + 2.0 * plane) / 4.0e6;
  return 0.5 * ff_products_us(es, tokens, n, m, backward, es == 2) > moves;
}

// ------------------------------------------------------------------ workspace
struct FfLayout {
  long long ldn;               // row length of a padded X: n in whole 16-byte pieces
  size_t X;                    // padded: a copy of X; the weights' copies take W
  long long ldd;               // row length of packed and intermediate arrays: m in whole 16-byte pieces
  size_t partial;              // shares of sums, of one product at a time
  size_t dG, dU;               // backward: gradients at the pre-activations, tokens x ldd
  size_t position, kept, W[2], in[3], out[3];   // masked: where the channels went; packed weights, inputs and results
  size_t bytes;
  bool pads;
  bool fits;                   // every product's launch has a grid
};
// How a call deals with its mask: it has none, zeros in the epilogue (backward: and in a copy of the weights), packed channels.
enum FfMask { MASK_NONE, MASK_EPILOGUE, MASK_PACK };
FfLayout ff_layout(int es, long long tokens, long long n, long long m, bool backward, FfMask masked) {
  const bool packed = masked == MASK_PACK, cleaned = masked == MASK_EPILOGUE && backward;
  FfLayout L{};
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += ff_up(bytes);
    return at;
  };
  L.ldd = ff_cdiv(m, 8) * 8;
  L.ldn = ff_cdiv(n, 8) * 8;
  // (the packed channels' products run over ldd of them)
  const long long widest = packed ? L.ldd : m;
  L.fits = true;
  size_t shares = ff_partial_bytes(tokens, widest, n, 1, true, backward ? FF_GRAD : FF_FWD, es, &L.fits);
  if (backward) {
    const size_t x = ff_partial_bytes(tokens, n, widest, 2, false, FF_STORE, es, &L.fits), w = ff_partial_bytes(n, widest, tokens, 1, true, FF_STORE, es, &L.fits);
    shares = shares > x ? shares : x;
    shares = shares > w ? shares : w;
  }
  if (tokens == 0) L.fits = true;      // (no product is launched)
  L.partial = take(shares);
  const size_t plane = (size_t)tokens * L.ldd * es, weights = (size_t)n * L.ldd * es;
  if (backward) {
    L.dG = take(plane);
    L.dU = take(plane);
  }
  L.pads = ff_pads(es, tokens, n, m, backward, packed);
  if (L.pads) L.X = take((size_t)tokens * L.ldn * es);
  if (L.pads || packed || cleaned)
    for (size_t& w : L.W) w = take(weights);
  if (packed) {
    L.position = take((size_t)(m + 1) * 4);
    L.kept = take(4);
    if (backward)
      for (size_t& i : L.in) i = take(plane);
    for (int i = 0; i < (backward ? 2 : 3); i++) L.out[i] = take(backward ? weights : plane);
  }
  L.bytes = o + 256;
  return L;
}

static FfMask ff_mask(int es, long long tokens, long long n, long long m, bool backward, bool masked) {
  return !masked ? MASK_NONE : ff_packs(es, tokens, n, m, backward) ? MASK_PACK : MASK_EPILOGUE;
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
      launch(ff_skinny_kernel<EPI>, grid, block, stream, p);
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
  const FfPlan plan = ff_plan(p.M, p.N, ff_steps(p.K, p.segs), DUAL, EPI, ff_direct<A_KC, B_KC, T>(p), sizeof(T));
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

// dG and dU from saved pre-activations.
template <typename T>
__global__ __launch_bounds__(256) void ff_slopes_kernel(FfProduct p) {
  const long long quads = (p.N + 3) / 4, N = p.kept ? *p.kept : p.N;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < quads * p.M; i += (long long)gridDim.x * 256) {
    const long long row = i / quads, col = i % quads * 4;
    if (col >= N) continue;
    f32x4 g = {}, u = {};
    const T* pg = static_cast<const T*>(p.G) + row * p.ldg + col;
    const T* pu = static_cast<const T*>(p.U) + row * p.ldg + col;
    if (col + 4 <= N) {
      g = ff_load4(pg);
      u = ff_load4(pu);
    } else {
      for (int c = 0; c < N - col; c++) { g[c] = (float)pg[c]; u[c] = (float)pu[c]; }
    }
    ff_finish<FF_GRAD, true, T>(p, row, col, N, g, u, ff_upstream<T>(p, row, col, N));
  }
}
// Zeros into what an empty batch leaves.
template <typename T>
__global__ __launch_bounds__(256) void ff_zero_kernel(T* a, T* b, long long rows, long long cols, long long ld) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (long long)gridDim.x * 256)
    a[i / cols * ld + i % cols] = b[i / cols * ld + i % cols] = (T)0.0f;
}

int ff_check(int storage, int act, const mlproj_gated_block* b) {
  if (!b) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16 || act < MLPROJ_ACT_SILU || act > MLPROJ_ACT_RELU) return MLPROJ_ERR_BAD_VARIANT;
  if (b->tokens < 0 || b->n <= 0 || b->m <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (b->tokens > FF_MAX_DIM || b->n > FF_MAX_DIM || b->m > FF_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  if (b->ldx < b->n || b->ldw < b->m) return MLPROJ_ERR_BAD_DIMENSION;
  if (b->ldx > FF_MAX_DIM || b->ldw > FF_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  return MLPROJ_OK;
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

// Matrices to be moved into packed form or out of it, all in one launch.
template <typename T, bool PACK>
struct FfMove {
  FcArrays a{};
  FfMove(long long cols, const int* position, const int* kept) { a.cols = cols; a.position = position; a.kept = kept; }
  void add(const void* from, long long ld_from, void* to, long long ld_to, long long rows) {
    const int i = a.count++;
    a.from[i] = from; a.ld_from[i] = ld_from; a.to[i] = to; a.ld_to[i] = ld_to; a.rows[i] = rows;
  }
  void go(hipStream_t stream) {
    // about four workgroups per compute unit: each reads its columns' places once, for many rows
    const long long segments = ff_cdiv(a.cols, FC_COLS);
    long long most = FC_GROUPS / (segments * a.count);
    if (most < 1) most = 1;
    int groups = 0;
    for (int i = 0; i < a.count; i++) {
      const long long all = ff_cdiv(a.rows[i], FC_ROWS);
      a.groups[i] = (int)(all < most ? all : most);
      groups += a.groups[i];
    }
    mark(stream);
    launch(ff_move_kernel<T, PACK>, dim3((unsigned)ff_cdiv(a.cols, FC_COLS), (unsigned)groups), dim3(256), stream, a);
  }
};

// Copies of matrices in rows of whole 16-byte pieces, filled up with zeros; without `from` only the filling: the pieces
// from the last whole one on.
struct FfPad {
  const void* from[5];
  void* to[5];
  long long ld_from[5], ld_to[5], rows[5], cols[5];
  long long first[5];          // number of the first thread of a matrix
  long long threads;           // of all
  const unsigned char* mask[5];  // columns to be replaced by zeros, or null
  int count;
};
template <typename T>
__global__ __launch_bounds__(256) void ff_pad_kernel(FfPad a) {
  int i = 0;
  for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < a.threads; id += (long long)gridDim.x * 256) {
    while (i + 1 < a.count && id >= a.first[i + 1]) i++;
    const long long pieces = a.from[i] ? a.ld_to[i] / 8 : 1, at = id - a.first[i];
    const long long row = at >> 32 ? at / pieces : (unsigned)at / (unsigned)pieces;
    const long long col = a.from[i] ? (at - row * pieces) * 8 : a.ld_to[i] - 8;
    FfVec8<T> v = {};
    if (a.from[i]) v = ff_load8(static_cast<const T*>(a.from[i]) + row * a.ld_from[i] + col, a.cols[i] - col);
    if (a.mask[i])
#pragma unroll
      for (int j = 0; j < 8; j++)
        if (col + j < a.cols[i] && !a.mask[i][col + j]) v.v[j] = (T)0.0f;
    __builtin_memcpy(static_cast<T*>(a.to[i]) + row * a.ld_to[i] + col, &v, sizeof(v));
  }
}
struct FfPadder {
  FfPad a{};
  void add(const void* from, long long ld_from, void* to, long long ld_to, long long rows, long long cols, const unsigned char* mask = nullptr) {
    const int i = a.count++;
    a.from[i] = from; a.ld_from[i] = ld_from; a.to[i] = to; a.ld_to[i] = ld_to; a.rows[i] = rows; a.cols[i] = cols;
    a.mask[i] = mask;
    a.first[i] = a.threads;
    a.threads += rows * (from ? ld_to / 8 : 1);
  }
  template <typename T>
  void go(hipStream_t stream) {
    if (a.threads == 0) return;
    mark(stream);
    launch(ff_pad_kernel<T>, ff_strided_grid(a.threads), dim3(256), stream, a);
  }
};

// A block's weights and the channels its products run over: the caller's, copies in filled rows, or the kept ones in packed form.
struct FfChannels {
  const void *Wg, *Wu;
  long long ldw, m;            // m: how many there can be
  int *position = nullptr, *kept = nullptr;
  bool filled = false;         // the weights are the workspace's, rows filled up with zeros
};
FfChannels ff_channels(const mlproj_gated_block* b, const FfLayout& L, char* ws, bool pack, hipStream_t stream) {
  FfChannels c{b->Wg, b->Wu, b->ldw, b->m};
  if (!pack) return c;
  c.position = reinterpret_cast<int*>(ws + L.position);
  c.kept = reinterpret_cast<int*>(ws + L.kept);
  mark(stream);
  launch(ff_index_kernel, dim3(1), dim3(FC_THREADS), stream, b->mask, b->m, c.position, c.kept);
  c.Wg = ws + L.W[0]; c.Wu = ws + L.W[1];
  c.ldw = c.m = L.ldd;
  c.filled = true;
  return c;
}

// X, and copies: of X where the plan pads; of the weights where it pads (unless they are packed anyway, or not read), or where
// pruned columns have to be zeros (`clean`).
struct FfInput {
  const void* at;
  long long ld;
  bool filled;
};
template <typename T>
FfInput ff_input(const mlproj_gated_block* b, const FfLayout& L, char* ws, bool pack, bool weights, bool clean, FfChannels& ch, hipStream_t stream) {
  FfInput X{b->X, b->ldx, false};
  FfPadder pad;
  if (L.pads && b->n % 8) {
    pad.add(b->X, b->ldx, ws + L.X, L.ldn, b->tokens, b->n);
    X = {ws + L.X, L.ldn, true};
  }
  if (!pack && weights && (L.pads || clean)) {
    pad.add(b->Wg, b->ldw, ws + L.W[0], L.ldd, b->n, b->m, clean ? b->mask : nullptr);
    pad.add(b->Wu, b->ldw, ws + L.W[1], L.ldd, b->n, b->m, clean ? b->mask : nullptr);
    ch.Wg = ws + L.W[0]; ch.Wu = ws + L.W[1]; ch.ldw = L.ldd; ch.filled = true;
    if (L.dU && b->m % 8) {      // dG and dU are summed over as well: whole pieces there too
      pad.add(nullptr, 0, ws + L.dG, L.ldd, b->tokens, 0);
      pad.add(nullptr, 0, ws + L.dU, L.ldd, b->tokens, 0);
    }
  }
  pad.go<T>(stream);
  return X;
}

template <typename T>
int run_forward(int act, const mlproj_gated_block* b, void* H, long long ldh, void* G, void* U, long long ldg,
                void* workspace, hipStream_t stream) {
  const FfMask masked = ff_mask(sizeof(T), b->tokens, b->n, b->m, false, b->mask != nullptr);
  const bool pack = masked == MASK_PACK;
  const FfLayout L = ff_layout(sizeof(T), b->tokens, b->n, b->m, false, masked);
  char* ws = static_cast<char*>(workspace);
  FfChannels ch = ff_channels(b, L, ws, pack, stream);
  if (pack) {
    FfMove<T, true> in(b->m, ch.position, ch.kept);
    in.add(b->Wg, b->ldw, ws + L.W[0], L.ldd, b->n);
    in.add(b->Wu, b->ldw, ws + L.W[1], L.ldd, b->n);
    in.go(stream);
  }
  const FfInput X = ff_input<T>(b, L, ws, pack, true, false, ch, stream);
  FfProduct p{};
  p.segs = 1; p.act = act;
  p.A0 = X.at; p.lda = X.ld; p.a_filled = X.filled;
  p.B0 = ch.Wg; p.B1 = ch.Wu; p.ldb = ch.ldw; p.b_filled = ch.filled;
  p.M = b->tokens; p.N = ch.m; p.K = b->n;
  p.C0 = H; p.ldc = ldh;
  p.G = G; p.U = U; p.ldg = ldg;
  void* packed[3] = {ws + L.out[0], ws + L.out[1], ws + L.out[2]};
  if (pack) {
    p.kept = ch.kept;
    p.C0 = packed[0]; p.ldc = L.ldd;
    if (G) { p.G = packed[1]; p.U = packed[2]; p.ldg = L.ldd; }
  } else {
    p.keep = b->mask;
  }
  ff_product<T, true, false, true, FF_FWD>(p, ws + L.partial, stream);
  if (pack) {
    FfMove<T, false> out(b->m, ch.position, ch.kept);
    out.add(packed[0], L.ldd, H, ldh, b->tokens);
    if (G) {
      out.add(packed[1], L.ldd, G, ldg, b->tokens);
      out.add(packed[2], L.ldd, U, ldg, b->tokens);
    }
    out.go(stream);
  }
  mark(stream);
  return launch_status();
}

template <typename T>
int run_backward(int act, const mlproj_gated_block* b, const void* dH, long long ldh, const void* G, const void* U, long long ldg,
                 void* dX, long long lddx, void* dWg, void* dWu, long long lddw, void* workspace, hipStream_t stream) {
  if (b->tokens == 0) {
    if (dWg) {
      mark(stream);
      launch(ff_zero_kernel<T>, ff_strided_grid(b->n * b->m), dim3(256), stream, static_cast<T*>(dWg), static_cast<T*>(dWu), b->n, b->m, lddw);
    }
    mark(stream);
    return launch_status();
  }
  const FfMask masked = ff_mask(sizeof(T), b->tokens, b->n, b->m, true, b->mask != nullptr);
  const bool pack = masked == MASK_PACK, clean = masked == MASK_EPILOGUE && dX;
  const FfLayout L = ff_layout(sizeof(T), b->tokens, b->n, b->m, true, masked);
  char* ws = static_cast<char*>(workspace);
  FfChannels ch = ff_channels(b, L, ws, pack, stream);
  if (pack) {
    // what runs over the channels: the weights where a product reads them, dH and the saved pre-activations
    void *W[2] = {ws + L.W[0], ws + L.W[1]}, *in[3] = {ws + L.in[0], ws + L.in[1], ws + L.in[2]};
    FfMove<T, true> weights(b->m, ch.position, ch.kept), planes(b->m, ch.position, ch.kept);
    if (dX || !G) {
      weights.add(b->Wg, b->ldw, W[0], L.ldd, b->n);
      weights.add(b->Wu, b->ldw, W[1], L.ldd, b->n);
      weights.go(stream);
    }
    planes.add(dH, ldh, in[0], L.ldd, b->tokens);
    if (G) {
      planes.add(G, ldg, in[1], L.ldd, b->tokens);
      planes.add(U, ldg, in[2], L.ldd, b->tokens);
      G = in[1]; U = in[2]; ldg = L.ldd;
    }
    planes.go(stream);
    dH = in[0]; ldh = L.ldd;
  }
  const FfInput X = ff_input<T>(b, L, ws, pack, dX || !G, clean, ch, stream);
  T *dG = reinterpret_cast<T*>(ws + L.dG), *dU = reinterpret_cast<T*>(ws + L.dU);
  {
    FfProduct p{};
    p.segs = 1; p.act = act;
    p.M = b->tokens; p.N = ch.m; p.K = b->n;
    p.C0 = dG; p.C1 = dU; p.ldc = L.ldd;
    p.dH = dH; p.ldh = ldh;
    p.kept = ch.kept;
    p.keep = pack ? nullptr : b->mask;
    if (G) {
      p.G = const_cast<void*>(G); p.U = const_cast<void*>(U); p.ldg = ldg;
      mark(stream);
      launch(ff_slopes_kernel<T>, ff_strided_grid(ff_cdiv(ch.m, 4) * b->tokens), dim3(256), stream, p);
    } else {
      p.A0 = X.at; p.lda = X.ld; p.a_filled = X.filled;
      p.B0 = ch.Wg; p.B1 = ch.Wu; p.ldb = ch.ldw; p.b_filled = ch.filled;
      ff_product<T, true, false, true, FF_GRAD>(p, ws + L.partial, stream);
    }
  }
  if (dX) {
    FfProduct p{};
    p.segs = 2;
    p.A0 = dG; p.A1 = dU; p.lda = L.ldd; p.a_filled = ch.filled;
    p.B0 = ch.Wg; p.B1 = ch.Wu; p.ldb = ch.ldw; p.b_filled = ch.filled;
    p.M = b->tokens; p.N = b->n; p.K = ch.m;
    p.C0 = dX; p.ldc = lddx;
    p.kept = ch.kept;
    ff_product<T, true, true, false, FF_STORE>(p, ws + L.partial, stream);
  }
  if (dWg) {
    void* packed[2] = {ws + L.out[0], ws + L.out[1]};
    FfProduct p{};
    p.segs = 1;
    p.A0 = X.at; p.lda = X.ld; p.a_filled = X.filled;
    p.B0 = dG; p.B1 = dU; p.ldb = L.ldd; p.b_filled = true;
    p.M = b->n; p.N = ch.m; p.K = b->tokens;
    p.keep = pack ? nullptr : b->mask;
    p.C0 = pack ? packed[0] : dWg; p.C1 = pack ? packed[1] : dWu; p.ldc = pack ? L.ldd : lddw;
    p.kept = ch.kept;
    ff_product<T, false, false, true, FF_STORE>(p, ws + L.partial, stream);
    if (pack) {
      FfMove<T, false> out(b->m, ch.position, ch.kept);
      out.add(packed[0], L.ldd, dWg, lddw, b->n);
      out.add(packed[1], L.ldd, dWu, lddw, b->n);
      out.go(stream);
    }
  }
  mark(stream);
  return launch_status();
}

int ff_workspace(int storage, long long tokens, long long n, long long m, int backward, int masked, size_t* out) {
  if (!out) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16) return MLPROJ_ERR_BAD_VARIANT;
  if (tokens < 0 || n <= 0 || m <= 0 || (backward | 1) != 1 || (masked | 1) != 1) return MLPROJ_ERR_BAD_DIMENSION;
  if (tokens > FF_MAX_DIM || n > FF_MAX_DIM || m > FF_MAX_DIM || tokens * m > (1LL << 38) || tokens * n > (1LL << 38) || n * m > (1LL << 38)) return MLPROJ_ERR_TOO_LARGE;
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const FfLayout plain = ff_layout(es, tokens, n, m, backward != 0, MASK_NONE);
  if (!plain.fits) return MLPROJ_ERR_TOO_LARGE;
  *out = plain.bytes;
  if (masked) {      // serves calls without a mask as well
    const FfLayout with = ff_layout(es, tokens, n, m, backward != 0, ff_mask(es, tokens, n, m, backward != 0, true));
    if (!with.fits) return MLPROJ_ERR_TOO_LARGE;
    *out = *out > with.bytes ? *out : with.bytes;
  }
  return MLPROJ_OK;
}

}  // namespace
}  // namespace mlproj

using namespace mlproj;

extern "C" {

int mlproj_gated_ff_workspace_bytes(int storage, long long tokens, long long n, long long m, int backward, int masked,
                                    size_t* bytes_out) {
  return ff_workspace(storage, tokens, n, m, backward, masked, bytes_out);
}

int mlproj_gated_ff_route(int storage, int product, long long tokens, long long n, long long m) {
  size_t bytes;
  FF_TRY(ff_workspace(storage, tokens, n, m, 1, 1, &bytes));
  if (product < 0 || product > 3) return MLPROJ_ERR_BAD_VARIANT;
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool direct = es == 2, backward = product > 0;
  FfPlan plan;
  if (product < 2) plan = ff_plan(tokens, m, ff_steps(n, 1), true, backward ? FF_GRAD : FF_FWD, direct, es);
  else if (product == 2) plan = ff_plan(tokens, n, ff_steps(m, 2), false, FF_STORE, direct, es);
  else plan = ff_plan(n, m, ff_steps(tokens, 1), true, FF_STORE, direct, es);
  const bool low = plan.kind == 4;
  return (low ? 1 : plan.kind) + 16 * ff_packs(es, tokens, n, m, backward) + 32 * plan.parts + 64 * low + 256 * plan.splits;
}

int gated_ff_forward(int storage, int activation, const mlproj_gated_block* b, void* H, long long ldh, void* G, void* U,
                     long long ldg, void* workspace, size_t workspace_bytes, void* stream) {
  FF_TRY(ff_check(storage, activation, b));
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool some = b->tokens > 0;
  size_t need;
  FF_TRY(ff_workspace(storage, b->tokens, b->n, b->m, 0, b->mask != nullptr, &need));
  FF_TRY(ff_check_array(b->X, some, b->n, b->ldx, es));
  FF_TRY(ff_check_array(b->Wg, some, b->m, b->ldw, es));
  FF_TRY(ff_check_array(b->Wu, some, b->m, b->ldw, es));
  FF_TRY(ff_check_array(H, some, b->m, ldh, es));
  FF_TRY(ff_check_array(G, U != nullptr, b->m, ldg, es));
  FF_TRY(ff_check_array(U, G != nullptr, b->m, ldg, es));
  FF_TRY(ff_check_workspace(workspace, workspace_bytes, need));
  if (!some) return MLPROJ_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return run_forward<float>(activation, b, H, ldh, G, U, ldg, workspace, s);
  if (storage == MLPROJ_STORE_BF16) return run_forward<bf16_t>(activation, b, H, ldh, G, U, ldg, workspace, s);
  return run_forward<f16_t>(activation, b, H, ldh, G, U, ldg, workspace, s);
}

int gated_ff_backward(int storage, int activation, const mlproj_gated_block* b, const void* dH, long long ldh, const void* G,
                      const void* U, long long ldg, void* dX, long long lddx, void* dWg, void* dWu, long long lddw,
                      void* workspace, size_t workspace_bytes, void* stream) {
  FF_TRY(ff_check(storage, activation, b));
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool some = b->tokens > 0;
  size_t need;
  FF_TRY(ff_workspace(storage, b->tokens, b->n, b->m, 1, b->mask != nullptr, &need));
  FF_TRY(ff_check_array(b->X, some, b->n, b->ldx, es));
  FF_TRY(ff_check_array(b->Wg, some, b->m, b->ldw, es));
  FF_TRY(ff_check_array(b->Wu, some, b->m, b->ldw, es));
  FF_TRY(ff_check_array(dH, some, b->m, ldh, es));
  FF_TRY(ff_check_array(G, U != nullptr && some, b->m, ldg, es));
  FF_TRY(ff_check_array(U, G != nullptr && some, b->m, ldg, es));
  FF_TRY(ff_check_array(dX, false, b->n, lddx, es));
  FF_TRY(ff_check_array(dWg, dWu != nullptr, b->m, lddw, es));
  FF_TRY(ff_check_array(dWu, dWg != nullptr, b->m, lddw, es));
  FF_TRY(ff_check_workspace(workspace, workspace_bytes, need));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return run_backward<float>(activation, b, dH, ldh, G, U, ldg, dX, lddx, dWg, dWu, lddw, workspace, s);
  if (storage == MLPROJ_STORE_BF16) return run_backward<bf16_t>(activation, b, dH, ldh, G, U, ldg, dX, lddx, dWg, dWu, lddw, workspace, s);
  return run_backward<f16_t>(activation, b, dH, ldh, G, U, ldg, dX, lddx, dWg, dWu, lddw, workspace, s);
}

}  // extern "C"
