// mlproj: matrices in 8 bits with a power of two per 32 entries: packing, products of 8-bit tokens with 8-bit weights, plan and
// C ABI.  The products' kernels: q8tile.h, q8few.h; rounding: q8.h.
#include "ffcommon.h"
#include "ffplan.h"
#include "q8.h"
#include "q8few.h"
#include "q8tile.h"

namespace mlproj {
namespace {

// ------------------------------------------------------------------ packing
struct Q8Pack {
  const void* A;
  unsigned char *codes, *scales;
  long long lda, ld, lds, rows, n, wide;
};
// Eight entries of a row per thread, a group in four neighbouring lanes.  Bound by HBM.
template <typename T>
__global__ __launch_bounds__(256) void q8_pack_rows_kernel(Q8Pack a) {
  const long long pieces = a.wide / 8, all = a.rows * pieces;
  for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < all; id += (long long)gridDim.x * 256) {
    const long long row = id >> 32 ? id / pieces : (unsigned)id / (unsigned)pieces, at = (id - row * pieces) * 8;
    const FfVec8<T> raw = ff_load8(static_cast<const T*>(a.A) + row * a.lda + at, a.n - at);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (float)raw.v[i];
    unsigned codes[2];
    const unsigned scale = q8_round<8>(v, codes);
    __builtin_memcpy(__builtin_assume_aligned(a.codes + row * a.ld + at, 8), codes, 8);
    if (at % Q8_GROUP == 0) a.scales[row * a.lds + at / Q8_GROUP] = (unsigned char)scale;
  }
}
// By columns: a thread has a column's 128 entries of a block, neighbouring threads neighbouring columns, and writes them as a
// whole row of codes.
template <typename T>
__global__ __launch_bounds__(256) void q8_pack_columns_kernel(Q8Pack a) {
  const long long across = (a.rows + 255) / 256, k0 = blockIdx.x / across * Q8_BLOCK, row = blockIdx.x % across * 256 + threadIdx.x;
  if (row >= a.rows) return;
  unsigned scales = 0;
#pragma unroll 1
  for (int g = 0; g < 4; g++) {
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; i++) {
      const long long k = k0 + g * 32 + i;
      v[i] = k < a.n ? (float)static_cast<const T*>(a.A)[k * a.lda + row] : 0.0f;
    }
    unsigned codes[8];
    scales |= q8_round<32>(v, codes) << (8 * g);
    __builtin_memcpy(__builtin_assume_aligned(a.codes + row * a.ld + k0 + g * 32, 16), codes, 32);
  }
  *reinterpret_cast<unsigned*>(a.scales + row * a.lds + k0 / Q8_GROUP) = scales;
}

// ------------------------------------------------------------------ plan
// The cheapest tiles and number of shares of the sum by what was measured: a block of 128 of a tile by how many workgroups the
// compute unit holds, a tile beside its blocks (more where others on the unit want the same), and joining shares.  Fitted to
// both products of 40 shapes with 16-bit results and 18 with fp32 ones, 17 x 92 -> 593 to 4096 x 16384 -> 4096, each in every tile
// and with every number of shares: the plan's choice takes 1.2 % more than the best one on average, 14 % at most.  256 x 256 tiles
// (one workgroup per compute unit) have the fastest blocks, 64 x 128 (two) fill the chip where there are few: 4096 x 4096 -> 4096 takes
// 70 us in them, in 128 x 128 (two) 86, in 64 x 128 126; 300 x 300 -> 5000 18, 11 and 8.  (256 x 256 with fp32 results would need
// more registers than there are.)
constexpr long long Q8_FEW = 16;       // most tokens that go without tiles
struct Q8Kind {
  int name, rows, cols, places;
  double block[2], tile, crowd;        // us; one workgroup on the unit, two
};
struct Q8Plan { int kind, splits; double us; };
Q8Plan q8_plan(long long M, long long N, long long blocks, bool dual, bool exact) {
  if (M <= Q8_FEW) return {3, 1, 0.0};
  static const Q8Kind kinds[2][3] = {
      {{0, 256, 256, 1, {1.46, 0.0}, 5.0, 0.0}, {1, 128, 128, 2, {0.60, 1.01}, 2.4, 0.87}, {4, 64, 128, 2, {0.50, 0.74}, 1.1, 1.5}},
      {{1, 128, 128, 2, {0.94, 1.51}, 2.2, 0.80}, {4, 64, 128, 2, {0.67, 0.97}, 0.55, 4.2}, {}}};
  constexpr double LAUNCH = 4.0, JOIN = 2.5;
  Q8Plan best{1, 1, 1e30};
  const double planes = 4.0 * M * N * (dual ? 2 : 1);
  for (const Q8Kind& k : kinds[exact]) {
    if (k.rows == 0) continue;
    const long long tiles = ff_cdiv(M, k.rows) * ff_cdiv(N, dual ? k.cols / 2 : k.cols);
    for (int splits = 1; splits <= 64; splits *= 2) {
      if (splits > 1 && (blocks < splits || planes * splits > 512e6)) break;
      const long long groups = tiles * splits, units = 256LL * k.places, rest = groups % units, each = ff_cdiv(blocks, splits);
      auto turn = [&](long long on) { return each * k.block[on - 1] + k.tile * (1.0 + k.crowd * (on - 1)); };
      double us = LAUNCH + (double)(groups / units) * turn(k.places);
      if (rest) us += turn(ff_cdiv(rest, 256));
      if (splits > 1) us += JOIN + planes * 2 * splits / 5.0e6;
      if (us < best.us) best = {k.name, splits, us};
    }
  }
  return best;
}
// Whether a pair of products of few tokens with 16-bit results takes 32 columns per workgroup and not 16 (q8few.h).
bool q8_few_wide(long long tokens, long long m, long long n) {
  if (ff_cdiv(m, 4096) % 2) return false;                       // half of the last 32-column workgroups' places would be empty
  if (m > 8192) return tokens >= 8 || n <= 2048;
  return tokens >= 8 && n >= 4096 && (m < 8192 || n < 8192);
}
// Workgroups (along x) of a product's launch.
long long q8_groups(int kind, long long M, long long N, bool dual, int splits) {
  const int half = dual ? 2 : 1;
  switch (kind) {
    case 0: return ff_cdiv(M, 256) * ff_cdiv(N, 256 / half) * splits;
    case 1: return ff_cdiv(M, 128) * ff_cdiv(N, 128 / half) * splits;
    case 3: return ff_cdiv(N, Q8F_COLS);
    default: return ff_cdiv(M, 64) * ff_cdiv(N, 128 / half) * splits;
  }
}
size_t q8_workspace(long long M, long long N, long long n, bool dual, bool* fits) {
  size_t most = 0;
  for (bool exact : {false, true}) {
    const Q8Plan plan = q8_plan(M, N, q8_wide(n) / Q8_BLOCK, dual, exact);
    if (q8_groups(plan.kind, M, N, dual, plan.splits) > FF_MOST_THREADS / 512) *fits = false;
    const size_t bytes = plan.splits > 1 ? (size_t)plan.splits * (dual ? 2 : 1) * M * (ff_cdiv(N, 4) * 4) * 4 : 0;
    most = bytes > most ? bytes : most;
  }
  return ff_up(most) + 256;
}

// ------------------------------------------------------------------ launches
template <typename T, bool DUAL, int EPI>
void q8_tiles(const Q8Product& q, int kind, hipStream_t stream) {
  constexpr bool EXACT = sizeof(T) == 4;
  mark(stream);
  const dim3 grid((unsigned)q8_groups(kind, q.p.M, q.p.N, DUAL, q.p.splits));
  if constexpr (!EXACT) {
    if (kind == 0) {
      launch(q8_tile_kernel<T, DUAL, EPI, 256, 256, 2, 4, EXACT>, grid, dim3(512), stream, q);
      return;
    }
  }
  if (kind == 1) launch(q8_tile_kernel<T, DUAL, EPI, 128, 128, 2, 2, EXACT>, grid, dim3(256), stream, q);
  else launch(q8_tile_kernel<T, DUAL, EPI, 64, 128, 2, 2, EXACT>, grid, dim3(256), stream, q);
}
template <typename T, bool DUAL, int EPI>
int q8_product(Q8Product q, void* workspace, hipStream_t stream) {
  constexpr bool EXACT = sizeof(T) == 4;
  FfProduct& p = q.p;
  const Q8Plan plan = q8_plan(p.M, p.N, p.K / Q8_BLOCK, DUAL, EXACT);
  p.splits = plan.splits;
  p.partial = static_cast<float*>(workspace);
  if (plan.kind == 3) {
    mark(stream);
    auto go = [&](auto* kernel, int columns) { launch(kernel, dim3((unsigned)ff_cdiv(p.N, columns)), dim3(512), stream, q); };
    if constexpr (DUAL) {
      if constexpr (!EXACT) {
        if (q8_few_wide(p.M, p.N, p.K)) {
          go(q8_few_kernel<T, true, EPI, 2, 4, 8, false>, 32);
          mark(stream);
          return launch_status();
        }
      }
      go(q8_few_kernel<T, true, EPI, 1, 4, 8, EXACT>, 16);
    } else {
      if (p.K >= 64 * Q8_BLOCK) go(q8_few_kernel<T, false, EPI, 1, 8, 8, EXACT>, 16);
      else go(q8_few_kernel<T, false, EPI, 1, 4, 8, EXACT>, 16);
    }
  } else if (p.splits == 1) {
    q8_tiles<T, DUAL, EPI>(q, plan.kind, stream);
  } else {
    q8_tiles<T, DUAL, FF_PARTIAL>(q, plan.kind, stream);
    mark(stream);
    const long long quads = ff_cdiv(p.N, 4) * p.M;
    if (p.splits >= 16) launch(ff_join_kernel<T, DUAL, EPI, 8>, dim3((unsigned)ff_cdiv(quads, 32)), dim3(256), stream, p);
    else launch(ff_join_kernel<T, DUAL, EPI, 1>, dim3((unsigned)ff_cdiv(quads, 256)), dim3(256), stream, p);
  }
  mark(stream);
  return launch_status();
}

// Rows of a tile are reached by 32-bit offsets.
constexpr long long Q8_MAX_STRIDE = 1 << 22;
int q8_operand(const mlproj_q8* q, long long n, bool needed) {
  if (!q) return MLPROJ_ERR_NULL_POINTER;
  if (q->rows < 0 || q->n <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (q->rows > Q8_MAX_DIM || q->n > Q8_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  FF_TRY(q8_check(q, q->rows, n, needed && q->rows > 0));
  return q->ld > Q8_MAX_STRIDE || q->lds > Q8_MAX_STRIDE ? MLPROJ_ERR_TOO_LARGE : MLPROJ_OK;
}
Q8Product q8_start(const mlproj_q8* x, const mlproj_q8* w0, const mlproj_q8* w1) {
  Q8Product q{};
  FfProduct& p = q.p;
  p.segs = 1;
  p.A0 = x->codes; p.lda = x->ld; q.sA = static_cast<const unsigned char*>(x->scales); q.ldsa = x->lds;
  p.B0 = w0->codes; p.ldb = w0->ld; q.sB0 = static_cast<const unsigned char*>(w0->scales); q.ldsb = w0->lds;
  if (w1) { p.B1 = w1->codes; q.sB1 = static_cast<const unsigned char*>(w1->scales); }
  p.M = x->rows; p.N = w0->rows; p.K = q8_wide(x->n);
  return q;
}
int q8_sizes(long long tokens, long long n, long long m, bool dual, size_t* workspace) {
  if (tokens < 0 || n <= 0 || m <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (tokens > Q8_MAX_DIM || n > Q8_MAX_DIM || m > Q8_MAX_DIM || tokens * m > (1LL << 38) || tokens * n > (1LL << 38) || n * m > (1LL << 38)) return MLPROJ_ERR_TOO_LARGE;
  bool fits = true;
  *workspace = q8_workspace(tokens, m, n, dual, &fits);
  return fits || tokens == 0 ? MLPROJ_OK : MLPROJ_ERR_TOO_LARGE;
}

}  // namespace
}  // namespace mlproj

using namespace mlproj;

extern "C" {

int q8_pack(int storage, int by_columns, const void* A, long long lda, const mlproj_q8* packed, void* stream) {
  if (!packed) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16 || (by_columns | 1) != 1) return MLPROJ_ERR_BAD_VARIANT;
  const long long rows = packed->rows, n = packed->n;
  if (rows < 0 || n <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (rows > Q8_MAX_DIM || n > Q8_MAX_DIM || rows * n > (1LL << 38)) return MLPROJ_ERR_TOO_LARGE;
  const bool some = rows > 0;
  FF_TRY(ff_check_array(A, some, by_columns ? rows : n, lda, storage == MLPROJ_STORE_F32 ? 4 : 2));
  FF_TRY(q8_check(packed, rows, n, some));
  if (!some) return MLPROJ_OK;
  const Q8Pack a{A, static_cast<unsigned char*>(packed->codes), static_cast<unsigned char*>(packed->scales), lda, packed->ld, packed->lds, rows, n, q8_wide(n)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  mark(s);
  auto go = [&](auto* rows_kernel, auto* columns_kernel) {
    if (by_columns) launch(columns_kernel, dim3((unsigned)(ff_cdiv(rows, 256) * (a.wide / Q8_BLOCK))), dim3(256), s, a);
    else launch(rows_kernel, ff_strided_grid(rows * (a.wide / 8)), dim3(256), s, a);
  };
  if (storage == MLPROJ_STORE_F32) go(q8_pack_rows_kernel<float>, q8_pack_columns_kernel<float>);
  else if (storage == MLPROJ_STORE_BF16) go(q8_pack_rows_kernel<bf16_t>, q8_pack_columns_kernel<bf16_t>);
  else go(q8_pack_rows_kernel<f16_t>, q8_pack_columns_kernel<f16_t>);
  mark(s);
  return launch_status();
}

int mlproj_q8_workspace_bytes(long long tokens, long long n, long long m, int gated, size_t* bytes_out) {
  if (!bytes_out) return MLPROJ_ERR_NULL_POINTER;
  if ((gated | 1) != 1) return MLPROJ_ERR_BAD_DIMENSION;
  return q8_sizes(tokens, n, m, gated != 0, bytes_out);
}

int q8_linear(int storage, int activation, const mlproj_q8* x, const mlproj_q8* W, const void* bias, const void* residual, long long ldr,
              void* y, long long ldy, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !W) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16 || activation < MLPROJ_ACT_SILU || activation > MLPROJ_ACT_NONE) return MLPROJ_ERR_BAD_VARIANT;
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool some = x->rows > 0;
  size_t need;
  FF_TRY(q8_sizes(x->rows, x->n, W->rows, false, &need));
  FF_TRY(q8_operand(x, x->n, some));
  FF_TRY(q8_operand(W, x->n, some));
  FF_TRY(ff_check_array(bias, false, W->rows, W->rows, es));
  FF_TRY(ff_check_array(residual, false, W->rows, ldr, es));
  FF_TRY(ff_check_array(y, some, W->rows, ldy, es));
  FF_TRY(ff_check_workspace(workspace, workspace_bytes, need));
  if (!some) return MLPROJ_OK;
  Q8Product q = q8_start(x, W, nullptr);
  q.p.act = activation;
  q.p.bias = bias;
  q.p.dH = residual; q.p.ldh = ldr;
  q.p.C0 = y; q.p.ldc = ldy;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return q8_product<float, false, FF_PLAIN>(q, workspace, s);
  if (storage == MLPROJ_STORE_BF16) return q8_product<bf16_t, false, FF_PLAIN>(q, workspace, s);
  return q8_product<f16_t, false, FF_PLAIN>(q, workspace, s);
}

int q8_gated(int storage, int activation, const mlproj_q8* x, const mlproj_q8* Wg, const mlproj_q8* Wu, void* h, long long ldh,
             void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !Wg || !Wu) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16 || activation < MLPROJ_ACT_SILU || activation > MLPROJ_ACT_RELU) return MLPROJ_ERR_BAD_VARIANT;
  const bool some = x->rows > 0;
  size_t need;
  FF_TRY(q8_sizes(x->rows, x->n, Wg->rows, true, &need));
  FF_TRY(q8_operand(x, x->n, some));
  FF_TRY(q8_operand(Wg, x->n, some));
  FF_TRY(q8_operand(Wu, x->n, some));
  if (Wu->rows != Wg->rows || Wu->ld != Wg->ld || Wu->lds != Wg->lds) return MLPROJ_ERR_BAD_DIMENSION;
  FF_TRY(ff_check_array(h, some, Wg->rows, ldh, storage == MLPROJ_STORE_F32 ? 4 : 2));
  FF_TRY(ff_check_workspace(workspace, workspace_bytes, need));
  if (!some) return MLPROJ_OK;
  Q8Product q = q8_start(x, Wg, Wu);
  q.p.act = activation;
  q.p.C0 = h; q.p.ldc = ldh;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return q8_product<float, true, FF_FWD>(q, workspace, s);
  if (storage == MLPROJ_STORE_BF16) return q8_product<bf16_t, true, FF_FWD>(q, workspace, s);
  return q8_product<f16_t, true, FF_FWD>(q, workspace, s);
}

}  // extern "C"
