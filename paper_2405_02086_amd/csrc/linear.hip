// mlproj: the product with bias, activation, dropout and residual in its epilogue, forward and backward, and dropout by itself:
// kernels of the elementwise passes, plans and the C ABI.  The products' kernels are those of the gated block (ffplan.h).
#include "ffcommon.h"
#include "ffplan.h"

namespace mlproj {
namespace {

// ------------------------------------------------------------------ gradient at the pre-activations
// dZ = act'(Z) D(dY), rounded to the storage type (it is an operand of the products that follow), and the sums of its columns
// before they are rounded.  Without an activation dZ is left without dropout's factor, which the products apply to their sums in
// fp32: dY's entries and zeros need no rounding, dY / (1 - p) does (bf16 errors of dX and dW are 1.7e-3 of a result's norm, and were
// 2.4e-3 with the factor here).  A thread has eight columns and every row of its worker; the workers' sums go out in fp32 and are
// added in their order, so that results are the same every time.  Z, dZ and the sums are each optional.  Bound by HBM: dropout on
// 4096 x 4096 bf16 takes 18 us (3.7 TB/s), gelu's slope and the sums of 1000 x 10000 fp32 29 (4.4 TB/s) and 5 to join them.
struct LnSlopes {
  const void *dY, *Z;
  void* dZ;
  float* partial;              // [workgroups along y][m], or null
  long long lddy, ldz, lddz, tokens, m;
  int act, lanes;              // lanes: threads side by side along a row, a power of two up to 64
  Dropout drop;
  float factor;                // of the sums: dropout's where dZ is left without it (drop.scale is 1 then), else 1
};
constexpr int LN_THREADS = 256;
template <typename T>
__global__ __launch_bounds__(LN_THREADS) void ln_slopes_kernel(LnSlopes a) {
  __shared__ float sums[LN_THREADS][9];
  dropout_at_step(a.drop);
  const int lane = threadIdx.x & (a.lanes - 1), worker = threadIdx.x / a.lanes, workers = LN_THREADS / a.lanes;
  const long long col = ((long long)blockIdx.x * a.lanes + lane) * 8;
  float sum[8] = {};
  if (col < a.m) {
    for (long long row = (long long)blockIdx.y * workers + worker; row < a.tokens; row += (long long)gridDim.y * workers) {
      const FfVec8<T> y = ff_load8(static_cast<const T*>(a.dY) + row * a.lddy + col, a.m - col);
      FfVec8<T> z = {}, out;
      if (a.Z) z = ff_load8(static_cast<const T*>(a.Z) + row * a.ldz + col, a.m - col);
#pragma unroll
      for (int h = 0; h < 2; h++) {
        f32x4 v, value, slope = {1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = (float)y.v[4 * h + i];
        if (a.Z) {
          f32x4 at;
#pragma unroll
          for (int i = 0; i < 4; i++) at[i] = (float)z.v[4 * h + i];
          ff_gate4<sizeof(T) == 4>(a.act, at, value, slope);
        }
        if (a.drop.threshold) v = dropout4(a.drop, row, (col >> 2) + h, v, slope);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          v[i] = col + 4 * h + i < a.m ? v[i] * slope[i] : 0.0f;
          sum[4 * h + i] += v[i] * a.factor;
          out.v[4 * h + i] = ff_round<T>(v[i]);
        }
      }
      // (rows of dZ are in whole pieces, filled up with zeros)
      if (a.dZ) __builtin_memcpy(static_cast<T*>(a.dZ) + row * a.lddz + col, &out, sizeof(out));
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < 8; i++) sums[threadIdx.x][i] = sum[i];
  __syncthreads();
  for (int j = threadIdx.x; j < a.lanes * 8; j += LN_THREADS) {
    const long long c = (long long)blockIdx.x * a.lanes * 8 + j;
    if (c >= a.m) break;
    float s = 0.0f;
    for (int w = 0; w < workers; w++) s += sums[w * a.lanes + j / 8][j % 8];
    a.partial[blockIdx.y * a.m + c] = s;
  }
}
// The workgroups' sums: 32 columns x 8 runs of workgroups here; of more columns than a launch has threads for, the next ones a
// grid further on.
constexpr long long LN_MOST_COLUMN_GROUPS = 1 << 21;
__global__ __launch_bounds__(256) void ln_columns_kernel(const float* partial, int groups, long long m, float* out) {
  __shared__ float part[8][32];
  const int cx = threadIdx.x & 31, gy = threadIdx.x >> 5;
  for (long long first = (long long)blockIdx.x * 32; first < m; first += (long long)gridDim.x * 32) {
    const long long col = first + cx;
    float s = 0.0f;
    if (col < m)
#pragma unroll 8
      for (int g = gy; g < groups; g += 8) s += partial[g * m + col];
    part[gy][cx] = s;
    __syncthreads();
    if (gy == 0 && col < m) {
#pragma unroll
      for (int i = 1; i < 8; i++) s += part[i][cx];
      out[col] = s;
    }
    __syncthreads();
  }
}
// What an empty batch leaves.
template <typename T>
__global__ __launch_bounds__(256) void ln_zero_kernel(T* dW, long long rows, long long cols, long long ld, float* dbias) {
  const long long first = (long long)blockIdx.x * 256 + threadIdx.x, stride = (long long)gridDim.x * 256;
  if (dW)
    for (long long i = first; i < rows * cols; i += stride) dW[i / cols * ld + i % cols] = (T)0.0f;
  if (dbias)
    for (long long i = first; i < cols; i += stride) dbias[i] = 0.0f;
}

// Threads side by side and workgroups along the rows: about eight workgroups per compute unit, and no more than rows.
struct LnShape { int lanes; long long across; int down; };
LnShape ln_shape(long long tokens, long long m) {
  const long long pieces = ff_cdiv(m, 8);
  LnShape s{64, ff_cdiv(pieces, 64), 1};
  while (s.lanes > 1 && s.lanes / 2 >= pieces) s.lanes /= 2;
  const long long rows = ff_cdiv(tokens, LN_THREADS / s.lanes), want = ff_cdiv(2048, s.across);
  s.down = (int)(rows < want ? (rows > 0 ? rows : 1) : want);
  return s;
}

// ------------------------------------------------------------------ dropout by itself
// y = residual + D(x), in pieces of 16 bytes.  Bound by HBM (16384 x 4096 bf16 with a residual 74 us, 5.4 TB/s) and, where little is
// read, by the generator (dropout.h).
struct LnDrop {
  const void *x, *residual;
  void* y;
  long long ldx, ldr, ldy, tokens, n, pieces;
  Dropout drop;
};
template <typename T>
__global__ __launch_bounds__(256) void ln_dropout_kernel(LnDrop a) {
  constexpr int VEC = 16 / sizeof(T);
  struct alignas(sizeof(T)) Piece { T v[VEC]; };
  dropout_at_step(a.drop);
  // (the workgroup's first piece by a division of its own, its others from there)
  const unsigned pieces = (unsigned)a.pieces;
  for (long long first = (long long)blockIdx.x * 256; first < a.tokens * a.pieces; first += (long long)gridDim.x * 256) {
    long long row = first >> 32 ? first / a.pieces : (unsigned)first / pieces;
    unsigned in = (unsigned)(first - row * a.pieces) + threadIdx.x;
    if (pieces >= 256) {
      if (in >= pieces) { in -= pieces; row++; }
    } else {
      const unsigned on = in / pieces;
      in -= on * pieces;
      row += on;
    }
    if (row >= a.tokens) break;
    const long long col = (long long)in * VEC, valid = a.n - col;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx + col;
    const T* r = static_cast<const T*>(a.residual) + row * a.ldr + col;
    T* y = static_cast<T*>(a.y) + row * a.ldy + col;
    Piece px, pr = {};
    if (valid >= VEC) {
      __builtin_memcpy(&px, x, sizeof(px));
      if (a.residual) __builtin_memcpy(&pr, r, sizeof(pr));
    } else {
#pragma unroll
      for (int i = 0; i < VEC; i++) {
        px.v[i] = i < valid ? x[i] : (T)0.0f;
        pr.v[i] = a.residual && i < valid ? r[i] : (T)0.0f;
      }
    }
#pragma unroll
    for (int h = 0; h < VEC / 4; h++) {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] = (float)px.v[4 * h + i];
      if (a.drop.threshold) v = dropout4(a.drop, row, (col >> 2) + h, v);
#pragma unroll
      for (int i = 0; i < 4; i++) px.v[4 * h + i] = ff_round<T>(a.residual ? (float)pr.v[4 * h + i] + v[i] : v[i]);
    }
    if (valid >= VEC) {
      __builtin_memcpy(y, &px, sizeof(px));
    } else {
#pragma unroll
      for (int i = 0; i < VEC; i++)
        if (i < valid) y[i] = px.v[i];
    }
  }
}

// ------------------------------------------------------------------ plan and workspace
double ln_products_us(int es, long long tokens, long long n, long long m, bool backward, bool direct) {
  if (!backward) return ff_plan(tokens, m, ff_steps(n, 1), false, FF_LINEAR, direct, es).us;
  return ff_plan(tokens, n, ff_steps(m, 1), false, FF_STORE, direct, es).us + ff_plan(n, m, ff_steps(tokens, 1), false, FF_STORE, direct, es).us;
}
// Whether 16-bit operands whose rows are not in whole 16-byte pieces are copied into rows that are: where that is
// cheaper than the staged tiles by the plan.  Copies are reckoned at 4 TB/s, read and written (large
// ones reach 5), and 5 us.
bool ln_pads(int es, long long tokens, long long n, long long m, bool backward) {
  if (es != 2 || (n % 8 == 0 && m % 8 == 0)) return false;
  const double elements = (n % 8 ? (double)tokens * n : 0.0) + (m % 8 ? (double)n * m : 0.0);
  return ln_products_us(es, tokens, n, m, backward, true) + 5.0 + elements * 2 * es / 4.0e6 < ln_products_us(es, tokens, n, m, backward, false);
}
struct LnLayout {
  long long ldn, ldm;          // rows of n and m entries in whole 16-byte pieces
  size_t partial;              // shares of sums, of one product at a time
  size_t X, W;                 // padded copies
  size_t dZ, columns;          // backward: the gradient at the pre-activations, sums of its columns
  size_t bytes;
  bool pads, fits;
};
LnLayout ln_layout(int es, long long tokens, long long n, long long m, bool backward) {
  LnLayout L{};
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += ff_up(bytes);
    return at;
  };
  L.ldn = ff_cdiv(n, 8) * 8;
  L.ldm = ff_cdiv(m, 8) * 8;
  L.fits = true;
  size_t shares;
  if (backward) {
    const size_t x = ff_partial_bytes(tokens, n, m, 1, false, FF_STORE, es, &L.fits), w = ff_partial_bytes(n, m, tokens, 1, false, FF_STORE, es, &L.fits);
    shares = x > w ? x : w;
  } else {
    shares = ff_partial_bytes(tokens, m, n, 1, false, FF_LINEAR, es, &L.fits);
  }
  if (tokens == 0) L.fits = true;
  L.partial = take(shares);
  L.pads = ln_pads(es, tokens, n, m, backward);
  if (L.pads && n % 8) L.X = take((size_t)tokens * L.ldn * es);
  if (L.pads && m % 8) L.W = take((size_t)n * L.ldm * es);
  if (backward) {
    L.dZ = take((size_t)tokens * L.ldm * es);
    L.columns = take((size_t)ln_shape(tokens, m).down * m * 4);
  }
  L.bytes = o + 256;
  return L;
}
int ln_workspace(int storage, long long tokens, long long n, long long m, int backward, size_t* out) {
  if (!out) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16) return MLPROJ_ERR_BAD_VARIANT;
  if (tokens < 0 || n <= 0 || m <= 0 || (backward | 1) != 1) return MLPROJ_ERR_BAD_DIMENSION;
  if (tokens > FF_MAX_DIM || n > FF_MAX_DIM || m > FF_MAX_DIM || tokens * m > (1LL << 38) || tokens * n > (1LL << 38) || n * m > (1LL << 38)) return MLPROJ_ERR_TOO_LARGE;
  const LnLayout L = ln_layout(storage == MLPROJ_STORE_F32 ? 4 : 2, tokens, n, m, backward != 0);
  if (!L.fits) return MLPROJ_ERR_TOO_LARGE;
  *out = L.bytes;
  return MLPROJ_OK;
}

// An operand, the caller's or a copy in filled rows.
struct LnOperand {
  const void* at;
  long long ld;
  bool filled;
};
struct LnOperands { LnOperand X, W; };
template <typename T>
LnOperands ln_operands(const mlproj_linear* b, const LnLayout& L, char* ws, bool x, bool w, hipStream_t stream) {
  LnOperands o{{b->X, b->ldx, false}, {b->W, b->ldw, false}};
  FfPadder pad;
  if (L.pads && b->n % 8 && x) {
    pad.add(b->X, b->ldx, ws + L.X, L.ldn, b->tokens, b->n);
    o.X = {ws + L.X, L.ldn, true};
  }
  if (L.pads && b->m % 8 && w) {
    pad.add(b->W, b->ldw, ws + L.W, L.ldm, b->n, b->m);
    o.W = {ws + L.W, L.ldm, true};
  }
  pad.go<T>(stream);
  return o;
}

template <typename T>
int run_forward(int act, const mlproj_linear* b, const void* residual, long long ldr, void* Y, long long ldy, void* Z, long long ldz,
                void* workspace, hipStream_t stream) {
  const LnLayout L = ln_layout(sizeof(T), b->tokens, b->n, b->m, false);
  char* ws = static_cast<char*>(workspace);
  const LnOperands o = ln_operands<T>(b, L, ws, true, true, stream);
  FfProduct p{};
  p.segs = 1; p.act = act;
  p.A0 = o.X.at; p.lda = o.X.ld; p.a_filled = o.X.filled;
  p.B0 = o.W.at; p.ldb = o.W.ld; p.b_filled = o.W.filled;
  p.M = b->tokens; p.N = b->m; p.K = b->n;
  p.C0 = Y; p.ldc = ldy;
  p.G = Z; p.ldg = ldz;
  p.dH = residual; p.ldh = ldr;
  p.bias = b->bias;
  p.drop = dropout_start(b->dropout);
  ff_product<T, true, false, false, FF_LINEAR>(p, ws + L.partial, stream);
  mark(stream);
  return launch_status();
}

template <typename T>
int run_backward(int act, const mlproj_linear* b, const void* dY, long long lddy, const void* Z, long long ldz, void* dX, long long lddx,
                 void* dW, long long lddw, float* dbias, void* workspace, hipStream_t stream) {
  if (b->tokens == 0) {
    if (dW || dbias) {
      mark(stream);
      launch(ln_zero_kernel<T>, ff_strided_grid(dW ? b->n * b->m : b->m), dim3(256), stream, static_cast<T*>(dW), b->n, b->m, lddw, dbias);
    }
    mark(stream);
    return launch_status();
  }
  const LnLayout L = ln_layout(sizeof(T), b->tokens, b->n, b->m, true);
  char* ws = static_cast<char*>(workspace);
  const Dropout drop = dropout_start(b->dropout);
  const bool slopes = act != MLPROJ_ACT_NONE, products = dX || dW;
  const float factor = !slopes && drop.threshold ? drop.scale : 1.0f;
  LnOperand dZ{dY, lddy, false};
  // dY itself is dZ where there is neither activation nor dropout, and its rows may stay as they are
  const bool write = products && (slopes || drop.threshold || (L.pads && b->m % 8));
  if (write || dbias) {
    const LnShape s = ln_shape(b->tokens, b->m);
    LnSlopes a{};
    a.dY = dY; a.lddy = lddy; a.Z = slopes ? Z : nullptr; a.ldz = ldz;
    a.dZ = write ? ws + L.dZ : nullptr; a.lddz = L.ldm;
    a.partial = dbias ? reinterpret_cast<float*>(ws + L.columns) : nullptr;
    a.tokens = b->tokens; a.m = b->m; a.act = act; a.lanes = s.lanes;
    a.drop = drop;
    a.factor = factor;
    if (!slopes) a.drop.scale = 1.0f;
    mark(stream);
    launch(ln_slopes_kernel<T>, dim3((unsigned)s.across, (unsigned)s.down), dim3(LN_THREADS), stream, a);
    if (write) dZ = {ws + L.dZ, L.ldm, true};
    if (dbias) {
      mark(stream);
      const long long columns = ff_cdiv(b->m, 32);
      launch(ln_columns_kernel, dim3((unsigned)(columns < LN_MOST_COLUMN_GROUPS ? columns : LN_MOST_COLUMN_GROUPS)), dim3(256), stream, a.partial, s.down, b->m, dbias);
    }
  }
  const LnOperands o = ln_operands<T>(b, L, ws, dW != nullptr, dX != nullptr, stream);
  if (dX) {
    FfProduct p{};
    p.segs = 1;
    p.A0 = dZ.at; p.lda = dZ.ld; p.a_filled = dZ.filled && o.W.filled;
    p.B0 = o.W.at; p.ldb = o.W.ld; p.b_filled = o.W.filled;
    p.M = b->tokens; p.N = b->n; p.K = b->m;
    p.C0 = dX; p.ldc = lddx;
    p.scale = factor;
    ff_product<T, true, true, false, FF_SCALED>(p, ws + L.partial, stream);
  }
  if (dW) {
    FfProduct p{};
    p.segs = 1;
    p.A0 = o.X.at; p.lda = o.X.ld; p.a_filled = o.X.filled;
    p.B0 = dZ.at; p.ldb = dZ.ld; p.b_filled = dZ.filled;
    p.M = b->n; p.N = b->m; p.K = b->tokens;
    p.C0 = dW; p.ldc = lddw;
    p.scale = factor;
    ff_product<T, false, false, false, FF_SCALED>(p, ws + L.partial, stream);
  }
  mark(stream);
  return launch_status();
}

int ln_check(int storage, int act, const mlproj_linear* b) {
  if (!b) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16 || act < MLPROJ_ACT_SILU || act > MLPROJ_ACT_NONE) return MLPROJ_ERR_BAD_VARIANT;
  if (b->tokens < 0 || b->n <= 0 || b->m <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (b->tokens > FF_MAX_DIM || b->n > FF_MAX_DIM || b->m > FF_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  return dropout_check(b->dropout);
}

}  // namespace
}  // namespace mlproj

using namespace mlproj;

extern "C" {

int mlproj_linear_workspace_bytes(int storage, long long tokens, long long n, long long m, int backward, size_t* bytes_out) {
  return ln_workspace(storage, tokens, n, m, backward, bytes_out);
}

int linear_forward(int storage, int activation, const mlproj_linear* b, const void* residual, long long ldr, void* Y, long long ldy,
                   void* Z, long long ldz, void* workspace, size_t workspace_bytes, void* stream) {
  FF_TRY(ln_check(storage, activation, b));
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool some = b->tokens > 0;
  size_t need;
  FF_TRY(ln_workspace(storage, b->tokens, b->n, b->m, 0, &need));
  FF_TRY(ff_check_array(b->X, some, b->n, b->ldx, es));
  FF_TRY(ff_check_array(b->W, some, b->m, b->ldw, es));
  FF_TRY(ff_check_array(b->bias, false, b->m, b->m, es));
  FF_TRY(ff_check_array(residual, false, b->m, ldr, es));
  FF_TRY(ff_check_array(Y, some, b->m, ldy, es));
  FF_TRY(ff_check_array(Z, false, b->m, ldz, es));
  FF_TRY(ff_check_workspace(workspace, workspace_bytes, need));
  if (!some) return MLPROJ_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return run_forward<float>(activation, b, residual, ldr, Y, ldy, Z, ldz, workspace, s);
  if (storage == MLPROJ_STORE_BF16) return run_forward<bf16_t>(activation, b, residual, ldr, Y, ldy, Z, ldz, workspace, s);
  return run_forward<f16_t>(activation, b, residual, ldr, Y, ldy, Z, ldz, workspace, s);
}

int linear_backward(int storage, int activation, const mlproj_linear* b, const void* dY, long long lddy, const void* Z, long long ldz,
                    void* dX, long long lddx, void* dW, long long lddw, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  FF_TRY(ln_check(storage, activation, b));
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool some = b->tokens > 0;
  size_t need;
  FF_TRY(ln_workspace(storage, b->tokens, b->n, b->m, 1, &need));
  FF_TRY(ff_check_array(b->X, some && dW, b->n, b->ldx, es));
  FF_TRY(ff_check_array(b->W, some && dX, b->m, b->ldw, es));
  FF_TRY(ff_check_array(dY, some, b->m, lddy, es));
  FF_TRY(ff_check_array(Z, some && activation != MLPROJ_ACT_NONE, b->m, ldz, es));
  FF_TRY(ff_check_array(dX, false, b->n, lddx, es));
  FF_TRY(ff_check_array(dW, false, b->m, lddw, es));
  FF_TRY(ff_check_array(dbias, false, b->m, b->m, 4));
  FF_TRY(ff_check_workspace(workspace, workspace_bytes, need));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return run_backward<float>(activation, b, dY, lddy, Z, ldz, dX, lddx, dW, lddw, dbias, workspace, s);
  if (storage == MLPROJ_STORE_BF16) return run_backward<bf16_t>(activation, b, dY, lddy, Z, ldz, dX, lddx, dW, lddw, dbias, workspace, s);
  return run_backward<f16_t>(activation, b, dY, lddy, Z, ldz, dX, lddx, dW, lddw, dbias, workspace, s);
}

int dropout_forward(int storage, const mlproj_dropout* dropout, long long tokens, long long n, const void* x, long long ldx, const void* residual,
                    long long ldr, void* y, long long ldy, void* stream) {
  if (!dropout) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16) return MLPROJ_ERR_BAD_VARIANT;
  if (tokens < 0 || n <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (tokens > FF_MAX_DIM || n > FF_MAX_DIM || tokens * n > (1LL << 38)) return MLPROJ_ERR_TOO_LARGE;
  FF_TRY(dropout_check(dropout));
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool some = tokens > 0;
  FF_TRY(ff_check_array(x, some, n, ldx, es));
  FF_TRY(ff_check_array(residual, false, n, ldr, es));
  FF_TRY(ff_check_array(y, some, n, ldy, es));
  if (!some) return MLPROJ_OK;
  LnDrop a{x, residual, y, ldx, ldr, ldy, tokens, n, ff_cdiv(n, 16 / es), dropout_start(dropout)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid = ff_strided_grid(a.tokens * a.pieces);
  mark(s);
  if (storage == MLPROJ_STORE_F32) launch(ln_dropout_kernel<float>, grid, dim3(256), s, a);
  else if (storage == MLPROJ_STORE_BF16) launch(ln_dropout_kernel<bf16_t>, grid, dim3(256), s, a);
  else launch(ln_dropout_kernel<f16_t>, grid, dim3(256), s, a);
  mark(s);
  return launch_status();
}

}  // extern "C"
