// mlproj: the norms before and after a block, fused with its gate and the residual scale; kernels, plan and C ABI.
#include "ffcommon.h"
#include "host.h"

namespace mlproj {
namespace {

// ------------------------------------------------------------------ rows in registers
// A row's entries are dealt in 16-byte pieces: piece i of a row belongs to thread i % THREADS of the row's
// threads (a wavefront, or a workgroup of 256 or 1024), CH of them per thread, and stays in its registers from the one
// load to the one store.  Loads take any address; the last piece of a row is filled up element by element.
// Both directions are bound by HBM: forward reads x and b and writes r and y once, backward reads four
// arrays and writes two.
template <typename T> constexpr int BN_VEC = 16 / sizeof(T);

struct BnArgs {
  const void *x, *b, *w_post, *gate, *w_pre;   // forward: x; backward: r in its place
  void *r, *y;
  const void *dr, *dy;
  void *dx, *db, *dgate;
  float* partial;                               // [3][workgroups][n] sums over a workgroup's rows
  long long ldx, ldb, gate_stride, ldr, ldy, lddr, lddy, lddx, lddb, dgate_stride;
  long long tokens, n;
  float scale, eps;
  int want_post, want_gate, want_pre;           // backward: which sums over tokens are wanted
};

template <typename T, int VEC>
__device__ __forceinline__ void bn_load(const T* p, long long valid, float (&out)[VEC]) {
  if (valid >= VEC) {
    struct alignas(sizeof(T)) { T v[VEC]; } t;
    __builtin_memcpy(&t, p, sizeof(t));
#pragma unroll
    for (int i = 0; i < VEC; i++) out[i] = (float)t.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i++) out[i] = i < valid ? (float)p[i] : 0.0f;
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void bn_store(T* p, long long valid, const float (&x)[VEC]) {
  if (valid >= VEC) {
    struct alignas(sizeof(T)) { T v[VEC]; } t;
#pragma unroll
    for (int i = 0; i < VEC; i++) t.v[i] = ff_round<T>(x[i]);
    __builtin_memcpy(p, &t, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i++)
      if (i < valid) p[i] = ff_round<T>(x[i]);
  }
}

// Sums N values over the row's threads, everyone gets them.  `slot`: LDS of [2][N][16], the halves used in turn so
// that one barrier per sum is enough.
template <int THREADS, int N>
__device__ __forceinline__ void bn_sum(float (&v)[N], float (*slot)[16], int lane, int wave) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1)
#pragma unroll
    for (int i = 0; i < N; i++) v[i] += __shfl_xor(v[i], s);
  if constexpr (THREADS > 64) {
    constexpr int WAVES = THREADS / 64;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; i++) slot[i][wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) {
      float t = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; w++) t += slot[i][w];
      v[i] = t;
    }
  }
}

// HELD: the row's pieces fit the registers (CH per thread); otherwise CH of them at a time, and every phase
// reads them again (from L2, where a row still is).
template <typename T, int THREADS, int CH, bool HELD>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void bn_forward_kernel(BnArgs a) {
  constexpr int VEC = BN_VEC<T>;
  constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ float slots[2][1][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = THREADS < 256 ? lane : threadIdx.x;
  const long long row = (long long)blockIdx.x * ROWS + (ROWS > 1 ? wave : 0);
  if (row >= a.tokens) return;                 // (with THREADS > 64 the whole workgroup)
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* b = a.b ? static_cast<const T*>(a.b) + row * a.ldb : nullptr;
  const T* gate = static_cast<const T*>(a.gate) + row * a.gate_stride;
  const T* w_post = static_cast<const T*>(a.w_post);
  const T* w_pre = static_cast<const T*>(a.w_pre);
  T* r = static_cast<T*>(a.r) + row * a.ldr;
  T* y = static_cast<T*>(a.y) + row * a.ldy;
  const long long n = a.n, per = (long long)THREADS * VEC * CH;
  const long long passes = HELD ? 1 : (n + per - 1) / per;
  const float inv_n = 1.0f / (float)n;
  float vx[CH][VEC], vb[CH][VEC];
  float rb = 0.0f, sum[1];

  auto load = [&](long long pass) {
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const long long at = pass * per + ((long long)c * THREADS + t) * VEC;
      bn_load<T, VEC>(x + at, n - at, vx[c]);
      if (b) bn_load<T, VEC>(b + at, n - at, vb[c]);
    }
  };
  auto join = [&](long long pass) {            // vx becomes r
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const long long at = pass * per + ((long long)c * THREADS + t) * VEC;
      float g[VEC], w[VEC];
      bn_load<T, VEC>(gate + at, n - at, g);
      bn_load<T, VEC>(w_post + at, n - at, w);
#pragma unroll
      for (int i = 0; i < VEC; i++) vx[c][i] += a.scale * g[i] * (vb[c][i] * rb * w[i]);
    }
  };

  if (b) {
    sum[0] = 0.0f;
    for (long long pass = 0; pass < passes; pass++) {
      load(pass);
#pragma unroll
      for (int c = 0; c < CH; c++)
#pragma unroll
        for (int i = 0; i < VEC; i++) sum[0] += vb[c][i] * vb[c][i];
    }
    bn_sum<THREADS, 1>(sum, slots[0], lane, wave);
    rb = 1.0f / sqrtf(sum[0] * inv_n + a.eps);
  } else if constexpr (HELD) {
    load(0);
  }
  float rr = 0.0f;
  if (w_pre) {
    sum[0] = 0.0f;
    for (long long pass = 0; pass < passes; pass++) {
      if constexpr (!HELD) load(pass);
      if (b) join(pass);
#pragma unroll
      for (int c = 0; c < CH; c++)
#pragma unroll
        for (int i = 0; i < VEC; i++) sum[0] += vx[c][i] * vx[c][i];
    }
    bn_sum<THREADS, 1>(sum, slots[1], lane, wave);
    rr = 1.0f / sqrtf(sum[0] * inv_n + a.eps);
  }
  for (long long pass = 0; pass < passes; pass++) {
    if constexpr (!HELD) load(pass);
    if (b && (!HELD || !w_pre)) join(pass);
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const long long at = pass * per + ((long long)c * THREADS + t) * VEC;
      if (at >= n) break;
      if (b) bn_store<T, VEC>(r + at, n - at, vx[c]);
      if (w_pre) {
        float w[VEC];
        bn_load<T, VEC>(w_pre + at, n - at, w);
#pragma unroll
        for (int i = 0; i < VEC; i++) w[i] *= vx[c][i] * rr;
        bn_store<T, VEC>(y + at, n - at, w);
      }
    }
  }
}

// One round of sums per row: with e = w_pre dy and f = scale gate w_post,
//   mean(r e), mean(r^2), mean(b^2), and the three parts of sum(b f dx), dx = dr + rr e - r rr^3 mean(r e):
//   sum(b f dr), sum(b f e), sum(b f r).
// A workgroup takes every gridDim-th row and keeps the sums over its rows of the columns its threads hold, which go
// out as one partial per workgroup and are summed, in their order, by bn_columns_kernel: the same bits
// every time.  With one gate per channel dgate and dw_post are both multiples of sum dx b / rms(b).
template <typename T, int THREADS, int CH, bool HELD, bool TOKEN_GATE>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void bn_backward_kernel(BnArgs a) {
  constexpr int VEC = BN_VEC<T>;
  constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ float slots[2][6][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = THREADS < 256 ? lane : threadIdx.x;
  const long long n = a.n, per = (long long)THREADS * VEC * CH;
  const long long passes = HELD ? 1 : (n + per - 1) / per;
  const float inv_n = 1.0f / (float)n;
  const T* w_post = static_cast<const T*>(a.w_post);
  const T* w_pre = static_cast<const T*>(a.w_pre);
  const long long worker = (long long)blockIdx.x * ROWS + (ROWS > 1 ? wave : 0);
  const long long workers = (long long)gridDim.x * ROWS;
  float* partial = a.partial + worker * n;
  const long long plane = workers * n;
  float s_post[CH][VEC] = {}, s_pre[CH][VEC] = {};
  int turn = 0;

  for (long long row = worker; row < a.tokens; row += workers, turn ^= 1) {
    const T* r = static_cast<const T*>(a.x) + row * a.ldx;
    const T* b = a.b ? static_cast<const T*>(a.b) + row * a.ldb : nullptr;
    const T* dr = a.dr ? static_cast<const T*>(a.dr) + row * a.lddr : nullptr;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const T* gate = static_cast<const T*>(a.gate) + row * a.gate_stride;
    float vr[CH][VEC], vb[CH][VEC] = {}, vd[CH][VEC] = {}, vy[CH][VEC] = {};
    auto load = [&](long long pass) {
#pragma unroll
      for (int c = 0; c < CH; c++) {
        const long long at = pass * per + ((long long)c * THREADS + t) * VEC;
        bn_load<T, VEC>(r + at, n - at, vr[c]);
        if (b) bn_load<T, VEC>(b + at, n - at, vb[c]);
        if (dr) bn_load<T, VEC>(dr + at, n - at, vd[c]);
        if (w_pre) bn_load<T, VEC>(dy + at, n - at, vy[c]);
      }
    };
    float sum[6] = {};
    for (long long pass = 0; pass < passes; pass++) {
      load(pass);
#pragma unroll
      for (int c = 0; c < CH; c++) {
        const long long at = pass * per + ((long long)c * THREADS + t) * VEC;
        float f[VEC] = {}, w[VEC] = {};
        if (b) {
          float g[VEC];
          bn_load<T, VEC>(gate + at, n - at, g);
          bn_load<T, VEC>(w_post + at, n - at, f);
#pragma unroll
          for (int i = 0; i < VEC; i++) f[i] *= a.scale * g[i];
        }
        if (w_pre) bn_load<T, VEC>(w_pre + at, n - at, w);
#pragma unroll
        for (int i = 0; i < VEC; i++) {
          const float e = w[i] * vy[c][i], bf = vb[c][i] * f[i];
          sum[0] += vr[c][i] * e;
          sum[1] += vr[c][i] * vr[c][i];
          sum[2] += vb[c][i] * vb[c][i];
          sum[3] += bf * vd[c][i];
          sum[4] += bf * e;
          sum[5] += bf * vr[c][i];
        }
      }
    }
    bn_sum<THREADS, 6>(sum, slots[turn], lane, wave);
    const float rr = w_pre ? 1.0f / sqrtf(sum[1] * inv_n + a.eps) : 0.0f;
    const float rb = 1.0f / sqrtf(sum[2] * inv_n + a.eps);
    const float kr = w_pre ? rr * rr * rr * (sum[0] * inv_n) : 0.0f;
    const float kb = rb * rb * rb * ((sum[3] + rr * sum[4] - kr * sum[5]) * inv_n);
    for (long long pass = 0; pass < passes; pass++) {
      if constexpr (!HELD) load(pass);
#pragma unroll
      for (int c = 0; c < CH; c++) {
        const long long at = pass * per + ((long long)c * THREADS + t) * VEC;
        if (at >= n) break;
        float dx[VEC], w[VEC] = {};
        if (w_pre) bn_load<T, VEC>(w_pre + at, n - at, w);
#pragma unroll
        for (int i = 0; i < VEC; i++) dx[i] = vd[c][i] + (rr * (w[i] * vy[c][i]) - kr * vr[c][i]);
        if (a.dx) bn_store<T, VEC>(static_cast<T*>(a.dx) + row * a.lddx + at, n - at, dx);
        float pre[VEC], post[VEC] = {};
#pragma unroll
        for (int i = 0; i < VEC; i++) pre[i] = vy[c][i] * vr[c][i] * rr;
        if (b) {
          float g[VEC], wp[VEC], db[VEC], dg[VEC];
          bn_load<T, VEC>(gate + at, n - at, g);
          bn_load<T, VEC>(w_post + at, n - at, wp);
#pragma unroll
          for (int i = 0; i < VEC; i++) {
            const float sdx = a.scale * dx[i], bh = vb[c][i] * rb;
            db[i] = rb * (sdx * g[i] * wp[i]) - kb * vb[c][i];
            dg[i] = sdx * wp[i] * bh;
            post[i] = TOKEN_GATE ? sdx * g[i] * bh : sdx * bh;
          }
          if (a.db) bn_store<T, VEC>(static_cast<T*>(a.db) + row * a.lddb + at, n - at, db);
          if (TOKEN_GATE && a.dgate) bn_store<T, VEC>(static_cast<T*>(a.dgate) + row * a.dgate_stride + at, n - at, dg);
        }
        if constexpr (HELD) {
#pragma unroll
          for (int i = 0; i < VEC; i++) { s_post[c][i] += post[i]; s_pre[c][i] += pre[i]; }
        } else {
          // too many columns for registers: the sums live in the worker's own partials
          for (int i = 0; i < VEC && at + i < n; i++) {
            const bool fresh = row == worker;
            if (a.want_post || a.want_gate) partial[at + i] = post[i] + (fresh ? 0.0f : partial[at + i]);
            if (a.want_pre) partial[plane + at + i] = pre[i] + (fresh ? 0.0f : partial[plane + at + i]);
          }
        }
      }
    }
  }
  if constexpr (HELD) {
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const long long at = ((long long)c * THREADS + t) * VEC;
      if (at >= n) break;
      if (a.want_post || a.want_gate) bn_store<float, VEC>(partial + at, n - at, s_post[c]);
      if (a.want_pre) bn_store<float, VEC>(partial + plane + at, n - at, s_pre[c]);
    }
  } else if (worker >= a.tokens) {
    for (long long j = t; j < n; j += THREADS) partial[j] = partial[plane + j] = 0.0f;
  }
}

// The sums over workers: 32 columns x 8 groups of workers per workgroup, joined in LDS in a fixed order.
template <typename T>
__global__ __launch_bounds__(256) void bn_columns_kernel(BnArgs a, int workers, bool token_gate, float* dw_post, float* dgate, float* dw_pre) {
  __shared__ float part[2][8][32];
  const int cx = threadIdx.x & 31, gy = threadIdx.x >> 5;
  const long long col = (long long)blockIdx.x * 32 + cx;
  const bool post = a.want_post || a.want_gate;
  float s0 = 0.0f, s1 = 0.0f;
  if (col < a.n) {
    const float* p = a.partial + col;
    const long long plane = (long long)workers * a.n;
    for (int w = gy; w < workers; w += 8) {
      if (post) s0 += p[w * a.n];
      if (a.want_pre) s1 += p[plane + w * a.n];
    }
  }
  part[0][gy][cx] = s0;
  part[1][gy][cx] = s1;
  __syncthreads();
  if (gy == 0 && col < a.n) {
    s0 = s1 = 0.0f;
    for (int i = 0; i < 8; i++) { s0 += part[0][i][cx]; s1 += part[1][i][cx]; }
    if (a.want_pre) dw_pre[col] = s1;
    if (token_gate) {
      if (a.want_post) dw_post[col] = s0;
    } else {
      // s0 = sum of scale dx b / rms(b)
      if (a.want_post) dw_post[col] = s0 * (float)static_cast<const T*>(a.gate)[col];
      if (a.want_gate) dgate[col] = s0 * (float)static_cast<const T*>(a.w_post)[col];
    }
  }
}

// ------------------------------------------------------------------ plan
constexpr int BN_WORKERS = 512;      // workgroups of the backward pass (two per compute unit)
constexpr long long BN_MAX_DIM = 1LL << 30;

// f(threads per row, pieces per thread, held) for rows of n elements
template <typename T, typename F>
void bn_shape(long long n, F&& f) {
  const long long pieces = (n + BN_VEC<T> - 1) / BN_VEC<T>;
  using std::integral_constant;
#define BN_CASE(TH, CHUNKS, H) f(integral_constant<int, TH>{}, integral_constant<int, CHUNKS>{}, integral_constant<bool, H>{})
  if (pieces <= 64) BN_CASE(64, 1, true);
  else if (pieces <= 128) BN_CASE(64, 2, true);
  else if (pieces <= 256) BN_CASE(256, 1, true);
  else if (pieces <= 512) BN_CASE(256, 2, true);
  else if (pieces <= 1024) BN_CASE(1024, 1, true);
  else if (pieces <= 2048) BN_CASE(1024, 2, true);
  else BN_CASE(1024, 2, false);
#undef BN_CASE
}

long long bn_row_groups(int threads, long long tokens) {
  const int rows = threads < 256 ? 256 / threads : 1;
  return (tokens + rows - 1) / rows;
}

template <typename T>
int run_forward(const BnArgs& a, hipStream_t stream) {
  bn_shape<T>(a.n, [&](auto th, auto ch, auto held) {
    mark(stream);
    launch(bn_forward_kernel<T, th.value, ch.value, held.value>, dim3((unsigned)bn_row_groups(th.value, a.tokens)),
           dim3(th.value < 256 ? 256 : th.value), stream, a);
  });
  mark(stream);
  return launch_status();
}

template <typename T>
int run_backward(const BnArgs& a, bool token_gate, float* dw_post, float* dgate, float* dw_pre, hipStream_t stream) {
  bn_shape<T>(a.n, [&](auto th, auto ch, auto held) {
    long long groups = bn_row_groups(th.value, a.tokens);
    if (groups > BN_WORKERS) groups = BN_WORKERS;
    const int workers = (int)groups * (th.value < 256 ? 256 / th.value : 1);
    const dim3 block(th.value < 256 ? 256 : th.value);
    if (groups > 0) {
      mark(stream);
      if (token_gate) launch(bn_backward_kernel<T, th.value, ch.value, held.value, true>, dim3((unsigned)groups), block, stream, a);
      else launch(bn_backward_kernel<T, th.value, ch.value, held.value, false>, dim3((unsigned)groups), block, stream, a);
    }
    if (a.want_post || a.want_gate || a.want_pre) {
      mark(stream);
      launch(bn_columns_kernel<T>, dim3((unsigned)((a.n + 31) / 32)), dim3(256), stream, a, workers, token_gate, dw_post, dgate, dw_pre);
    }
  });
  mark(stream);
  return launch_status();
}

int bn_check(int storage, const mlproj_norm_block* b) {
  if (!b) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16) return MLPROJ_ERR_BAD_VARIANT;
  if (b->tokens < 0 || b->n <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (b->tokens > BN_MAX_DIM || b->n > BN_MAX_DIM || (b->tokens > 0 && b->n > (1LL << 38) / b->tokens)) return MLPROJ_ERR_TOO_LARGE;
  if (!(b->eps >= 0.0f) || b->eps > 3.0e38f || !(b->scale - b->scale == 0.0f)) return MLPROJ_ERR_BAD_VALUE;
  return MLPROJ_OK;
}
int bn_array(const void* p, bool needed, long long row, long long ld, int es) {
  if (!p) return needed ? MLPROJ_ERR_NULL_POINTER : MLPROJ_OK;
  if (ld < row) return MLPROJ_ERR_BAD_DIMENSION;
  if (ld > BN_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  return aligned(p, es) ? MLPROJ_OK : MLPROJ_ERR_ALIGNMENT;
}
// the arrays both directions read
int bn_inputs(const mlproj_norm_block* k, int es) {
  const bool some = k->tokens > 0, block = k->w_post != nullptr;
  int st = block ? bn_array(k->b, some, k->n, k->ldb, es) : MLPROJ_OK;
  if (st == MLPROJ_OK) st = bn_array(k->w_post, false, k->n, k->n, es);
  if (st == MLPROJ_OK) st = bn_array(block ? k->gate : nullptr, some && block, k->n, k->gate_stride == 0 ? k->n : k->gate_stride, es);
  if (st == MLPROJ_OK) st = bn_array(k->w_pre, false, k->n, k->n, es);
  return st;
}
#define BN_TRY(x)                          \
  do {                                     \
    const int st_ = (x);                   \
    if (st_ != MLPROJ_OK) return st_;      \
  } while (0)

BnArgs bn_start(const mlproj_norm_block* k) {
  BnArgs a{};
  a.b = k->w_post ? k->b : nullptr; a.ldb = k->ldb;
  a.w_post = k->w_post; a.gate = k->gate; a.gate_stride = k->gate_stride; a.w_pre = k->w_pre;
  a.tokens = k->tokens; a.n = k->n;
  a.scale = k->scale; a.eps = k->eps;
  return a;
}

size_t bn_workspace(long long tokens, long long n) {
  // as many workers as the smallest rows take: four per workgroup
  const long long workers = tokens < 4 * BN_WORKERS ? (tokens + 3) / 4 * 4 : 4 * BN_WORKERS;
  const long long few = tokens < BN_WORKERS ? tokens : BN_WORKERS;
  // rows of at most 128 pieces take a wavefront each (1024 16-bit elements), longer ones a workgroup
  const long long w = n <= 1024 ? workers : few;
  return (size_t)(w > 0 ? w : 1) * n * 2 * sizeof(float) + 256;
}

}  // namespace
}  // namespace mlproj

using namespace mlproj;

extern "C" {

int block_norm_forward(int storage, const mlproj_norm_block* k, const void* x, long long ldx, void* r, long long ldr,
                       void* y, long long ldy, void* stream) {
  BN_TRY(bn_check(storage, k));
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool some = k->tokens > 0;
  BN_TRY(bn_inputs(k, es));
  BN_TRY(bn_array(x, some, k->n, ldx, es));
  BN_TRY(bn_array(r, some && k->w_post, k->n, ldr, es));
  BN_TRY(bn_array(y, some && k->w_pre, k->n, ldy, es));
  if (!some) return MLPROJ_OK;
  BnArgs a = bn_start(k);
  a.x = x; a.ldx = ldx; a.r = r; a.ldr = ldr; a.y = y; a.ldy = ldy;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return run_forward<float>(a, s);
  if (storage == MLPROJ_STORE_BF16) return run_forward<bf16_t>(a, s);
  return run_forward<f16_t>(a, s);
}

int mlproj_block_norm_workspace_bytes(long long tokens, long long n, size_t* bytes_out) {
  if (!bytes_out) return MLPROJ_ERR_NULL_POINTER;
  if (tokens < 0 || n <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (tokens > BN_MAX_DIM || n > BN_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  *bytes_out = bn_workspace(tokens, n);
  return MLPROJ_OK;
}

int block_norm_backward(int storage, const mlproj_norm_block* k, const void* r, long long ldr, const void* dr, long long lddr,
                        const void* dy, long long lddy, void* dx, long long lddx, void* db, long long lddb, float* dw_post,
                        void* dgate, long long dgate_stride, float* dw_pre, void* workspace, size_t workspace_bytes, void* stream) {
  BN_TRY(bn_check(storage, k));
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  const bool some = k->tokens > 0, block = k->w_post != nullptr, token_gate = k->gate_stride != 0;
  BN_TRY(bn_inputs(k, es));
  BN_TRY(bn_array(r, some, k->n, ldr, es));
  BN_TRY(bn_array(dr, false, k->n, lddr, es));
  BN_TRY(bn_array(dy, some && k->w_pre, k->n, lddy, es));
  BN_TRY(bn_array(dx, some, k->n, lddx, es));
  BN_TRY(bn_array(db, false, k->n, lddb, es));
  BN_TRY(bn_array(dw_post, false, k->n, k->n, 4));
  BN_TRY(bn_array(dgate, false, k->n, token_gate ? dgate_stride : k->n, token_gate ? es : 4));
  BN_TRY(bn_array(dw_pre, false, k->n, k->n, 4));
  if (!workspace) return MLPROJ_ERR_NULL_POINTER;
  if (workspace_bytes < bn_workspace(k->tokens, k->n) || !aligned(workspace, 256)) return MLPROJ_ERR_WORKSPACE;
  BnArgs a = bn_start(k);
  a.x = r; a.ldx = ldr; a.dr = dr; a.lddr = lddr; a.dy = dy; a.lddy = lddy;
  a.dx = dx; a.lddx = lddx; a.db = db; a.lddb = lddb;
  a.dgate = token_gate ? dgate : nullptr; a.dgate_stride = dgate_stride;
  a.partial = static_cast<float*>(workspace);
  a.want_post = block && dw_post;
  a.want_gate = block && !token_gate && dgate;
  a.want_pre = k->w_pre && dw_pre;
  float* dg = token_gate ? nullptr : static_cast<float*>(dgate);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return run_backward<float>(a, token_gate, dw_post, dg, dw_pre, s);
  if (storage == MLPROJ_STORE_BF16) return run_backward<bf16_t>(a, token_gate, dw_post, dg, dw_pre, s);
  return run_backward<f16_t>(a, token_gate, dw_post, dg, dw_pre, s);
}

}  // extern "C"
