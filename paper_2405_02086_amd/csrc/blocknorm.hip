// mlproj: the norms before and after a block, fused with its gate and the residual scale; kernels, plan and C ABI.
#include "ffcommon.h"
#include "host.h"

namespace mlproj {
namespace {

// ------------------------------------------------------------------ rows in registers
// A row's entries are dealt in pieces of 16 bytes: piece i of a row belongs to thread i % THREADS of the row's threads (16, a
// wavefront, or a workgroup of 256 or 512), CH of them per thread, and stays in its registers from the one load to the one store.
// Both directions are bound by HBM: forward reads x and b and writes r and y once, backward reads four
// arrays and writes two.  A row group takes many rows: the vectors (weights, a gate per channel) stay in registers
// too, and the next row's loads go out before the present row is reduced, as far as there are registers for it.
// 64M entries, bf16, one gate per channel: rows of 4096 take 99 us forward (5.4 TB/s) and 166 backward (4.9), of 8192 98 and
// 164, of 3000 114 and 178, of 3003 (rows no longer start on 16 bytes) 151 and 208, of 16384 (no room for the next row) 135 and 236.
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
  for (int s = 1; s < (THREADS < 64 ? THREADS : 64); s <<= 1)
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

constexpr int BN_LONG = 512;
// Rows too long for registers: CH pieces per thread at a time, and every phase reads them again (from L2, where a row
// still is).
template <typename T>
__global__ __launch_bounds__(BN_LONG) void bn_forward_long_kernel(BnArgs a) {
  constexpr int THREADS = BN_LONG, CH = 2;
  constexpr int VEC = BN_VEC<T>;
  __shared__ float slots[2][1][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = threadIdx.x;
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* b = a.b ? static_cast<const T*>(a.b) + row * a.ldb : nullptr;
  const T* gate = static_cast<const T*>(a.gate) + row * a.gate_stride;
  const T* w_post = static_cast<const T*>(a.w_post);
  const T* w_pre = static_cast<const T*>(a.w_pre);
  T* r = static_cast<T*>(a.r) + row * a.ldr;
  T* y = static_cast<T*>(a.y) + row * a.ldy;
  const long long n = a.n, per = (long long)THREADS * VEC * CH;
  const long long passes = (n + per - 1) / per;
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
  }
  float rr = 0.0f;
  if (w_pre) {
    sum[0] = 0.0f;
    for (long long pass = 0; pass < passes; pass++) {
      load(pass);
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
    load(pass);
    if (b) join(pass);
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

template <typename T, bool TOKEN_GATE>
__global__ __launch_bounds__(BN_LONG) void bn_backward_long_kernel(BnArgs a) {
  constexpr int THREADS = BN_LONG, CH = 2;
  constexpr int VEC = BN_VEC<T>;
  __shared__ float slots[2][6][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = threadIdx.x;
  const long long n = a.n, per = (long long)THREADS * VEC * CH;
  const long long passes = (n + per - 1) / per;
  const float inv_n = 1.0f / (float)n;
  const T* w_post = static_cast<const T*>(a.w_post);
  const T* w_pre = static_cast<const T*>(a.w_pre);
  const long long worker = blockIdx.x;
  const long long workers = gridDim.x;
  float* partial = a.partial + worker * n;
  const long long plane = workers * n;
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
      load(pass);
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

// ------------------------------------------------------------------ held rows
// A piece is 16 bytes of neighbouring entries, as it lies in memory, zeros past the row's end; and as numbers.  (fp32 rows
// that do not start on 16 bytes went entry by entry before partial pieces stopped being waited for: rows of 2047, 2049 or 4095
// are 2 to 8 % faster that way, rows of 513, 1001 or 3003 16 to 30 % slower, and a second set of kernels is not worth it.)
// (A piece wholly past the end must not take the path of a partial one: its entries, put together one by one, are waited for
// there, and with them the next row's loads.  64M entries in rows of 5000 bf16, backward: 304 -> 204 us.)
template <typename T>
__device__ __forceinline__ u32x4 bn_raw(const T* p, long long valid) {
  constexpr int VEC = BN_VEC<T>;
  u32x4 r = {};
  if (valid >= VEC) {
    __builtin_memcpy(&r, p, 16);
  } else if (valid > 0) {
    T t[VEC];
#pragma unroll
    for (int i = 0; i < VEC; i++) t[i] = i < valid ? p[i] : (T)0.0f;
    __builtin_memcpy(&r, t, 16);
  }
  return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void bn_numbers(u32x4 raw, float (&out)[VEC]) {
  T t[VEC];
  __builtin_memcpy(t, &raw, sizeof(t));
#pragma unroll
  for (int i = 0; i < VEC; i++) out[i] = (float)t[i];
}

// The pieces a thread holds of a row of an array (nothing where the array is absent), or of a vector.  `fetch` loads
// without waiting for anything: of a last piece that is not whole the row's last 16 bytes, which `settle` moves into place
// (64M entries in rows of 2047 bf16, backward: 317 -> 196 us).
template <typename T, int THREADS, int CH>
struct BnPieces {
  static constexpr int VEC = BN_VEC<T>;
  u32x4 raw[CH];
  __device__ __forceinline__ void load(const T* row, long long n, int t) {
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const long long at = ((long long)c * THREADS + t) * VEC;
      raw[c] = bn_raw<T>(row + at, row ? n - at : 0);
    }
  }
  template <bool AHEAD>
  __device__ __forceinline__ void fetch(const T* row, long long n, int t) {
    if (!AHEAD || n < VEC) {
      load(row, n, t);
      return;
    }
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const long long at = ((long long)c * THREADS + t) * VEC, first = at < n - VEC ? at : n - VEC;
      raw[c] = {};
      if (at < n) __builtin_memcpy(&raw[c], row + first, 16);
    }
  }
  template <bool AHEAD>
  __device__ __forceinline__ void settle(long long n, int t) {
    if constexpr (AHEAD) {
      if (n < VEC || n % VEC == 0) return;
#pragma unroll
      for (int c = 0; c < CH; c++) {
        const long long valid = n - ((long long)c * THREADS + t) * VEC;
        if (valid <= 0 || valid >= VEC) continue;
        // (VEC - valid) entries to the front: by two dwords, one, and half of one
        const int off = (int)(VEC - valid) * (int)sizeof(T);
        u32x4 w = raw[c];
        if (off & 8) w = u32x4{w[2], w[3], 0, 0};
        if (off & 4) w = u32x4{w[1], w[2], w[3], 0};
        if (off & 2) w = u32x4{__builtin_amdgcn_alignbit(w[1], w[0], 16), __builtin_amdgcn_alignbit(w[2], w[1], 16), __builtin_amdgcn_alignbit(w[3], w[2], 16), w[3] >> 16};
        raw[c] = w;
      }
    }
  }
};

template <int THREADS> constexpr int BN_GROUP = THREADS < 256 ? 256 : THREADS;   // threads of a workgroup
template <int THREADS> constexpr int BN_ROWS = BN_GROUP<THREADS> / THREADS;      // rows it has in hand

template <typename T, int THREADS, int CH, bool AHEAD>
__global__ __launch_bounds__(BN_GROUP<THREADS>) void bn_forward_kernel(BnArgs a) {
  constexpr int ROWS = BN_ROWS<THREADS>;
  using Pieces = BnPieces<T, THREADS, CH>;
  constexpr int VEC = BN_VEC<T>;
  __shared__ float slots[2][2][1][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = threadIdx.x % THREADS;
  const long long n = a.n, workers = (long long)gridDim.x * ROWS;
  const float inv_n = 1.0f / (float)n;
  const T *b = static_cast<const T*>(a.b), *gate = static_cast<const T*>(a.gate);
  const bool block = b != nullptr, pre = a.w_pre != nullptr, token_gate = a.gate_stride != 0;
  const T* x = static_cast<const T*>(a.x);
  const T *p_post = static_cast<const T*>(a.w_post), *p_pre = static_cast<const T*>(a.w_pre);
  Pieces w_post, w_pre, channel_gate, nx, nb, ng;
  // a piece of a vector: held, or read again
  auto piece = [&](const Pieces& held, const T* from, int c, float (&out)[VEC]) {
    const long long at = ((long long)c * THREADS + t) * VEC;
    bn_numbers<T, VEC>(AHEAD ? held.raw[c] : bn_raw<T>(from + at, from ? n - at : 0), out);
  };
  auto fetch = [&](long long row) {
    nx.template fetch<AHEAD>(x + row * a.ldx, n, t);
    if (block) nb.template fetch<AHEAD>(b + row * a.ldb, n, t);
    if (block && token_gate) ng.template fetch<AHEAD>(gate + row * a.gate_stride, n, t);
  };
  long long row = (long long)blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / THREADS : 0);
  if (row >= a.tokens) return;                 // (with THREADS > 64 the whole workgroup)
  fetch(row);
  if (AHEAD) {
    w_post.load(p_post, n, t);
    w_pre.load(p_pre, n, t);
    channel_gate.load(token_gate ? nullptr : gate, n, t);
  }
  for (int turn = 0; row < a.tokens; row += workers, turn ^= 1) {
    Pieces cx = nx, cb = nb, cg = ng;
    if (AHEAD && row + workers < a.tokens) fetch(row + workers);
    cx.template settle<AHEAD>(n, t);
    cb.template settle<AHEAD>(n, t);
    if (token_gate) cg.template settle<AHEAD>(n, t);
    float v[CH][VEC], sum[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < CH; c++) bn_numbers<T, VEC>(cx.raw[c], v[c]);
    if (block) {
#pragma unroll
      for (int c = 0; c < CH; c++) {
        float f[VEC];
        bn_numbers<T, VEC>(cb.raw[c], f);
#pragma unroll
        for (int i = 0; i < VEC; i++) sum[0] += f[i] * f[i];
      }
      bn_sum<THREADS, 1>(sum, slots[turn][0], lane, wave);
      const float rb = 1.0f / sqrtf(sum[0] * inv_n + a.eps);
#pragma unroll
      for (int c = 0; c < CH; c++) {
        float f[VEC], g[VEC], w[VEC];
        bn_numbers<T, VEC>(cb.raw[c], f);
        if (token_gate) bn_numbers<T, VEC>(cg.raw[c], g);
        else piece(channel_gate, gate, c, g);
        piece(w_post, p_post, c, w);
#pragma unroll
        for (int i = 0; i < VEC; i++) v[c][i] += a.scale * g[i] * (f[i] * rb * w[i]);
      }
    }
    float rr = 0.0f;
    if (pre) {
      sum[0] = 0.0f;
#pragma unroll
      for (int c = 0; c < CH; c++)
#pragma unroll
        for (int i = 0; i < VEC; i++) sum[0] += v[c][i] * v[c][i];
      bn_sum<THREADS, 1>(sum, slots[turn][1], lane, wave);
      rr = 1.0f / sqrtf(sum[0] * inv_n + a.eps);
    }
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const long long at = ((long long)c * THREADS + t) * VEC;
      if (at >= n) break;
      if (block) bn_store<T, VEC>(static_cast<T*>(a.r) + row * a.ldr + at, n - at, v[c]);
      if (pre) {
        float w[VEC];
        piece(w_pre, p_pre, c, w);
#pragma unroll
        for (int i = 0; i < VEC; i++) w[i] *= v[c][i] * rr;
        bn_store<T, VEC>(static_cast<T*>(a.y) + row * a.ldy + at, n - at, w);
      }
    }
    if (!AHEAD && row + workers < a.tokens) fetch(row + workers);
  }
}

// One round of sums per row: with e = w_pre dy and f = scale gate w_post,
//   mean(r e), mean(r^2), mean(b^2), and the three parts of sum(b f dx), dx = dr + rr e - r rr^3 mean(r e):
//   sum(b f dr), sum(b f e), sum(b f r).
// A worker (a row's threads) takes every workers-th row and keeps the sums over its rows of the columns its threads
// hold, which go out as one partial per workgroup and are summed, in their order, by bn_columns_kernel: the same bits
// every time.  With one gate per channel dgate and dw_post are both multiples of sum dx b / rms(b).
template <typename T, int THREADS, int CH, bool AHEAD, bool TOKEN_GATE>
__global__ __launch_bounds__(BN_GROUP<THREADS>) void bn_backward_kernel(BnArgs a) {
  constexpr int ROWS = BN_ROWS<THREADS>;
  using Pieces = BnPieces<T, THREADS, CH>;
  constexpr int VEC = BN_VEC<T>;
  __shared__ float slots[2][6][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = threadIdx.x % THREADS;
  const long long n = a.n;
  const float inv_n = 1.0f / (float)n;
  const long long worker = (long long)blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / THREADS : 0), workers = (long long)gridDim.x * ROWS;
  const T *r = static_cast<const T*>(a.x), *b = static_cast<const T*>(a.b), *dr = static_cast<const T*>(a.dr), *dy = static_cast<const T*>(a.dy);
  const T* gate = static_cast<const T*>(a.gate);
  const bool block = b != nullptr, pre = a.w_pre != nullptr;
  const T *p_post = static_cast<const T*>(a.w_post), *p_pre = static_cast<const T*>(a.w_pre);
  Pieces w_post, w_pre, channel_gate, nr, nb = {}, nd = {}, ny = {}, ng = {};
  auto piece = [&](const Pieces& held, const T* from, int c, float (&out)[VEC]) {
    const long long at = ((long long)c * THREADS + t) * VEC;
    bn_numbers<T, VEC>(AHEAD ? held.raw[c] : bn_raw<T>(from + at, from ? n - at : 0), out);
  };
  auto fetch = [&](long long row) {
    nr.template fetch<AHEAD>(r + row * a.ldx, n, t);
    if (block) nb.template fetch<AHEAD>(b + row * a.ldb, n, t);
    if (dr) nd.template fetch<AHEAD>(dr + row * a.lddr, n, t);
    if (pre) ny.template fetch<AHEAD>(dy + row * a.lddy, n, t);
    if (TOKEN_GATE && block) ng.template fetch<AHEAD>(gate + row * a.gate_stride, n, t);
  };
  // the sums of a thread's own columns: in registers, or in LDS where rows are long and registers few
  constexpr bool IN_LDS = THREADS >= 512;
  __shared__ float lds_sums[IN_LDS ? 2 * CH * VEC * THREADS : 1];
  float s_post[IN_LDS ? 1 : CH][VEC] = {}, s_pre[IN_LDS ? 1 : CH][VEC] = {};
  auto add = [&](int which, float (&held)[VEC], int c, int i, float x) {
    if (IN_LDS) lds_sums[((which * CH + c) * VEC + i) * THREADS + t] += x;
    else held[i] += x;
  };
  if (IN_LDS)
    for (int i = 0; i < 2 * CH * VEC; i++) lds_sums[i * THREADS + t] = 0.0f;
  if (worker < a.tokens) fetch(worker);
  if (AHEAD) {
    w_post.load(p_post, n, t);
    w_pre.load(p_pre, n, t);
    if (!TOKEN_GATE) channel_gate.load(gate, n, t);
  }
  int turn = 0;
  for (long long row = worker; row < a.tokens; row += workers, turn ^= 1) {
    Pieces cr = nr, cb = nb, cd = nd, cy = ny, cg = ng;
    if (AHEAD && row + workers < a.tokens) fetch(row + workers);
    for (Pieces* p : {&cr, &cb, &cd, &cy}) p->template settle<AHEAD>(n, t);
    if (TOKEN_GATE) cg.template settle<AHEAD>(n, t);
    float sum[6] = {};
#pragma unroll
    for (int c = 0; c < CH; c++) {
      float vr[VEC], vb[VEC], vd[VEC], vy[VEC], g[VEC], wp[VEC], wq[VEC];
      bn_numbers<T, VEC>(cr.raw[c], vr);
      bn_numbers<T, VEC>(cb.raw[c], vb);
      bn_numbers<T, VEC>(cd.raw[c], vd);
      bn_numbers<T, VEC>(cy.raw[c], vy);
      if (TOKEN_GATE) bn_numbers<T, VEC>(cg.raw[c], g);
      else piece(channel_gate, gate, c, g);
      piece(w_post, p_post, c, wp);
      piece(w_pre, p_pre, c, wq);
#pragma unroll
      for (int i = 0; i < VEC; i++) {
        const float e = wq[i] * vy[i], bf = vb[i] * (wp[i] * (a.scale * g[i]));
        sum[0] += vr[i] * e;
        sum[1] += vr[i] * vr[i];
        sum[2] += vb[i] * vb[i];
        sum[3] += bf * vd[i];
        sum[4] += bf * e;
        sum[5] += bf * vr[i];
      }
    }
    bn_sum<THREADS, 6>(sum, slots[turn], lane, wave);
    // Below, 16-bit entries are widened again: kept wide since the sums they would take twice the registers, more than there
    // are in rows past 8192 (4096 rows of 16384 bf16, gate per channel: 412 -> 234 us), or than two workgroups of a compute unit
    // have (64M entries in rows of 1024 bf16: 180 -> 165 us).  The statement keeps the compiler from it; elsewhere it costs
    // up to 6 %.
    if constexpr (sizeof(T) == 2 && (!AHEAD || THREADS == 64))
#pragma unroll
      for (int c = 0; c < CH; c++) asm volatile("" : "+v"(cr.raw[c]), "+v"(cb.raw[c]), "+v"(cd.raw[c]), "+v"(cy.raw[c]), "+v"(cg.raw[c]));
    const float rr = pre ? 1.0f / sqrtf(sum[1] * inv_n + a.eps) : 0.0f;
    const float rb = 1.0f / sqrtf(sum[2] * inv_n + a.eps);
    const float kr = pre ? rr * rr * rr * (sum[0] * inv_n) : 0.0f;
    const float kb = rb * rb * rb * ((sum[3] + rr * sum[4] - kr * sum[5]) * inv_n);
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const long long at = ((long long)c * THREADS + t) * VEC;
      if (at >= n) break;
      float vr[VEC], vd[VEC], vy[VEC], wq[VEC], dx[VEC];
      bn_numbers<T, VEC>(cr.raw[c], vr);
      bn_numbers<T, VEC>(cd.raw[c], vd);
      bn_numbers<T, VEC>(cy.raw[c], vy);
      piece(w_pre, p_pre, c, wq);
#pragma unroll
      for (int i = 0; i < VEC; i++) {
        dx[i] = vd[i] + (rr * (wq[i] * vy[i]) - kr * vr[i]);
        add(1, s_pre[IN_LDS ? 0 : c], c, i, vy[i] * (vr[i] * rr));
      }
      if (a.dx) bn_store<T, VEC>(static_cast<T*>(a.dx) + row * a.lddx + at, n - at, dx);
      if (block) {
        float vb[VEC], g[VEC], wp[VEC], db[VEC], dg[VEC];
        bn_numbers<T, VEC>(cb.raw[c], vb);
        if (TOKEN_GATE) bn_numbers<T, VEC>(cg.raw[c], g);
        else piece(channel_gate, gate, c, g);
        piece(w_post, p_post, c, wp);
#pragma unroll
        for (int i = 0; i < VEC; i++) {
          const float sdx = a.scale * dx[i], bh = vb[i] * rb;
          db[i] = rb * (sdx * g[i] * wp[i]) - kb * vb[i];
          dg[i] = sdx * wp[i] * bh;
          add(0, s_post[IN_LDS ? 0 : c], c, i, TOKEN_GATE ? sdx * g[i] * bh : sdx * bh);
        }
        if (a.db) bn_store<T, VEC>(static_cast<T*>(a.db) + row * a.lddb + at, n - at, db);
        if (TOKEN_GATE && a.dgate) bn_store<T, VEC>(static_cast<T*>(a.dgate) + row * a.dgate_stride + at, n - at, dg);
      }
    }
    if (!AHEAD && row + workers < a.tokens) fetch(row + workers);
  }
  float* partial = a.partial + blockIdx.x * n;
  const long long plane = gridDim.x * n;
  if constexpr (ROWS > 1) {
    // the workgroup's workers first, in their order
    __shared__ float rows[2][ROWS][CH * VEC * THREADS];
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
      for (int i = 0; i < VEC; i++) {
        const int at = (c * THREADS + t) * VEC + i;
        rows[0][threadIdx.x / THREADS][at] = s_post[c][i];
        rows[1][threadIdx.x / THREADS][at] = s_pre[c][i];
      }
    __syncthreads();
    for (int j = threadIdx.x; j < n; j += 256) {
      float post = 0.0f, own = 0.0f;
#pragma unroll
      for (int r = 0; r < ROWS; r++) { post += rows[0][r][j]; own += rows[1][r][j]; }
      if (a.want_post || a.want_gate) partial[j] = post;
      if (a.want_pre) partial[plane + j] = own;
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < CH; c++) {
    const long long at = ((long long)c * THREADS + t) * VEC;
    if (at >= n) break;
    float post[VEC], own[VEC];
#pragma unroll
    for (int i = 0; i < VEC; i++) {
      post[i] = IN_LDS ? lds_sums[(c * VEC + i) * THREADS + t] : s_post[IN_LDS ? 0 : c][i];
      own[i] = IN_LDS ? lds_sums[((CH + c) * VEC + i) * THREADS + t] : s_pre[IN_LDS ? 0 : c][i];
    }
    if (a.want_post || a.want_gate) bn_store<float, VEC>(partial + at, n - at, post);
    if (a.want_pre) bn_store<float, VEC>(partial + plane + at, n - at, own);
  }
}

// The sums over workgroups: 32 columns x 32 groups of them per workgroup here, joined in LDS in a fixed order.  Rows of more columns
// than a launch has threads for: the next ones a grid further on.
constexpr long long BN_MOST_COLUMN_GROUPS = 1 << 21;
template <typename T>
__global__ __launch_bounds__(1024) void bn_columns_kernel(BnArgs a, int workers, bool token_gate, float* dw_post, float* dgate, float* dw_pre) {
  __shared__ float part[2][32][33];
  const int cx = threadIdx.x & 31, gy = threadIdx.x >> 5;
  const bool post = a.want_post || a.want_gate;
  for (long long first = (long long)blockIdx.x * 32; first < a.n; first += (long long)gridDim.x * 32) {
    const long long col = first + cx;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 2; k++) {
      if (col >= a.n || !(k == 0 ? post : a.want_pre != 0)) continue;
      const float* p = a.partial + k * (long long)workers * a.n + col;
#pragma unroll 8
      for (int w = gy; w < workers; w += 32) s[k] += p[w * a.n];
    }
    part[0][gy][cx] = s[0];
    part[1][gy][cx] = s[1];
    __syncthreads();
    if (gy == 0 && col < a.n) {
      float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
      for (int i = 0; i < 32; i++) { s0 += part[0][i][cx]; s1 += part[1][i][cx]; }
      if (a.want_pre) dw_pre[col] = s1;
      if (token_gate) {
        if (a.want_post) dw_post[col] = s0;
      } else {
        // s0 = sum of scale dx b / rms(b); without tokens the gate need not be there, and may hold anything
        const bool some = workers > 0;
        if (a.want_post) dw_post[col] = some ? s0 * (float)static_cast<const T*>(a.gate)[col] : 0.0f;
        if (a.want_gate) dgate[col] = some ? s0 * (float)static_cast<const T*>(a.w_post)[col] : 0.0f;
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ plan
constexpr long long BN_MAX_DIM = 1LL << 30;
// Most workgroups of a pass: as many as are resident at once (two of 256 threads with up to 256 registers, one larger one,
// per compute unit), so that the next row's loads always have a row to hide behind and partial sums stay few.
constexpr long long bn_most_groups(int threads) { return threads <= 256 ? 512 : 256; }

// f(threads per row, pieces per thread, next row ahead) for rows of n entries; 0 pieces: too long for registers.
template <typename T, typename F>
void bn_shape(long long n, F&& f) {
  const long long pieces = (n + BN_VEC<T> - 1) / BN_VEC<T>;
  constexpr int WIDE = sizeof(T) == 4 ? 2 : 1;
  using std::integral_constant;
#define BN_CASE(TH, CHUNKS, AHEAD) f(integral_constant<int, TH>{}, integral_constant<int, CHUNKS>{}, integral_constant<bool, AHEAD>{})
  if (pieces <= 16) BN_CASE(16, 1, true);
  else if (pieces <= 32) BN_CASE(16, 2, true);
  else if (pieces <= 64) BN_CASE(64, 1, true);
  else if (pieces <= 128) BN_CASE(64, 2, true);
  else if (pieces <= 256) BN_CASE(256, 1, true);
  else if (pieces <= 512) BN_CASE(256, 2, true);
  else if (pieces <= 1024) BN_CASE(512 / WIDE, 2 * WIDE, true);
  else if (pieces <= 2048) BN_CASE(512, 4, false);
  else {
    if constexpr (WIDE == 2) {
      if (pieces <= 4096) {
        BN_CASE(512, 8, false);
        return;
      }
    }
    f(integral_constant<int, BN_LONG>{}, integral_constant<int, 0>{}, integral_constant<bool, false>{});
  }
#undef BN_CASE
}

long long bn_groups(int threads, long long tokens) {
  const int rows = threads < 256 ? 256 / threads : 1;
  const long long groups = (tokens + rows - 1) / rows, most = bn_most_groups(threads);
  return groups < most ? groups : most;
}

template <typename T>
int run_forward(const BnArgs& a, hipStream_t stream) {
  bn_shape<T>(a.n, [&](auto th, auto ch, auto ahead) {
    mark(stream);
    if constexpr (ch.value == 0)
      launch(bn_forward_long_kernel<T>, dim3((unsigned)a.tokens), dim3(BN_LONG), stream, a);
    else
      launch(bn_forward_kernel<T, th.value, ch.value, ahead.value>, dim3((unsigned)bn_groups(th.value, a.tokens)), dim3(BN_GROUP<th.value>), stream, a);
  });
  mark(stream);
  return launch_status();
}

template <typename T>
int run_backward(const BnArgs& a, bool token_gate, float* dw_post, float* dgate, float* dw_pre, hipStream_t stream) {
  bn_shape<T>(a.n, [&](auto th, auto ch, auto ahead) {
    const long long groups = bn_groups(th.value, a.tokens);
    const dim3 grid((unsigned)groups), block(BN_GROUP<th.value>);
    if (groups > 0) {
      mark(stream);
      if constexpr (ch.value == 0) {
        if (token_gate) launch(bn_backward_long_kernel<T, true>, grid, block, stream, a);
        else launch(bn_backward_long_kernel<T, false>, grid, block, stream, a);
      } else {
        if (token_gate) launch(bn_backward_kernel<T, th.value, ch.value, ahead.value, true>, grid, block, stream, a);
        else launch(bn_backward_kernel<T, th.value, ch.value, ahead.value, false>, grid, block, stream, a);
      }
    }
    if (a.want_post || a.want_gate || a.want_pre) {
      mark(stream);
      const long long columns = (a.n + 31) / 32;
      launch(bn_columns_kernel<T>, dim3((unsigned)(columns < BN_MOST_COLUMN_GROUPS ? columns : BN_MOST_COLUMN_GROUPS)), dim3(1024), stream, a, (int)groups, token_gate,
             dw_post, dgate, dw_pre);
    }
  });
  mark(stream);
  return launch_status();
}

int bn_check(int storage, const mlproj_norm_block* b) {
  if (!b) return MLPROJ_ERR_NULL_POINTER;
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16) return MLPROJ_ERR_BAD_VARIANT;
  if (b->tokens < 0 || b->n <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  // (rows too long for registers have a workgroup of 512 threads each: past 2^14 entries, 2^37 in all are less than 2^23 of them)
  if (b->tokens > BN_MAX_DIM || b->n > BN_MAX_DIM || (b->tokens > 0 && b->n > (1LL << 37) / b->tokens)) return MLPROJ_ERR_TOO_LARGE;
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
  const bool block = k->w_post != nullptr;     // without it b and gate are not used: the kernels go by these pointers
  a.b = block ? k->b : nullptr; a.ldb = k->ldb;
  a.w_post = k->w_post; a.w_pre = k->w_pre;
  a.gate = block ? k->gate : nullptr; a.gate_stride = block ? k->gate_stride : 0;
  a.tokens = k->tokens; a.n = k->n;
  a.scale = k->scale; a.eps = k->eps;
  return a;
}

size_t bn_workspace(long long tokens, long long n) {
  // the most workgroups any storage type has
  long long most = 1;
  auto count = [&](auto th, auto, auto) {
    const long long groups = bn_groups(th.value, tokens);
    most = groups > most ? groups : most;
  };
  bn_shape<bf16_t>(n, count);
  bn_shape<float>(n, count);
  return (size_t)most * n * 2 * sizeof(float) + 256;
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
