// mlproj: products of few tokens with weights in 4 bits and group scales: packing, the kernel and the C ABI.
#include "ffcommon.h"
#include "ffstaged.h"
#include "host.h"

namespace mlproj {
namespace {

constexpr int W4_ROWS = 128, W4_COLS = 16, W4_BYTES = 1024;   // a block: rows, columns, bytes of codes

struct W4Args {
  const unsigned char* codes[2];   // gate (or the one matrix), up
  const bf16_t* scales[2];
  const void* x;
  void* y;
  long long ldx, ldy, tokens;
  long long n, m;
  int kblocks, act;
};

// Eight codes as eight elements of the type the matrix cores take; exact in both.
__device__ __forceinline__ bf16x8 w4_widen(unsigned v, bf16_t) {
  typedef bf16_t pair_t __attribute__((ext_vector_type(2)));
  pair_t p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 1.0f, 1),
                 __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 1.0f, 3)};
  bf16x8 r;
  __builtin_memcpy(&r, p, 16);
  return r;
}
__device__ __forceinline__ f16x8 w4_widen(unsigned v, f16_t) {
  typedef f16_t pair_t __attribute__((ext_vector_type(2)));
  pair_t p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, 1.0f, 1),
                 __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, 1.0f, 3)};
  f16x8 r;
  __builtin_memcpy(&r, p, 16);
  return r;
}

// A workgroup computes CB x 16 columns (of one matrix, or of both) for up to 16 MT tokens; its wavefronts share out the
// row blocks, U at a time, and join their sums in LDS, in their order.  A wavefront's load of a block is 1 KiB in one
// instruction, already in the layout of the matrix cores' second operand, and the hardware widens two codes per instruction; a
// group's sum leaves the matrix cores unscaled, in the lane that holds its column's scale.  fp32 tokens are cut into
// three bf16 parts (ffstaged.h), which with weights of two significant bits loses nothing.  Cut that way an infinity leaves a NaN; keeping
// it apart costs a call of one token 15 %, so a workgroup does that only in a second run, if a NaN came out of the first (to look
// for one costs 4 %).
//
// Bound by HBM at one token where there are columns enough: n m / 2 bytes of codes and 2 n m / group of scales; where there are few, by
// the rounds of loads that a wavefront waits for (16384 -> 4096, weights in the memory-side cache: one token, four rounds of two
// blocks, 8.7 us; sixteen, which every workgroup reads from L2, 128 rows of them 4 KiB and of a column block 1 KiB, eight rounds, 10.4).
// So: one column block per
// workgroup and 16 wavefronts while that is what fills the chip, two where there are columns enough, four (and 32
// tokens) where the tokens dominate.  us, with 1 x 16 / 2 x 8 / 4 x 8 (column blocks x wavefronts): one token 16384 ->
// 4096 10.8 / 14 / 22, one token 4096 -> 2 x 16384 18 / 14 / 17, 16 tokens 4096 -> 2 x 16384 24 / 17 / 17, 16 tokens 16384
// -> 8192 26 / 20 / 24; 64 tokens 4096 -> 2 x 16384 65 / 44 / 49, with 32 tokens at a time 34.
//
// A row block's tokens are loaded in whole rows, 256 bytes (fp32: 512) of one after the other, and turned into operands through
// a corner of LDS that belongs to the wavefront (VIA_LDS): loading operands straight, lane l token l % 16, every four
// lanes touch four cache lines, and at 16 tokens the lookups cost more than the weights (16384 -> 4096, groups of 32: 18.7
// us).  With at most four tokens the lines are few and the straight way is shorter.
template <typename T, bool GATED, int MT, int CB, int U, int WAVES, int GROUP, bool VIA_LDS>
__global__ __launch_bounds__(WAVES * 64) void w4_kernel(W4Args a) {
  using E = typename FfParts<T>::type;
  using F = typename FfFrag<E>::type;
  constexpr int P = FfParts<T>::count, MATS = GATED ? 2 : 1, PER = W4_ROWS / GROUP, SETS = CB * MATS;
  // tokens in whole rows: 16-byte pieces of a row, rows a load covers, loads
  constexpr int VEC = 16 / sizeof(T), PIECES = W4_ROWS / VEC, ROWS = 64 / PIECES, XLOADS = 16 * MT / ROWS;
  constexpr int HELD = VIA_LDS ? 16 * MT * PIECES : 0, SUMS = SETS * MT * 64;      // 16-byte pieces per row block, per wavefront
  __shared__ u32x4 lds[WAVES * (U * HELD > SUMS ? U * HELD : SUMS)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long cb0 = (long long)blockIdx.x * CB, t0 = (long long)blockIdx.y * (16 * MT);
  const long long cbs = (a.m + W4_COLS - 1) / W4_COLS;
  const T* x = static_cast<const T*>(a.x);
  f32x4 acc[SETS][MT] = {};
  auto run = [&](auto infinities) {
    for (int kb = wave; kb < a.kblocks; kb += WAVES * U) {
      u32x4 w[U][SETS];
      bf16_t s[U][SETS][PER];
      F xf[U][VIA_LDS ? 1 : MT][P][4];
      u32x4 xr[U][VIA_LDS ? XLOADS : 1];
#pragma unroll
      for (int u = 0; u < U; u++) {
        // past the end: the last block again, not used
        const int k = kb + u * WAVES < a.kblocks ? kb + u * WAVES : a.kblocks - 1;
#pragma unroll
        for (int i = 0; i < SETS; i++) {
          const long long cb = cb0 + i % CB < cbs ? cb0 + i % CB : cbs - 1, at = cb * a.kblocks + k;
          w[u][i] = *reinterpret_cast<const u32x4*>(a.codes[i / CB] + at * W4_BYTES + lane * 16);
          __builtin_memcpy(s[u][i], a.scales[i / CB] + (at * 16 + (lane & 15)) * PER, PER * 2);
        }
        const bool whole = (k + 1) * W4_ROWS <= a.n;
        // (rows past the tokens are the last one again: what they come to is not stored)
        if constexpr (VIA_LDS) {
#pragma unroll
          for (int j = 0; j < XLOADS; j++) {
            const long long t = t0 + j * ROWS + lane / PIECES;
            const int at = k * W4_ROWS + lane % PIECES * VEC;
            const T* from = x + (t < a.tokens ? t : a.tokens - 1) * a.ldx + at;
            if (whole) {
              __builtin_memcpy(&xr[u][j], from, 16);
            } else {
              T v[VEC];
#pragma unroll
              for (int i = 0; i < VEC; i++) v[i] = at + i < a.n ? from[i] : (T)0.0f;
              __builtin_memcpy(&xr[u][j], v, 16);
            }
          }
        } else {
#pragma unroll
          for (int mt = 0; mt < MT; mt++) {
            const long long t = t0 + mt * 16 + (lane & 15);
            const T* row = x + (t < a.tokens ? t : a.tokens - 1) * a.ldx;
#pragma unroll
            for (int q = 0; q < 4; q++) {
              const int at = k * W4_ROWS + q * 32 + (lane >> 4) * 8;
              u32x4 parts[P];
              fs_parts<T, infinities.value>(ff_load8(row + at, whole ? 8 : a.n - at), parts);
#pragma unroll
              for (int p = 0; p < P; p++) __builtin_memcpy(&xf[u][mt][p][q], &parts[p], 16);
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; u++) {
        if (kb + u * WAVES >= a.kblocks) break;
        u32x4* mine = lds + (wave * U + u) * HELD;
        if constexpr (VIA_LDS) {
          // (pieces permuted by the row's number: eight rows' pieces spread over all banks)
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
          for (int j = 0; j < XLOADS; j++) {
            const int r = j * ROWS + lane / PIECES;
            mine[r * PIECES + (lane % PIECES ^ (r & 7))] = xr[u][j];
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          __builtin_amdgcn_wave_barrier();
        }
        f32x4 part[SETS][MT] = {};
#pragma unroll
        for (int q = 0; q < 4; q++) {
          F xq[MT][P];
#pragma unroll
          for (int mt = 0; mt < MT; mt++) {
            if constexpr (VIA_LDS) {
              FfVec8<T> v;
              constexpr int EACH = 8 / VEC;
              const int r = mt * 16 + (lane & 15);
#pragma unroll
              for (int e = 0; e < EACH; e++) {
                const u32x4 piece = mine[r * PIECES + (((q * 4 + (lane >> 4)) * EACH + e) ^ (r & 7))];
                __builtin_memcpy(&v.v[e * VEC], &piece, 16);
              }
              u32x4 parts[P];
              fs_parts<T, infinities.value>(v, parts);
#pragma unroll
              for (int p = 0; p < P; p++) __builtin_memcpy(&xq[mt][p], &parts[p], 16);
            } else {
#pragma unroll
              for (int p = 0; p < P; p++) xq[mt][p] = xf[u][VIA_LDS ? 0 : mt][p][q];
            }
          }
#pragma unroll
          for (int i = 0; i < SETS; i++) {
            const F wf = w4_widen(w[u][i][q], E{});
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
#pragma unroll
              for (int p = P - 1; p >= 0; p--) part[i][mt] = ff_mfma(xq[mt][p], wf, part[i][mt]);
              if ((q + 1) * 32 % GROUP == 0) {
                acc[i][mt] += (float)s[u][i][q * 32 / GROUP] * part[i][mt];
                part[i][mt] = f32x4{};
              }
            }
          }
        }
      }
    }
  };
  run(std::false_type{});
  if constexpr (P > 1) {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < SETS; i++)
#pragma unroll
      for (int mt = 0; mt < MT; mt++)
#pragma unroll
        for (int v = 0; v < 4; v++) nan = nan || acc[i][mt][v] != acc[i][mt][v];
    if (__syncthreads_or(nan)) {
#pragma unroll
      for (int i = 0; i < SETS; i++)
#pragma unroll
        for (int mt = 0; mt < MT; mt++) acc[i][mt] = f32x4{};
      run(std::true_type{});
    }
  }
  if (VIA_LDS) __syncthreads();                 // the sums take the tokens' place
  f32x4* sums = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int i = 0; i < SETS; i++)
#pragma unroll
    for (int mt = 0; mt < MT; mt++) sums[((wave * SETS + i) * MT + mt) * 64 + lane] = acc[i][mt];
  __syncthreads();
  // entry e of a set: token e / 16, column e % 16; it is value (e / 16) % 4 of lane 16 (e / 64) + e % 16
  for (int e = threadIdx.x; e < CB * MT * 256; e += WAVES * 64) {
    const int c = e / (MT * 256), f = e % (MT * 256), mt = f >> 8, in = f & 255, src = (in >> 6) * 16 + (in & 15), v = (in >> 4) & 3;
    const long long t = t0 + f / 16, col = (cb0 + c) * W4_COLS + (in & 15);
    if (t >= a.tokens || col >= a.m) continue;
    float r[MATS] = {};
#pragma unroll
    for (int i = 0; i < MATS; i++)
#pragma unroll
      for (int k = 0; k < WAVES; k++) r[i] += sums[((k * SETS + i * CB + c) * MT + mt) * 64 + src][v];
    float out = r[0];
    if constexpr (GATED) {
      f32x4 value, slope;
      ff_gate4<sizeof(T) == 4>(a.act, f32x4{r[0], 0.0f, 0.0f, 0.0f}, value, slope);
      out = value[0] * r[MATS - 1];
    }
    static_cast<T*>(a.y)[t * a.ldy + col] = ff_round<T>(out);
  }
}

// One thread per column and group.
template <typename T>
__global__ __launch_bounds__(256) void w4_pack_kernel(const T* W, long long ldw, long long n, long long m, int group,
                                                      unsigned* codes, bf16_t* scales, int kblocks, long long columns) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const int per = W4_ROWS / group;
  if (i >= columns * kblocks * per) return;
  const long long col = i % columns, g = i / columns, kb = g / per;
  const int gi = (int)(g % per);
  const long long row0 = g * group;
  const T* w = W + row0 * ldw + col;
  const long long rows = col >= m || row0 >= n ? 0 : (n - row0 < group ? n - row0 : group);
  float top = 0.0f;
  for (long long r = 0; r < rows; r++) {
    const float size = fabsf((float)w[r * ldw]);
    top = size > top || size != size ? size : top;       // a NaN stays: the scale is NaN then, and with it the products
  }
  const bf16_t rounded = (bf16_t)(top / 6.0f);
  const float scale = (float)rounded;
  const long long block = (col / W4_COLS) * kblocks + kb;
  scales[(block * 16 + col % W4_COLS) * per + gi] = rounded;
  for (int q = gi * group / 32; q < (gi + 1) * group / 32; q++) {
    for (int hi = 0; hi < 4; hi++) {
      unsigned word = 0;
      for (int j = 0; j < 8; j++) {
        const long long r = q * 32 + hi * 8 + j - (long long)gi * group;
        if (r >= rows) continue;
        const float value = (float)w[r * ldw];
        const float v = scale > 0.0f ? fabsf(value) / scale : 0.0f;
        unsigned code = (v > 0.25f) + (v > 0.75f) + (v > 1.25f) + (v > 1.75f) + (v > 2.5f) + (v > 3.5f) + (v > 5.0f);
        if (value < 0.0f) code |= 8;
        word |= code << (4 * j);
      }
      codes[block * (W4_BYTES / 4) + (hi * 16 + col % W4_COLS) * 4 + q] = word;
    }
  }
}

constexpr long long W4_MAX_DIM = 1LL << 30;
#define W4_TRY(x)                          \
  do {                                     \
    const int st_ = (x);                   \
    if (st_ != MLPROJ_OK) return st_;      \
  } while (0)

int w4_check(const mlproj_w4* w, bool arrays) {
  if (!w) return MLPROJ_ERR_NULL_POINTER;
  if (w->group != 32 && w->group != 64 && w->group != 128) return MLPROJ_ERR_BAD_VARIANT;
  if (w->n <= 0 || w->m <= 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (w->n > W4_MAX_DIM || w->m > W4_MAX_DIM || w->n > (1LL << 38) / w->m) return MLPROJ_ERR_TOO_LARGE;
  if (!arrays) return MLPROJ_OK;
  if (!w->codes || !w->scales) return MLPROJ_ERR_NULL_POINTER;
  return aligned(w->codes, 16) && aligned(w->scales, 8) ? MLPROJ_OK : MLPROJ_ERR_ALIGNMENT;
}
int w4_array(const void* p, bool needed, long long row, long long ld, int es) {
  if (!p) return needed ? MLPROJ_ERR_NULL_POINTER : MLPROJ_OK;
  if (ld < row) return MLPROJ_ERR_BAD_DIMENSION;
  if (ld > W4_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  return aligned(p, es) ? MLPROJ_OK : MLPROJ_ERR_ALIGNMENT;
}

// Column blocks that a launch of less than 2^32 threads takes: workgroups of so many have 512 threads and two blocks, or four
// with at least 8 tokens (w4_run).
bool w4_fits(long long m, long long tokens) { return (m + W4_COLS - 1) / W4_COLS <= (tokens >= 8 ? (1LL << 25) - 4 : (1LL << 24) - 2); }

template <typename T, bool GATED, int MT, int CB, int U, int WAVES, bool VIA_LDS>
void w4_launch(const W4Args& a, int group, hipStream_t stream) {
  const long long cbs = (a.m + W4_COLS - 1) / W4_COLS;
  const dim3 grid((unsigned)((cbs + CB - 1) / CB), (unsigned)((a.tokens + 16 * MT - 1) / (16 * MT))), block(WAVES * 64);
  mark(stream);
  if (group == 32) launch(w4_kernel<T, GATED, MT, CB, U, WAVES, 32, VIA_LDS>, grid, block, stream, a);
  else if (group == 64) launch(w4_kernel<T, GATED, MT, CB, U, WAVES, 64, VIA_LDS>, grid, block, stream, a);
  else launch(w4_kernel<T, GATED, MT, CB, U, WAVES, 128, VIA_LDS>, grid, block, stream, a);
}

template <typename T, bool GATED>
int w4_run(const W4Args& a, int group, hipStream_t stream) {
  // a grid has at most 65535 workgroups along y: more tokens than they take go out in several launches
  constexpr long long MOST = 65535LL * 16;
  W4Args b = a;
  for (long long t = 0; t < a.tokens; t += MOST) {
    b.tokens = a.tokens - t < MOST ? a.tokens - t : MOST;
    b.x = static_cast<const T*>(a.x) + t * a.ldx;
    b.y = static_cast<T*>(a.y) + t * a.ldy;
    const long long cbs = (a.m + W4_COLS - 1) / W4_COLS, groups = cbs * ((b.tokens + 15) / 16);
    if (sizeof(T) == 2 && b.tokens > 16 && cbs * ((b.tokens + 31) / 32) >= 1024) {
      if constexpr (sizeof(T) == 2) w4_launch<T, GATED, 2, 4, 1, 8, false>(b, group, stream);
    } else if (groups >= 1024 && b.tokens >= 8) {
      w4_launch<T, GATED, 1, 4, 1, 8, false>(b, group, stream);
    } else if (groups >= 512) {
      if (b.tokens > 4) w4_launch<T, GATED, 1, 2, 1, 8, true>(b, group, stream);
      else w4_launch<T, GATED, 1, 2, 2, 8, false>(b, group, stream);
    } else {
      if (b.tokens > 4) w4_launch<T, GATED, 1, 1, 1, 16, true>(b, group, stream);
      else w4_launch<T, GATED, 1, 1, 2, 16, false>(b, group, stream);
    }
  }
  mark(stream);
  return launch_status();
}

int w4_product(int storage, int act, const mlproj_w4* g, const mlproj_w4* u, const void* x, long long ldx, long long tokens,
               void* y, long long ldy, void* stream) {
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16 || act < MLPROJ_ACT_SILU || act > MLPROJ_ACT_RELU) return MLPROJ_ERR_BAD_VARIANT;
  if (tokens < 0) return MLPROJ_ERR_BAD_DIMENSION;
  if (tokens > W4_MAX_DIM) return MLPROJ_ERR_TOO_LARGE;
  W4_TRY(w4_check(g, tokens > 0));
  if (u) {
    W4_TRY(w4_check(u, tokens > 0));
    if (u->n != g->n || u->m != g->m || u->group != g->group) return MLPROJ_ERR_BAD_DIMENSION;
  }
  const int es = storage == MLPROJ_STORE_F32 ? 4 : 2;
  W4_TRY(w4_array(x, tokens > 0, g->n, ldx, es));
  W4_TRY(w4_array(y, tokens > 0, g->m, ldy, es));
  if (tokens == 0) return MLPROJ_OK;
  if (!w4_fits(g->m, tokens)) return MLPROJ_ERR_TOO_LARGE;
  W4Args a{};
  a.codes[0] = static_cast<const unsigned char*>(g->codes);
  a.scales[0] = static_cast<const bf16_t*>(g->scales);
  if (u) {
    a.codes[1] = static_cast<const unsigned char*>(u->codes);
    a.scales[1] = static_cast<const bf16_t*>(u->scales);
  }
  a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.tokens = tokens;
  a.n = g->n; a.m = g->m; a.act = act;
  a.kblocks = (int)((g->n + W4_ROWS - 1) / W4_ROWS);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (storage == MLPROJ_STORE_F32) return u ? w4_run<float, true>(a, g->group, s) : w4_run<float, false>(a, g->group, s);
  if (storage == MLPROJ_STORE_BF16) return u ? w4_run<bf16_t, true>(a, g->group, s) : w4_run<bf16_t, false>(a, g->group, s);
  return u ? w4_run<f16_t, true>(a, g->group, s) : w4_run<f16_t, false>(a, g->group, s);
}

}  // namespace
}  // namespace mlproj

using namespace mlproj;

extern "C" {

int mlproj_w4_bytes(long long n, long long m, int group, size_t* codes_out, size_t* scales_out) {
  if (!codes_out || !scales_out) return MLPROJ_ERR_NULL_POINTER;
  const mlproj_w4 w = {n, m, group, nullptr, nullptr};
  W4_TRY(w4_check(&w, false));
  const size_t blocks = (size_t)((m + W4_COLS - 1) / W4_COLS) * (size_t)((n + W4_ROWS - 1) / W4_ROWS);
  *codes_out = blocks * W4_BYTES;
  *scales_out = blocks * 16 * (W4_ROWS / group) * 2;
  return MLPROJ_OK;
}

int w4_pack(int storage, const void* W, long long ldw, const mlproj_w4* packed, void* stream) {
  if (storage < MLPROJ_STORE_F32 || storage > MLPROJ_STORE_F16) return MLPROJ_ERR_BAD_VARIANT;
  W4_TRY(w4_check(packed, true));
  W4_TRY(w4_array(W, true, packed->m, ldw, storage == MLPROJ_STORE_F32 ? 4 : 2));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const long long columns = (packed->m + W4_COLS - 1) / W4_COLS * W4_COLS;
  const int kblocks = (int)((packed->n + W4_ROWS - 1) / W4_ROWS);
  const long long threads = columns * kblocks * (W4_ROWS / packed->group);
  if ((threads + 255) / 256 >= 1LL << 24) return MLPROJ_ERR_TOO_LARGE;      // 2^32 threads in a launch
  const dim3 grid((unsigned)((threads + 255) / 256));
  unsigned* codes = static_cast<unsigned*>(const_cast<void*>(packed->codes));
  bf16_t* scales = static_cast<bf16_t*>(const_cast<void*>(packed->scales));
  mark(s);
  if (storage == MLPROJ_STORE_F32) launch(w4_pack_kernel<float>, grid, dim3(256), s, static_cast<const float*>(W), ldw, packed->n, packed->m, packed->group, codes, scales, kblocks, columns);
  else if (storage == MLPROJ_STORE_BF16) launch(w4_pack_kernel<bf16_t>, grid, dim3(256), s, static_cast<const bf16_t*>(W), ldw, packed->n, packed->m, packed->group, codes, scales, kblocks, columns);
  else launch(w4_pack_kernel<f16_t>, grid, dim3(256), s, static_cast<const f16_t*>(W), ldw, packed->n, packed->m, packed->group, codes, scales, kblocks, columns);
  mark(s);
  return launch_status();
}

int w4_matvec(int storage, const mlproj_w4* W, const void* x, long long ldx, long long tokens, void* y, long long ldy, void* stream) {
  return w4_product(storage, MLPROJ_ACT_SILU, W, nullptr, x, ldx, tokens, y, ldy, stream);
}

int w4_gated_matvec(int storage, int activation, const mlproj_w4* Wg, const mlproj_w4* Wu, const void* x, long long ldx,
                    long long tokens, void* h, long long ldh, void* stream) {
  if (!Wu) return MLPROJ_ERR_NULL_POINTER;
  return w4_product(storage, activation, Wg, Wu, x, ldx, tokens, h, ldh, stream);
}

}  // extern "C"
