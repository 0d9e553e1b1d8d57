// Root-mean-square norm in front of the layer, with the addition of the residual, the E4M3 codes of the result for the FP8
// form of the expert GEMMs (one scale per row, largest magnitude / 448; code = cvt(y / scale)) and the gradients.
//
//   forward   s = round(x + residual),  rstd = (mean(s^2) + eps)^-1/2,  y = s rstd w
//   backward  a = dy w,  dx = rstd (a - s rstd^2 mean(a s)) + dsum,  dw = sum over the rows of dy s rstd
//
// Bound by HBM: a handful of fp32 operations per element read.  A row stays in the registers of its threads from its one read
// to its writes, but for two forms of the gradients that read it twice, from the caches: rows of more than 32 KiB, and the weight's
// gradient of few rows.  Statistics and all sums are fp32, and what is stored in the element type is rounded once.
#include <algorithm>
#include <initializer_list>

#include "forward_types.h"

namespace moe355 {

constexpr int kNormMaxCols = 32768;

// Sixteen bytes of a row.
template <typename T>
struct Piece {
  static constexpr int N = 16 / sizeof(T);
  uint4 raw;
  __device__ __forceinline__ void load(const T *p) { raw = *reinterpret_cast<const uint4 *>(p); }
  // with the non-temporal hint: what is read for the last time
  __device__ __forceinline__ void load_last(const T *p) {
    raw = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)));
  }
  __device__ __forceinline__ void zero() { raw = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[N]) {
    if constexpr (sizeof(T) == 4) {
      return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    } else {
      bf16x8 o;
#pragma unroll
      for (int q = 0; q < 8; ++q) o[q] = (bf16_t)v[q];
      return __builtin_bit_cast(uint4, o);
    }
  }
};

// Sum or maximum over the WAVES waves of a row; `slot` (LDS) is not used again before the next barrier but one.
template <int WAVES, typename V, typename OP>
__device__ __forceinline__ V row_reduce(V v, V *slot, OP op) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = op(v, __shfl_xor(v, off));
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    const int first = (threadIdx.x >> 6) / WAVES * WAVES;
    v = slot[first];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v = op(v, slot[first + i]);
  }
  return v;
}
struct AddF { __device__ float operator()(float a, float b) const { return a + b; } };
struct MaxU { __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; } };

struct NormArgs {
  const void *x, *residual, *weight;
  void *sum, *y;
  uint8_t *codes;
  float *scales, *rstd;
  int64_t rows;
  int cols;
  float eps, inv_cols;
};

// WAVES waves (1: four rows a workgroup, each its own wave; else one row a workgroup) with CHUNKS sixteen-byte pieces a thread.
// 4096 x 7168 in bf16 with residual, sum, y and codes: 49 us, 5.4 TB/s of what it has to move; one row 3.2 us.
template <typename T, int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void rmsnorm_kernel(const NormArgs a) {
  constexpr int N = Piece<T>::N, STRIDE = WAVES * 64 * N;
  __shared__ float sums[WAVES == 1 ? 1 : WAVES];
  __shared__ uint32_t tops[WAVES == 1 ? 1 : WAVES];
  const int t = WAVES == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * (WAVES == 1 ? 4 : 1) + (WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  if (row >= a.rows) return;  // (whole waves; with several waves a row never)
  const int64_t base = row * a.cols;
  const T *x = static_cast<const T *>(a.x) + base;
  const T *res = a.residual ? static_cast<const T *>(a.residual) + base : nullptr;
  const T *wt = static_cast<const T *>(a.weight);
  Piece<T> v[CHUNKS], w[CHUNKS];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int c = t * N + i * STRIDE;
    if (c < a.cols) v[i].load(x + c); else v[i].zero();
  }
  if (res) {
    Piece<T> r[CHUNKS];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = t * N + i * STRIDE;
      if (c < a.cols) r[i].load_last(res + c); else r[i].zero();
    }
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = t * N + i * STRIDE;
      float s[N];
#pragma unroll
      for (int q = 0; q < N; ++q) s[q] = v[i].get(q) + r[i].get(q);
      v[i].raw = Piece<T>::pack(s);  // the norm is that of the stored sum
      if (a.sum && c < a.cols) *reinterpret_cast<uint4 *>(static_cast<T *>(a.sum) + base + c) = v[i].raw;
    }
  }
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int c = t * N + i * STRIDE;
    if (c < a.cols) w[i].load(wt + c); else w[i].zero();
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
    for (int q = 0; q < N; ++q) ss = fmaf(v[i].get(q), v[i].get(q), ss);
  ss = row_reduce<WAVES>(ss, sums, AddF());
  const float rstd = 1.0f / sqrtf(fmaf(ss, a.inv_cols, a.eps));
  if (a.rstd && t == 0) a.rstd[row] = rstd;
  if (a.y) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = t * N + i * STRIDE;
      float o[N];
#pragma unroll
      for (int q = 0; q < N; ++q) o[q] = v[i].get(q) * rstd * w[i].get(q);
      if (c < a.cols) *reinterpret_cast<uint4 *>(static_cast<T *>(a.y) + base + c) = Piece<T>::pack(o);
    }
  }
  if (!a.codes) return;
  // Codes of the values before their rounding to the element type.  The maximum is that of the magnitudes' bit patterns, so
  // that a NaN or an infinity in the row shows as a scale that is not finite.
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
    for (int q = 0; q < N; ++q) top = MaxU()(top, __float_as_uint(v[i].get(q) * rstd * w[i].get(q)) & 0x7FFFFFFFu);
  top = row_reduce<WAVES>(top, tops, MaxU());
  const float amax = __uint_as_float(top);
  const float scale = top == 0u ? 1.0f : !(amax / 448.0f < 0x1p-126f) ? amax / 448.0f : 0x1p-126f;
  if (t == 0) a.scales[row] = scale;
  // The quotients by the scale are rounded correctly: with bf16 inputs y / scale = 448 v w / (v w of the largest), of which four in
  // 10^4 lie midway between two codes, and the last bit decides.  Both sides times 2^40 in rows of tiny values: the remainder of a
  // quotient that is not code 0 (2^-10 and more, 24 bits of it, times 24 of the scale) then stays above 2^-149.
  const float up = scale < 0x1p-80f ? 0x1p40f : 1.0f, divisor = scale * up;
  const float inv = 1.0f / divisor;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int c = t * N + i * STRIDE;
    uint32_t packed[N / 4];
#pragma unroll
    for (int g = 0; g < N / 4; ++g) {
      float q[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        q[j] = __builtin_amdgcn_fmed3f(quotient(v[i].get(4 * g + j) * rstd * w[i].get(4 * g + j) * up, divisor, inv), 448.0f, -448.0f);
      int code = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
      packed[g] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], code, true);
    }
    if (c < a.cols) {
      uint8_t *dst = a.codes + base + c;
      if constexpr (N == 8)
        *reinterpret_cast<uint2 *>(dst) = make_uint2(packed[0], packed[1]);
      else
        *reinterpret_cast<uint32_t *>(dst) = packed[0];
    }
  }
}

struct NormBackArgs {
  const void *sum, *weight, *dy, *dsum;
  const float *rstd;
  void *dx;
  float *partial;   // [workgroups][cols] sums of dy s rstd, null without the weight's gradient
  float *direct;    // few rows: the weight's gradient itself, by the workgroups from `parts` on
  int parts;        // workgroups that have rows
  int64_t rows;
  int cols;
  float inv_cols;
};

// The weight's gradient of few rows, straight from the rows (it needs nothing of dx): a workgroup has sixteen pieces of columns, its
// threads take 32 rows at a time (64 in workgroups of sixteen waves), and the sums of a column are added in order.
constexpr int kNormColumns = 16;  // pieces
template <typename T, int THREADS>
__device__ __forceinline__ void norm_weight_grad_columns(const NormBackArgs &a, int block, float *dweight) {
  constexpr int N = Piece<T>::N, SUBS = THREADS / kNormColumns;
  __shared__ float fold[SUBS][kNormColumns * N + 4];
  const int sub = threadIdx.x / kNormColumns, piece = threadIdx.x % kNormColumns;
  const int c = (block * kNormColumns + piece) * N;
  float dw[N];
#pragma unroll
  for (int q = 0; q < N; ++q) dw[q] = 0.f;
  if (c < a.cols) {
#pragma unroll 4
    for (int64_t row = sub; row < a.rows; row += SUBS) {
      Piece<T> s, g;
      s.load(static_cast<const T *>(a.sum) + row * a.cols + c);
      g.load(static_cast<const T *>(a.dy) + row * a.cols + c);
      const float rstd = a.rstd[row];
#pragma unroll
      for (int q = 0; q < N; ++q) dw[q] = fmaf(g.get(q) * s.get(q), rstd, dw[q]);
    }
  }
#pragma unroll
  for (int q = 0; q < N; ++q) fold[sub][piece * N + q] = dw[q];
  __syncthreads();
  const int mine = block * kNormColumns * N + threadIdx.x;
  if (threadIdx.x >= kNormColumns * N || mine >= a.cols) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < SUBS; ++i) sum += fold[i][threadIdx.x];
  dweight[mine] = sum;
}

// What a thread holds of a row.  LAST: nothing of the launch reads it again (4096 x 7168 47.6 -> 44.5 us, 8192 x 4096 51.4 -> 46.8).
template <typename T, int CHUNKS, bool LAST>
struct NormBackRow {
  Piece<T> s[CHUNKS], g[CHUNKS], r[CHUNKS];  // s, dy, dsum
  float rstd;
  __device__ __forceinline__ void load(const NormBackArgs &a, int64_t row, int t, int stride) {
    const bool there = row < a.rows;
    const int64_t base = row * a.cols;
    rstd = there ? a.rstd[row] : 0.f;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = t * Piece<T>::N + i * stride;
      s[i].zero();
      g[i].zero();
      r[i].zero();
      if (there && c < a.cols) {
        if constexpr (LAST) {
          s[i].load_last(static_cast<const T *>(a.sum) + base + c);
          g[i].load_last(static_cast<const T *>(a.dy) + base + c);
        } else {
          s[i].load(static_cast<const T *>(a.sum) + base + c);
          g[i].load(static_cast<const T *>(a.dy) + base + c);
        }
        if (a.dsum) r[i].load_last(static_cast<const T *>(a.dsum) + base + c);
      }
    }
  }
  // Values unpacked before this point are unpacked again behind it: sixteen registers a row less across the barrier.
  __device__ __forceinline__ void pin() {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
      asm volatile("" : "+v"(s[i].raw.x), "+v"(s[i].raw.y), "+v"(s[i].raw.z), "+v"(s[i].raw.w), "+v"(g[i].raw.x),
                   "+v"(g[i].raw.y), "+v"(g[i].raw.z), "+v"(g[i].raw.w));
  }
};

// The sums over a piece, and its part of dx.
template <typename T>
__device__ __forceinline__ float norm_back_sums(const Piece<T> &s, const Piece<T> &g, const Piece<T> &w, float rstd, float dot,
                                                float (&dw)[Piece<T>::N]) {
#pragma unroll
  for (int q = 0; q < Piece<T>::N; ++q) {
    const float gs = g.get(q) * s.get(q);
    dot = fmaf(gs, w.get(q), dot);
    dw[q] = fmaf(gs, rstd, dw[q]);
  }
  return dot;
}
template <typename T>
__device__ __forceinline__ void norm_back_store(const Piece<T> &s, const Piece<T> &g, const Piece<T> &w, const Piece<T> &r,
                                                float rstd, float mean, T *dst) {
  float o[Piece<T>::N];
#pragma unroll
  for (int q = 0; q < Piece<T>::N; ++q) o[q] = fmaf(rstd, fmaf(-mean, s.get(q), g.get(q) * w.get(q)), r.get(q));
  *reinterpret_cast<uint4 *>(dst) = Piece<T>::pack(o);
}

// Rows in turn, GROUPS of them at a time (WAVES waves each), the next ones on their way while the sum over a row is formed.  The
// threads' columns are the same in every row, so the weight's gradient is summed in registers; a workgroup writes one partial row.
// With the sum over those: 8192 x 4096 in bf16 with dsum 47 us, 5.7 TB/s; 4096 x 7168 45 us, 5.3.  FEW: workgroups from `parts` on
// form the weight's gradient instead.  Not HELD: rows of more than 32 KiB are read a second time behind their sum, from the caches, and
// none ahead (2048 x 32768 in bf16 134 us, 4.0 TB/s; held in registers, which do not suffice, 360).
template <typename T, int WAVES, int CHUNKS, int GROUPS, bool HELD, bool FEW>
__global__ __launch_bounds__(WAVES *GROUPS * 64) void rmsnorm_backward_kernel(const NormBackArgs a) {
  constexpr int N = Piece<T>::N, STRIDE = WAVES * 64 * N;
  __shared__ float sums[2][WAVES * GROUPS];
  __shared__ float fold[GROUPS > 1 ? STRIDE : 1];
  // (the same in a wave: rows are addressed from scalar registers)
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / (WAVES * 64)), t = threadIdx.x % (WAVES * 64);
  if (FEW && blockIdx.x >= (unsigned)a.parts) {
    norm_weight_grad_columns<T, WAVES * GROUPS * 64>(a, blockIdx.x - a.parts, a.direct);
    return;
  }
  const T *wt = static_cast<const T *>(a.weight);
  Piece<T> w[CHUNKS];
  float dw[CHUNKS][N];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int c = t * N + i * STRIDE;
    if (c < a.cols) w[i].load(wt + c); else w[i].zero();
#pragma unroll
    for (int q = 0; q < N; ++q) dw[i][q] = 0.f;
  }
  const int64_t step = (int64_t)a.parts * GROUPS;
  int64_t row = (int64_t)blockIdx.x * GROUPS + group;
  int turn = 0;
  if constexpr (HELD) {
    NormBackRow<T, CHUNKS, !FEW> now, next;
    now.load(a, row, t, STRIDE);
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < a.rows; first += step, row += step, turn ^= 1) {
      next.load(a, row + step, t, STRIDE);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) dot = norm_back_sums<T>(now.s[i], now.g[i], w[i], now.rstd, dot, dw[i]);
      dot = row_reduce<WAVES>(dot, sums[turn], AddF());
      now.pin();
      const float mean = dot * a.inv_cols * now.rstd * now.rstd;
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int c = t * N + i * STRIDE;
        if (row < a.rows && c < a.cols)
          norm_back_store<T>(now.s[i], now.g[i], w[i], now.r[i], now.rstd, mean, static_cast<T *>(a.dx) + row * a.cols + c);
      }
      now = next;
    }
  } else {  // (one group: the row is there)
    for (; row < a.rows; row += step, turn ^= 1) {
      const int64_t base = row * a.cols;
      const float rstd = a.rstd[row];
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int c = t * N + i * STRIDE;
        Piece<T> s, g;
        if (c >= a.cols) continue;
        s.load(static_cast<const T *>(a.sum) + base + c);
        g.load(static_cast<const T *>(a.dy) + base + c);
        dot = norm_back_sums<T>(s, g, w[i], rstd, dot, dw[i]);
      }
      dot = row_reduce<WAVES>(dot, sums[turn], AddF());
      const float mean = dot * a.inv_cols * rstd * rstd;
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int c = t * N + i * STRIDE;
        Piece<T> s, g, r;
        if (c >= a.cols) continue;
        s.load(static_cast<const T *>(a.sum) + base + c);
        g.load(static_cast<const T *>(a.dy) + base + c);
        if (a.dsum) r.load_last(static_cast<const T *>(a.dsum) + base + c); else r.zero();
        norm_back_store<T>(s, g, w[i], r, rstd, mean, static_cast<T *>(a.dx) + base + c);
      }
    }
  }
  if (FEW || !a.partial) return;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    if constexpr (GROUPS > 1) {  // the groups' sums in the order of the groups, one piece at a time
      for (int k = 1; k < GROUPS; ++k) {
        __syncthreads();
        if (group == k)
#pragma unroll
          for (int q = 0; q < N; ++q) fold[t * N + q] = dw[i][q];
        __syncthreads();
        if (group == 0)
#pragma unroll
          for (int q = 0; q < N; ++q) dw[i][q] += fold[t * N + q];
      }
    }
    const int c = t * N + i * STRIDE;
    if (group == 0 && c < a.cols) {
      float *dst = a.partial + (int64_t)blockIdx.x * a.cols + c;
#pragma unroll
      for (int q = 0; q < N; q += 4)
        *reinterpret_cast<float4 *>(dst + q) = make_float4(dw[i][q], dw[i][q + 1], dw[i][q + 2], dw[i][q + 3]);
    }
  }
}

// dw = the sum of the partial rows in a fixed order: 64 columns a workgroup, its sixteen waves take the rows in turn.
__global__ __launch_bounds__(1024) void rmsnorm_weight_grad_kernel(const float *__restrict__ partial, int parts, int cols,
                                                                   float *__restrict__ dw) {
  __shared__ float part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < cols)
#pragma unroll 16
    for (int p = wave; p < parts; p += 16) s += partial[(int64_t)p * cols + c];
  part[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || c >= cols) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += part[i][lane];
  dw[c] = s;
}

__global__ void rmsnorm_zero_kernel(float *__restrict__ p, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

// Waves of a row and pieces of a thread in the forward kernel: at most 32 columns a thread.  Few rows of more than 1024 columns take
// sixteen waves each, for the latency (64 x 7168: 4.1 us, with eight 4.6; 200 x 2048: 3.9 and with one 4.3; from 256 rows on fewer
// waves are as fast or faster: 1000 x 2048 6.4 against 8.6).
template <typename T, typename F>
static void with_row_form(int64_t rows, int cols, F &&f) {
  const auto at = [&](auto waves) {
    const int per = ceil_div(cols, decltype(waves)::value * 64 * Piece<T>::N);
    if (per <= 1) f(waves, std::integral_constant<int, 1>());
    else if (per <= 2) f(waves, std::integral_constant<int, 2>());
    else if (per <= 4) f(waves, std::integral_constant<int, 4>());
    else f(waves, std::integral_constant<int, 32 / Piece<T>::N>());
  };
  const bool few = rows < 256 && cols > 1024;
  if (cols <= 2048 && !few) at(std::integral_constant<int, 1>());
  else if (cols <= 4096 && !few) at(std::integral_constant<int, 4>());
  else if (cols <= 8192 && !few) at(std::integral_constant<int, 8>());
  else at(std::integral_constant<int, 16>());
}

// Workgroups of the backward kernel, each with a partial row of the weight's gradient: one on every CU, eight waves.  With the next
// rows on their way that fills HBM; more only add partial rows (bf16, us; 4096 x 7168, 8192 x 4096, 16384 x 2048: eight waves and 256
// workgroups 47.5, 51.8, 51.3, and 512 51.3, 53.9, 53.5; sixteen and 256 56.4, 52.9, 52.8; four and 1024 57.0, 60.3, 56.7).
constexpr int kNormBackWaves = 8, kNormParts = 256;
constexpr int64_t kNormLaunchRows = 1 << 21;   // rows of one launch of the forward kernel

// Up to here the weight's gradient comes from workgroups of the same launch that read s and dy again, beyond from partial rows and a
// launch of its own (bf16, us, one launch and two: 64 x 7168 4.1 and 7.6, 255 x 2048 5.2 and 7.3, 512 x 7168 11.1 and 13.3, 512 x 512
// 4.4 and 7.0, 1000 x 7168 20.2 and 18.5, 1000 x 512 8.0 and 8.4, 2000 x 2048 18.8 and 12.1).
constexpr int kNormFewRows = 512;

static int norm_check(int64_t rows, int cols, int dtype) {
  if (rows < 0 || rows > 0x7FFFFFFF || cols < 8 || cols % 8 != 0) return MOE_ERR_INVALID_ARG;
  if ((dtype != MOE_F32 && dtype != MOE_BF16) || cols > kNormMaxCols) return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

template <typename T>
static int norm_forward(NormArgs a, hipStream_t st) {
  const int64_t all = a.rows;
  for (int64_t first = 0; first < all; first += kNormLaunchRows) {  // (a grid's threads are counted in 32 bits)
    NormArgs part = a;
    const int64_t at = first * a.cols;
    part.x = static_cast<const T *>(a.x) + at;
    if (a.residual) part.residual = static_cast<const T *>(a.residual) + at;
    if (a.sum) part.sum = static_cast<T *>(a.sum) + at;
    if (a.y) part.y = static_cast<T *>(a.y) + at;
    if (a.codes) part.codes = a.codes + at;
    if (a.scales) part.scales = a.scales + first;
    if (a.rstd) part.rstd = a.rstd + first;
    part.rows = std::min(kNormLaunchRows, all - first);
    with_row_form<T>(all, a.cols, [&](auto waves, auto chunks) {
      constexpr int W = decltype(waves)::value, C = decltype(chunks)::value;
      hipLaunchKernelGGL((rmsnorm_kernel<T, W, C>), dim3((unsigned)(W == 1 ? (part.rows + 3) / 4 : part.rows)),
                         dim3(W == 1 ? 256 : W * 64), 0, st, part);
    });
    const int rc = launch_status();
    if (rc != MOE_OK) return rc;
  }
  return MOE_OK;
}

template <typename T>
static int norm_backward(NormBackArgs a, float *dweight, hipStream_t st) {
  const bool few = dweight && a.rows <= kNormFewRows && a.dx != a.dy;  // (there dy is read while dx is written)
  if (few) a.partial = nullptr;
  a.direct = few ? dweight : nullptr;
  const int columns = few ? ceil_div(a.cols, kNormColumns * Piece<T>::N) : 0;
  const auto run = [&](auto waves, auto chunks, auto held) {
    constexpr int W = decltype(waves)::value, G = std::max(1, kNormBackWaves / W), C = decltype(chunks)::value;
    a.parts = (int)std::min<int64_t>(kNormParts, (a.rows + G - 1) / G);
    constexpr bool HELD = decltype(held)::value;
    const dim3 grid((unsigned)(a.parts + columns)), block(W * G * 64);
    if (few)
      hipLaunchKernelGGL((rmsnorm_backward_kernel<T, W, C, G, HELD, true>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((rmsnorm_backward_kernel<T, W, C, G, HELD, false>), grid, block, 0, st, a);
  };
  const std::integral_constant<int, 1> c1;
  const std::integral_constant<int, 2> c2;
  const std::integral_constant<int, 4> c4;
  const std::integral_constant<int, 8> c8;
  const std::integral_constant<int, 16> c16;
  const int waves = ceil_div(a.cols, 64 * 2 * Piece<T>::N);  // with two pieces a thread
  if (waves <= 1) run(c1, c2, std::true_type());
  else if (waves <= 2) run(c2, c2, std::true_type());
  else if (waves <= 4) run(c4, c2, std::true_type());
  else if (waves <= 8) run(c8, c2, std::true_type());
  else if (waves <= 16) run(c16, c2, std::true_type());
  else if (waves <= 32) run(c16, c4, std::false_type());
  else if constexpr (Piece<T>::N == 4) run(c16, c8, std::false_type());
  const int rc = launch_status();
  if (rc != MOE_OK || !dweight || few) return rc;
  hipLaunchKernelGGL(rmsnorm_weight_grad_kernel, dim3(ceil_div(a.cols, 64)), dim3(1024), 0, st, a.partial, a.parts, a.cols,
                     dweight);
  return launch_status();
}

static bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
static bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// An array of a call (p null: not there).
struct Extent {
  const void *p;
  size_t bytes;
};
// Does `a` share memory with one of the others?
static bool overlaps(const Extent &a, std::initializer_list<Extent> others) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.p);
  for (const Extent &b : others) {
    const uintptr_t with = reinterpret_cast<uintptr_t>(b.p);
    if (a.p && b.p && a.bytes && b.bytes && at < with + b.bytes && with < at + a.bytes) return true;
  }
  return false;
}

}  // namespace moe355

using namespace moe355;

extern "C" int moe_rmsnorm(int64_t rows, int cols, int dtype, const void *x, const void *residual, const void *weight,
                           float eps, void *sum, void *y, void *codes, float *scales, float *rstd, void *stream) {
  const int rc = norm_check(rows, cols, dtype);
  if (rc != MOE_OK) return rc;
  if (!x || !weight || (!y && !codes) || (!codes != !scales) || (sum && !residual)) return MOE_ERR_INVALID_ARG;
  if (!(eps > 0.f) || !(eps < INFINITY)) return MOE_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(weight) || !aligned16(sum) || !aligned16(y) ||
      reinterpret_cast<uintptr_t>(codes) % 8 != 0 || !aligned4(scales) || !aligned4(rstd))
    return MOE_ERR_INVALID_ARG;
  if (y && (y == x || y == residual || y == sum || y == codes)) return MOE_ERR_INVALID_ARG;
  const size_t cells = (size_t)rows * cols, elt = dtype == MOE_BF16 ? 2 : 4;
  const Extent in{x, cells * elt}, res{residual, cells * elt}, w{weight, cols * elt}, s{sum, cells * elt}, out{y, cells * elt},
      q{codes, cells}, sc{scales, rows * sizeof(float)}, r{rstd, rows * sizeof(float)};
  if (overlaps(out, {in, res, w, s, q, sc, r}) || overlaps(q, {in, res, w, s, sc, r}) || overlaps(sc, {in, res, w, s, r}) ||
      overlaps(r, {in, res, w, s}) || overlaps(s, {w}) || (sum != x && overlaps(s, {in})) || (sum != residual && overlaps(s, {res})))
    return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  NormArgs a{x, residual, weight, sum, y, static_cast<uint8_t *>(codes), scales, rstd, rows, cols, eps, 1.0f / (float)cols};
  begin_launches();
  return dtype == MOE_BF16 ? norm_forward<bf16_t>(a, (hipStream_t)stream) : norm_forward<float>(a, (hipStream_t)stream);
}

extern "C" size_t moe_rmsnorm_backward_workspace_bytes(int64_t rows, int cols) {
  if (norm_check(rows, cols, MOE_F32) != MOE_OK) return 0;
  return (size_t)std::max<int64_t>(1, std::min<int64_t>(kNormParts, rows)) * cols * sizeof(float);
}

extern "C" int moe_rmsnorm_backward(int64_t rows, int cols, int dtype, const void *sum, const void *weight,
                                    const float *rstd, const void *dy, const void *dsum, void *dx, float *dweight,
                                    void *workspace, size_t workspace_bytes, void *stream) {
  int rc = norm_check(rows, cols, dtype);
  if (rc != MOE_OK) return rc;
  if (!sum || !weight || !rstd || !dy || !dx) return MOE_ERR_INVALID_ARG;
  if (dweight && (!workspace || workspace_bytes < moe_rmsnorm_backward_workspace_bytes(rows, cols))) return MOE_ERR_WORKSPACE;
  if (!aligned16(sum) || !aligned16(weight) || !aligned16(dy) || !aligned16(dsum) || !aligned16(dx) ||
      !aligned4(rstd) || !aligned4(dweight) || (dweight && !aligned16(workspace)))
    return MOE_ERR_INVALID_ARG;
  if (dx == sum) return MOE_ERR_INVALID_ARG;
  const size_t cells = (size_t)rows * cols, elt = dtype == MOE_BF16 ? 2 : 4;
  const Extent s{sum, cells * elt}, w{weight, cols * elt}, r{rstd, rows * sizeof(float)}, g{dy, cells * elt}, ds{dsum, cells * elt},
      out{dx, cells * elt}, dw{dweight, cols * sizeof(float)},
      ws{dweight ? workspace : nullptr, moe_rmsnorm_backward_workspace_bytes(rows, cols)};
  if (overlaps(out, {s, w, r, dw, ws}) || overlaps(dw, {s, w, r, g, ds, ws}) || overlaps(ws, {s, w, r, g, ds}) ||
      (dx != dy && overlaps(out, {g})) || (dx != dsum && overlaps(out, {ds})))
    return MOE_ERR_INVALID_ARG;
  hipStream_t st = (hipStream_t)stream;
  begin_launches();
  if (rows == 0) {
    if (!dweight) return MOE_OK;
    hipLaunchKernelGGL(rmsnorm_zero_kernel, dim3(ceil_div(cols, 256)), dim3(256), 0, st, dweight, cols);
    return launch_status();
  }
  NormBackArgs a{sum, weight, dy, dsum, rstd, dx, dweight ? static_cast<float *>(workspace) : nullptr, nullptr, 0, rows, cols,
                 1.0f / (float)cols};
  return dtype == MOE_BF16 ? norm_backward<bf16_t>(a, dweight, st) : norm_backward<float>(a, dweight, st);
}
