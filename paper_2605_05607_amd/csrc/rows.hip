// Rows in the layer's element type on their way back from the experts: the reduction over a token's local slots with the gate
// weights applied, and the gradients of that and of the sorting copy (moe_dispatch_gather).
//
//   back       y_t = sum over the local slots j of w_tj rows[inv(t, j)]
//   gradient   d_rows[inv(t, j)] = w_tj dy_t,   d_w_tj = <rows[inv(t, j)], dy_t>, 0 for a slot that is not local
//   sorting    dx_t = sum over the local slots of d_xs[inv(t, j)]
//
// Bound by HBM: every row is read or written once, one product an element.  Sums are fp32 in slot order, no atomics.
#include <algorithm>

#include "row_access.h"

namespace moe355 {

struct RowsArgs {
  const void *rows, *dy;
  const int32_t *topk_idx, *inv_perm, *offsets;
  const float *topk_w;  // null: rows are summed as they are
  void *out;            // y or dx; d_rows in the gradient
  float *d_w;
  int T, k, d, e_lo, E_loc, P_cap;
};

constexpr int kRowsWaves = 4;  // tokens per workgroup: one per wave
// Above, a wave takes four pieces of 512 columns (fp32: two; 8192 x 4096 62.6 us against 68.5) and bf16 rows of y leave with the
// non-temporal hint; up to here one piece, so that there are waves enough, and plain stores.  Microseconds of the two forms (few /
// many), bf16:
//   tokens                       64           512          1024         1536          3000
//   7168, 1 of 8 ranks, k = 8    2.8 / 3.5    5.1 / 5.2    6.7 / 7.0    11.3 / 9.1    21.3 / 18.3
//   2880, 1 of 4, k = 4          2.7 / 3.4    3.3 / 3.7    4.7 / 4.7     5.7 / 5.4     8.0 / 7.6
//   2048, 1 of 8, k = 8          2.6 / 3.4    3.0 / 3.6    3.7 / 4.2     4.5 / 4.9     6.4 / 6.1
//   4096, all local, k = 2       2.6 / 3.2    4.4 / 4.7    5.9 / 5.9     8.7 / 7.3    17.7 / 15.5
constexpr int kManyTokens = 1024;

// The layout row (or -1) and the weight of slot `lane` of token t: the pick, its row and its weight are requested together.
struct Slot {
  int row;
  float w;
};
__device__ __forceinline__ Slot slot_of_lane(const RowsArgs &a, int t, int lane) {
  const int base = a.offsets[a.e_lo];
  int e = -1, r = -1;
  float w = 1.0f;
  if (lane < a.k) {
    const size_t at = (size_t)t * a.k + lane;
    e = a.topk_idx[at];
    r = a.inv_perm[at] - base;
    if (a.topk_w) w = a.topk_w[at];
  }
  const bool local = e >= a.e_lo && e < a.e_lo + a.E_loc && r >= 0 && r < a.P_cap;
  return {local ? r : -1, w};
}

// One wave per token and part of its columns (blockIdx.y of gridDim.y parts, taken in turn): PIECES pieces of 512 columns at a
// time, and the loads of two slots in flight together.  STREAM: y leaves with the non-temporal hint, in bf16 (alone, 8192 tokens of 4096
// 24.6 us against 30.0; the norm that reads y right behind it gives more than that back: both together 78.6 against 78.4, and 4096
// tokens of 7168 71.8 against 65.7).  LAST: the rows come with it too (the sorting copy's gradient, whose rows nothing reads again: 5003
// tokens of 2880 with everything 54.5 -> 50.8 us, 8192 of 4096 114 -> 112; the experts' rows are read again by their gradient).
template <typename T, int PIECES, bool STREAM, bool LAST>
__global__ __launch_bounds__(kRowsWaves * 64) void combine_rows_kernel(const RowsArgs a) {
  const int lane = threadIdx.x & 63;
  const int t = blockIdx.x * kRowsWaves + (threadIdx.x >> 6);  // wave-uniform
  if (t >= a.T) return;
  const auto [row, w] = slot_of_lane(a, t, lane);
  const uint64_t slots = __ballot(row >= 0);
  T *out = static_cast<T *>(a.out) + (size_t)t * a.d;
  for (int c0 = lane * 8 + blockIdx.y * (512 * PIECES); c0 < a.d; c0 += 512 * PIECES * gridDim.y) {
    float acc[PIECES][8];
#pragma unroll
    for (int u = 0; u < PIECES; ++u)
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[u][q] = 0.f;
    for (uint64_t s = slots; s;) {
      const int j0 = __builtin_ctzll(s);
      s &= s - 1;
      const bool two = s != 0;
      const int j1 = two ? __builtin_ctzll(s) : j0;
      s &= s - 1;  // (0 stays 0)
      const T *src0 = static_cast<const T *>(a.rows) + (size_t)__builtin_amdgcn_readlane(row, j0) * a.d;
      const T *src1 = static_cast<const T *>(a.rows) + (size_t)__builtin_amdgcn_readlane(row, j1) * a.d;
      Row8<T> v0[PIECES], v1[PIECES];
#pragma unroll
      for (int u = 0; u < PIECES; ++u) {
        const int c = c0 + u * 512;
        if (c < a.d) {
          if constexpr (LAST) v0[u].load_last(src0 + c); else v0[u].load(src0 + c);
          if (two) {
            if constexpr (LAST) v1[u].load_last(src1 + c); else v1[u].load(src1 + c);
          }
        }
      }
      const float w0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j0));
      const float w1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j1));
#pragma unroll
      for (int u = 0; u < PIECES; ++u) {
        if (c0 + u * 512 < a.d) {
#pragma unroll
          for (int q = 0; q < 8; ++q) acc[u][q] = fmaf(w0, v0[u].get(q), acc[u][q]);
          if (two) {
#pragma unroll
            for (int q = 0; q < 8; ++q) acc[u][q] = fmaf(w1, v1[u].get(q), acc[u][q]);
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < PIECES; ++u)
      if (c0 + u * 512 < a.d) store8<T, STREAM>(out + c0 + u * 512, acc[u]);
  }
}

// One workgroup per token, two slots at a time (k = 8, all local: 128 tokens of 4096 10.0 us with one, 8.3; 4096 of 7168 211 and 208, 4.8
// TB/s).  A slot's dot product: per thread over its columns, then over the waves in LDS.  d_rows leave with the non-temporal hint in bf16
// (a training step's four calls around the experts, 8192 tokens of 4096, 112.5 us against 115.3, 5003 of 2880 49.9 against 54.6, where
// nothing reads the rows; with a product of 256 columns right behind, 4096 tokens of 7168, 104.7 against 101.0).
constexpr int kBackThreads = 256;
template <typename T>
__global__ __launch_bounds__(kBackThreads) void combine_rows_backward_kernel(const RowsArgs a) {
  constexpr int WAVES = kBackThreads / 64;
  __shared__ float dots[WAVES][kMaxTopK];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = blockIdx.x;
  const auto [row, w] = slot_of_lane(a, t, lane);
  const T *dy = static_cast<const T *>(a.dy) + (size_t)t * a.d;
  for (uint64_t s = __ballot(row >= 0); s;) {
    const int j0 = __builtin_ctzll(s);
    s &= s - 1;
    const bool two = s != 0;
    const int j1 = two ? __builtin_ctzll(s) : j0;
    s &= s - 1;  // (0 stays 0)
    const float w0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j0));
    const float w1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j1));
    const size_t at0 = (size_t)__builtin_amdgcn_readlane(row, j0) * a.d, at1 = (size_t)__builtin_amdgcn_readlane(row, j1) * a.d;
    const T *src = static_cast<const T *>(a.rows);
    T *dst = static_cast<T *>(a.out);
    float dot0 = 0.f, dot1 = 0.f;
    for (int c = threadIdx.x * 8; c < a.d; c += kBackThreads * 8) {
      Row8<T> g, v0, v1;
      float o[8];
      g.load(dy + c);
      v0.load(src + at0 + c);
      if (two) v1.load(src + at1 + c);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        dot0 = fmaf(g.get(q), v0.get(q), dot0);
        o[q] = w0 * g.get(q);
      }
      store8<T, true>(dst + at0 + c, o);
      if (two) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          dot1 = fmaf(g.get(q), v1.get(q), dot1);
          o[q] = w1 * g.get(q);
        }
        store8<T, true>(dst + at1 + c, o);
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      dot0 += __shfl_xor(dot0, off);
      dot1 += __shfl_xor(dot1, off);
    }
    if (lane == 0) {
      dots[wave][j0] = dot0;
      if (two) dots[wave][j1] = dot1;
    }
  }
  __syncthreads();
  if (threadIdx.x >= (unsigned)a.k) return;
  float dot = 0.f;
  if (row >= 0) {  // (thread j has slot j)
#pragma unroll
    for (int i = 0; i < WAVES; ++i) dot += dots[i][threadIdx.x];
  }
  a.d_w[(size_t)t * a.k + threadIdx.x] = dot;
}

constexpr int kMostTokens = 1 << 24;  // a workgroup of 256 threads for each, and a grid's threads are counted in 32 bits
constexpr int kMostColumns = 1 << 30;  // (column indexes run past the end by up to 2^27)
static bool tables_there(const moe_dispatch *tb) { return tb && tb->offsets && tb->inv_perm; }
static bool off16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }

static int combine_rows(const moe_shape *shape, const void *rows, const int32_t *topk_idx, const float *topk_w,
                        const moe_dispatch *tables, void *out, void *stream) {
  Derived dv;
  const int rc = check_shape(shape, &dv);
  if (rc != MOE_OK) return rc;
  if (!rows || !topk_idx || !tables_there(tables) || !out) return MOE_ERR_INVALID_ARG;
  if (off16(rows) || off16(out) || rows == out) return MOE_ERR_INVALID_ARG;
  if (shape->T >= kMostTokens || shape->d > kMostColumns) return MOE_ERR_UNSUPPORTED;
  if (shape->T == 0) return MOE_OK;
  RowsArgs a{rows, nullptr, topk_idx, tables->inv_perm, tables->offsets, topk_w, out, nullptr,
             shape->T, shape->k, shape->d, dv.e_lo, dv.E_loc, (int)dv.P_cap};
  const bool many = shape->T > kManyTokens;
  const int columns = !many ? 512 : shape->dtype == MOE_BF16 ? 2048 : 1024;  // of a wave
  const dim3 grid((unsigned)ceil_div(shape->T, kRowsWaves), (unsigned)std::min(65535, ceil_div(shape->d, columns)));
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kRowsWaves * 64), 0, (hipStream_t)stream, a); };
  begin_launches();
  const bool last = !topk_w;
  if (shape->dtype == MOE_BF16)
    !many  ? launch(combine_rows_kernel<bf16_t, 1, false, false>)
    : last ? launch(combine_rows_kernel<bf16_t, 4, true, true>)
           : launch(combine_rows_kernel<bf16_t, 4, true, false>);
  else
    !many  ? launch(combine_rows_kernel<float, 1, false, false>)
    : last ? launch(combine_rows_kernel<float, 2, true, true>)
           : launch(combine_rows_kernel<float, 2, true, false>);
  return launch_status();
}

}  // namespace moe355

using namespace moe355;

extern "C" int moe_combine_weighted(const moe_shape *shape, const void *rows, const int32_t *topk_idx, const float *topk_w,
                                    const moe_dispatch *tables, void *y, void *stream) {
  if (!topk_w) return MOE_ERR_INVALID_ARG;
  return combine_rows(shape, rows, topk_idx, topk_w, tables, y, stream);
}

extern "C" int moe_dispatch_gather_backward(const moe_shape *shape, const void *d_xs, const int32_t *topk_idx,
                                            const moe_dispatch *tables, void *dx, void *stream) {
  return combine_rows(shape, d_xs, topk_idx, nullptr, tables, dx, stream);
}

extern "C" int moe_combine_weighted_backward(const moe_shape *shape, const void *rows, const void *dy,
                                             const int32_t *topk_idx, const float *topk_w, const moe_dispatch *tables,
                                             void *d_rows, float *d_topk_w, void *stream) {
  Derived dv;
  const int rc = check_shape(shape, &dv);
  if (rc != MOE_OK) return rc;
  if (!rows || !dy || !topk_idx || !topk_w || !tables_there(tables) || !d_rows || !d_topk_w) return MOE_ERR_INVALID_ARG;
  if (off16(rows) || off16(dy) || off16(d_rows) || d_rows == dy) return MOE_ERR_INVALID_ARG;
  if (shape->T >= kMostTokens || shape->d > kMostColumns) return MOE_ERR_UNSUPPORTED;
  if (shape->T == 0) return MOE_OK;
  RowsArgs a{rows, dy, topk_idx, tables->inv_perm, tables->offsets, topk_w, d_rows, d_topk_w,
             shape->T, shape->k, shape->d, dv.e_lo, dv.E_loc, (int)dv.P_cap};
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)shape->T), dim3(kBackThreads), 0, (hipStream_t)stream, a);
  };
  begin_launches();
  shape->dtype == MOE_BF16 ? launch(combine_rows_backward_kernel<bf16_t>) : launch(combine_rows_backward_kernel<float>);
  return launch_status();
}
