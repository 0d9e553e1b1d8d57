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

// One wave per token and part of its columns (blockIdx.y of gridDim.y parts, taken in turn, 512 columns at a time).
template <typename T>
__global__ __launch_bounds__(kRowsWaves * 64) void combine_rows_kernel(const RowsArgs a) {
  const int lane = threadIdx.x & 63;
  const int t = blockIdx.x * kRowsWaves + (threadIdx.x >> 6);  // wave-uniform
  if (t >= a.T) return;
  const int row = combine_slot_row(a.topk_idx, a.inv_perm, t, a.k, lane, a.e_lo, a.E_loc, a.offsets[a.e_lo], a.P_cap);
  const float w = row >= 0 && a.topk_w ? a.topk_w[(size_t)t * a.k + lane] : 1.0f;
  const uint64_t slots = __ballot(row >= 0);
  T *out = static_cast<T *>(a.out) + (size_t)t * a.d;
  for (int c = lane * 8 + blockIdx.y * 512; c < a.d; c += 512 * gridDim.y) {
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (uint64_t s = slots; s; s &= s - 1) {
      const int j = __builtin_ctzll(s);
      const float wj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j));
      float v[8];
      load8(static_cast<const T *>(a.rows) + (size_t)__builtin_amdgcn_readlane(row, j) * a.d + c, v);
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[q] = fmaf(wj, v[q], acc[q]);
    }
    store8<T>(out + c, acc);
  }
}

// One workgroup per token.  A slot's dot product: per thread over its columns, then over the waves in LDS.
constexpr int kBackThreads = 256;
template <typename T>
__global__ __launch_bounds__(kBackThreads) void combine_rows_backward_kernel(const RowsArgs a) {
  constexpr int WAVES = kBackThreads / 64;
  __shared__ float dots[WAVES][kMaxTopK];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = blockIdx.x;
  const int row = combine_slot_row(a.topk_idx, a.inv_perm, t, a.k, lane, a.e_lo, a.E_loc, a.offsets[a.e_lo], a.P_cap);
  const float w = row >= 0 ? a.topk_w[(size_t)t * a.k + lane] : 0.0f;
  const T *dy = static_cast<const T *>(a.dy) + (size_t)t * a.d;
  if (lane < kMaxTopK) dots[wave][lane] = 0.f;
  for (uint64_t s = __ballot(row >= 0); s; s &= s - 1) {
    const int j = __builtin_ctzll(s);
    const float wj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j));
    const size_t at = (size_t)__builtin_amdgcn_readlane(row, j) * a.d;
    const T *src = static_cast<const T *>(a.rows) + at;
    T *dst = static_cast<T *>(a.out) + at;
    float dot = 0.f;
    for (int c = threadIdx.x * 8; c < a.d; c += kBackThreads * 8) {
      float g[8], v[8], o[8];
      load8(dy + c, g);
      load8(src + c, v);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        dot = fmaf(g[q], v[q], dot);
        o[q] = wj * g[q];
      }
      store8<T>(dst + c, o);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) dot += __shfl_xor(dot, off);
    if (lane == 0) dots[wave][j] = dot;
  }
  __syncthreads();
  if (threadIdx.x >= (unsigned)a.k) return;
  float dot = 0.f;  // (a slot that is not local has zeros)
#pragma unroll
  for (int i = 0; i < WAVES; ++i) dot += dots[i][threadIdx.x];
  a.d_w[(size_t)t * a.k + threadIdx.x] = dot;
}

static bool tables_there(const moe_dispatch *tb) { return tb && tb->offsets && tb->inv_perm; }
static bool off16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }

static int combine_rows(const moe_shape *shape, const void *rows, const int32_t *topk_idx, const float *topk_w,
                        const moe_dispatch *tables, void *out, void *stream) {
  Derived dv;
  const int rc = check_shape(shape, &dv);
  if (rc != MOE_OK) return rc;
  if (!rows || !topk_idx || !tables_there(tables) || !out) return MOE_ERR_INVALID_ARG;
  if (off16(rows) || off16(out) || rows == out) return MOE_ERR_INVALID_ARG;
  if (shape->T == 0) return MOE_OK;
  RowsArgs a{rows, nullptr, topk_idx, tables->inv_perm, tables->offsets, topk_w, out, nullptr,
             shape->T, shape->k, shape->d, dv.e_lo, dv.E_loc, (int)dv.P_cap};
  const int parts = std::max(1, std::min(ceil_div(shape->d, 512), 4096 / shape->T));
  const dim3 grid((unsigned)ceil_div(shape->T, kRowsWaves), (unsigned)parts);
  begin_launches();
  if (shape->dtype == MOE_BF16)
    hipLaunchKernelGGL(combine_rows_kernel<bf16_t>, grid, dim3(kRowsWaves * 64), 0, (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL(combine_rows_kernel<float>, grid, dim3(kRowsWaves * 64), 0, (hipStream_t)stream, a);
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
  if (shape->T == 0) return MOE_OK;
  RowsArgs a{rows, dy, topk_idx, tables->inv_perm, tables->offsets, topk_w, d_rows, d_topk_w,
             shape->T, shape->k, shape->d, dv.e_lo, dv.E_loc, (int)dv.P_cap};
  begin_launches();
  if (shape->dtype == MOE_BF16)
    hipLaunchKernelGGL(combine_rows_backward_kernel<bf16_t>, dim3((unsigned)shape->T), dim3(kBackThreads), 0,
                       (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL(combine_rows_backward_kernel<float>, dim3((unsigned)shape->T), dim3(kBackThreads), 0,
                       (hipStream_t)stream, a);
  return launch_status();
}
