// How a wave reads and writes pieces of rows, and finds the layout rows of a token.
#pragma once
#include "forward_types.h"

namespace moe355 {

// Eight consecutive outputs.  STREAM: with the non-temporal hint (a y row inside the fused call: nothing of the call
// reads it again, and the next call's operands keep their place in the caches).
template <typename OutT, bool STREAM = false>
__device__ __forceinline__ void store8(OutT *dst, const float (&v)[8]) {
  if constexpr (sizeof(OutT) == 4) {
    *reinterpret_cast<float4 *>(dst) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(dst + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    bf16x8 o;
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = (bf16_t)v[q];
    if constexpr (STREAM)
      __builtin_nontemporal_store(o, reinterpret_cast<bf16x8 *>(dst));
    else
      *reinterpret_cast<bf16x8 *>(dst) = o;
  }
}

// Eight columns of a row.
template <typename T>
struct Row8 {
  uint4 raw[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const uint4 *>(p)[i];
  }
  // with the non-temporal hint: what is read for the last time
  __device__ __forceinline__ void load_last(const T *p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      raw[i] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p) + i));
  }
  __device__ __forceinline__ float get(int q) const {
    const uint4 r = raw[q * (int)sizeof(T) / 16];
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[q & 3]);
    return __uint_as_float(q & 1 ? w[q >> 1] & 0xFFFF0000u : w[q >> 1] << 16);
  }
};

// Layout row of slot `lane` of token t if that slot is local (else -1): one lane per slot.
__device__ __forceinline__ int combine_slot_row(const int32_t *__restrict__ topk_idx,
                                                const int32_t *__restrict__ inv_perm, int t, int k, int lane,
                                                int e_lo, int E_loc, int base, int row_limit) {
  if (lane >= k) return -1;
  const int e = topk_idx[(size_t)t * k + lane];
  if (e < e_lo || e >= e_lo + E_loc) return -1;
  const int r = inv_perm[(size_t)t * k + lane] - base;
  return r >= 0 && r < row_limit ? r : -1;
}

}  // namespace moe355
