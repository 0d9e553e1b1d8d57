// One AdamW step over a list of tensors: fp32 parameters (and a bf16 copy of them), both states in 32 bits or in 8.
//
//   g = grad_scale grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// States in 8 bits: blocks of 256 values, each E4M3 codes of value / scale with scale = largest magnitude / 448 (1 for an
// all-zero block).  The second state is held as sqrt(v), whose range is half of v's in octaves, and the step uses the new
// states before they are rounded.  Codes are rounded up with the probability of what is cut off (16 random bits): a moving
// average changes by less than half a code from step to step (0.1 % against 6 %), so rounding to nearest would stop it.  A
// positive sqrt(v) never gets code 0, which would let the next step divide by eps alone.
//
// Bound by HBM: 24 bytes and the gradient per element with 32-bit states, 12 and the gradient with 8-bit ones.
#include <algorithm>
#include <cmath>

#include "forward_types.h"

namespace moe355 {

constexpr int kAdamBlock = MOE_ADAMW_BLOCK;
constexpr int kAdamThreads = 256;
constexpr int kAdamChunk = 4096;  // values of one workgroup
constexpr int kAdamTensors = 40;  // of one launch: their descriptions travel as kernel arguments

struct AdamTensor {
  float *param;
  bf16_t *copy;
  const void *grad;
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t n;
  float weight_decay;
  int32_t grad_bf16;
};
struct AdamArgs {
  AdamTensor tensor[kAdamTensors];
  uint32_t first[kAdamTensors + 1];  // first workgroup of every tensor
  int count, index0;                 // tensors of this launch, place of the first in the list
  float beta1, beta2, new1, new2, eps, log_beta1, log_beta2;  // new = 1 - beta
  moe_adamw_device now;              // without a device copy
  const moe_adamw_device *device;
};
static_assert(sizeof(AdamArgs) <= 4000, "kernel arguments");

// Thirty-two mixed bits (two rounds of xor with a shifted copy and an odd multiplier: the fractions of sqrt 2 and sqrt 3).
__device__ __forceinline__ uint32_t mix(uint32_t z) {
  z = (z ^ (z >> 16)) * 0x6A09E667u;
  z = (z ^ (z >> 15)) * 0xBB67AE85u;
  return z ^ (z >> 16);
}

// What a step needs, the same for every element.
struct AdamStep {
  float beta1, beta2, new1, new2, eps, keep, rate, root2, grad_scale;
};

template <bool BF16>
__device__ __forceinline__ void load_grad(const void *grad, int64_t i, float (&g)[4]) {
  if constexpr (BF16) {
    const uint2 raw = *reinterpret_cast<const uint2 *>(static_cast<const bf16_t *>(grad) + i);
    g[0] = __uint_as_float(raw.x << 16);
    g[1] = __uint_as_float(raw.x & 0xFFFF0000u);
    g[2] = __uint_as_float(raw.y << 16);
    g[3] = __uint_as_float(raw.y & 0xFFFF0000u);
  } else {
    const f32x4 raw = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(grad) + i);
#pragma unroll
    for (int q = 0; q < 4; ++q) g[q] = raw[q];
  }
}
__device__ __forceinline__ float grad_at(const void *grad, bool bf16, int64_t i) {
  return bf16 ? (float)static_cast<const bf16_t *>(grad)[i] : static_cast<const float *>(grad)[i];
}

// New m, v, sqrt(v) and parameter of one element.  The states' operations round one by one (no contraction, the correctly
// rounded square root): where a state is held in codes, the last bit of a value can decide which code it gets, and this way the
// codes are those of the formulas evaluated in fp32 by anyone.
__device__ __forceinline__ void adam_element(const AdamStep &s, float g, float &p, float &m, float &v, float &root) {
  {
#pragma clang fp contract(off)
    g = g * s.grad_scale;
    m = s.beta1 * m + s.new1 * g;
    v = s.beta2 * v + s.new2 * g * g;
    root = sqrtf(v);
  }
  p = fmaf(p, s.keep, -s.rate * m * __builtin_amdgcn_rcpf(fmaf(root, s.root2, s.eps)));
}

// E4M3 code of value / scale, rounded up where what is cut off exceeds the random bits (16, at the top of the 20 that are cut).
// Below 2^-6 the codes are multiples of 2^-9, as those of the octave above: 2^-6 is added and taken off again.
// The quotient is the correctly rounded one, from the correctly rounded reciprocal (Markstein 1990).
__device__ __forceinline__ uint32_t e4m3_stochastic(float v, float scale, float inv, uint32_t bits16) {
  const float a = fabsf(v), q0 = a * inv;
  const float q = fminf(fmaf(fmaf(-q0, scale, a), inv, q0), 448.0f);
  const bool small = q < 0x1p-6f;
  const uint32_t up = __float_as_uint(small ? q + 0x1p-6f : q) + (bits16 << 4);
  return (up >> 20) - (small ? 968u : 960u);
}

struct BlockScale {
  float scale, inv;
};
// The scale of the 256 values of a wave, from the largest bit pattern of their magnitudes (a NaN or an infinity gives a scale
// of NaN, so that the block shows it).  Below 2^-100 a block counts as zero: the reciprocal of its scale is no normal number.
__device__ __forceinline__ BlockScale block_scale(uint32_t top) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
  const float amax = __uint_as_float(top);
  if (top >= 0x7F800000u) return {__builtin_nanf(""), 0.0f};
  if (amax < 0x1p-100f) return {1.0f, amax == 0.0f ? 1.0f : 0.0f};
  const float scale = amax * (1.0f / 448.0f);
  return {scale, 1.0f / scale};
}

__device__ __forceinline__ float decode(uint32_t codes, int q) {
  switch (q) {
    case 0: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 0);
    case 1: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 1);
    case 2: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 2);
    default: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 3);
  }
}

// A workgroup takes 4096 values of a tensor, a wave 256 at a time, a lane four that lie side by side.
template <bool EIGHT>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamArgs a) {
  const moe_adamw_device now = a.device ? *a.device : a.now;
  if (!(fabsf(now.grad_scale) < INFINITY)) return;  // nothing is changed
  int k = 0;
  while (k + 1 < a.count && blockIdx.x >= a.first[k + 1]) ++k;
  const AdamTensor &x = a.tensor[k];
  AdamStep s;
  s.beta1 = a.beta1;
  s.beta2 = a.beta2;
  s.new1 = a.new1;
  s.new2 = a.new2;
  s.eps = a.eps;
  s.keep = 1.0f - now.lr * x.weight_decay;
  s.rate = now.lr / -expm1f((float)now.step * a.log_beta1);  // (1 - b^t without the cancellation)
  s.root2 = 1.0f / sqrtf(-expm1f((float)now.step * a.log_beta2));
  s.grad_scale = now.grad_scale;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t begin = (int64_t)(blockIdx.x - a.first[k]) * kAdamChunk;
  const uint32_t key = EIGHT ? mix(now.seed + mix((uint32_t)now.step + mix((uint32_t)(a.index0 + k) + 0x9E3779B9u))) : 0u;
#pragma unroll
  for (int b = 0; b < kAdamChunk / (kAdamThreads * 4); ++b) {
    const int64_t first = begin + (b * (kAdamThreads / 64) + wave) * kAdamBlock;
    if (first >= x.n) break;  // (the same in a wave)
    const int64_t i = first + lane * 4;
    const int here = (int)max((int64_t)0, min((int64_t)4, x.n - i));
    float p[4], g[4], m[4], v[4], root[4];
    const int64_t block = first / kAdamBlock;
    if (here == 4) {
      if (x.grad_bf16) load_grad<true>(x.grad, i, g); else load_grad<false>(x.grad, i, g);
      const f32x4 pv = *reinterpret_cast<const f32x4 *>(x.param + i);
#pragma unroll
      for (int q = 0; q < 4; ++q) p[q] = pv[q];
      if constexpr (EIGHT) {
        const uint32_t mc = *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(x.m) + i);
        const uint32_t vc = *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(x.v) + i);
        const float ms = x.m_scale[block], vs = x.v_scale[block];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          m[q] = decode(mc, q) * ms;
          const float r = decode(vc, q) * vs;
          v[q] = r * r;
        }
      } else {
        const f32x4 mv = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(x.m) + i);
        const f32x4 vv = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(x.v) + i);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          m[q] = mv[q];
          v[q] = vv[q];
        }
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        p[q] = g[q] = m[q] = v[q] = 0.f;
        if (q >= here) continue;
        g[q] = grad_at(x.grad, x.grad_bf16, i + q);
        p[q] = x.param[i + q];
        if constexpr (EIGHT) {
          m[q] = decode(static_cast<const uint8_t *>(x.m)[i + q], 0) * x.m_scale[block];
          const float r = decode(static_cast<const uint8_t *>(x.v)[i + q], 0) * x.v_scale[block];
          v[q] = r * r;
        } else {
          m[q] = static_cast<const float *>(x.m)[i + q];
          v[q] = static_cast<const float *>(x.v)[i + q];
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) adam_element(s, g[q], p[q], m[q], v[q], root[q]);
    uint32_t mc = 0u, vc = 0u;
    if constexpr (EIGHT) {
      uint32_t top_m = 0u, top_v = 0u;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < here) {
          top_m = max(top_m, __float_as_uint(m[q]) & 0x7FFFFFFFu);
          top_v = max(top_v, __float_as_uint(root[q]) & 0x7FFFFFFFu);
        }
      const BlockScale bm = block_scale(top_m), bv = block_scale(top_v);
      if (lane == 0) {
        x.m_scale[block] = bm.scale;
        x.v_scale[block] = bv.scale;
      }
      const uint32_t high = mix(key + (uint32_t)(i >> 32));
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t h = mix(((uint32_t)i + q) ^ high);
        const uint32_t cm = e4m3_stochastic(m[q], bm.scale, bm.inv, h & 0xFFFFu) | (__float_as_uint(m[q]) >> 31 << 7);
        uint32_t cv = e4m3_stochastic(root[q], bv.scale, bv.inv, h >> 16);
        cv = root[q] > 0.f ? max(cv, 1u) : cv;
        mc |= cm << (8 * q);
        vc |= cv << (8 * q);
      }
    }
    if (here == 4) {
      *reinterpret_cast<f32x4 *>(x.param + i) = f32x4{p[0], p[1], p[2], p[3]};
      if (x.copy) *reinterpret_cast<bf16x4 *>(x.copy + i) = bf16x4{(bf16_t)p[0], (bf16_t)p[1], (bf16_t)p[2], (bf16_t)p[3]};
      if constexpr (EIGHT) {
        *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(x.m) + i) = mc;
        *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(x.v) + i) = vc;
      } else {
        *reinterpret_cast<f32x4 *>(static_cast<float *>(x.m) + i) = f32x4{m[0], m[1], m[2], m[3]};
        *reinterpret_cast<f32x4 *>(static_cast<float *>(x.v) + i) = f32x4{v[0], v[1], v[2], v[3]};
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q >= here) continue;
        x.param[i + q] = p[q];
        if (x.copy) x.copy[i + q] = (bf16_t)p[q];
        if constexpr (EIGHT) {
          static_cast<uint8_t *>(x.m)[i + q] = (uint8_t)(mc >> (8 * q));
          static_cast<uint8_t *>(x.v)[i + q] = (uint8_t)(vc >> (8 * q));
        } else {
          static_cast<float *>(x.m)[i + q] = m[q];
          static_cast<float *>(x.v)[i + q] = v[q];
        }
      }
    }
  }
}

}  // namespace moe355

using namespace moe355;

extern "C" int moe_adamw_step(const moe_adamw_config *config, const moe_adamw_tensor *tensors, int count,
                              const moe_adamw_device *device, void *stream) {
  if (!config || count < 0 || (count > 0 && !tensors)) return MOE_ERR_INVALID_ARG;
  const moe_adamw_config &c = *config;
  if (!(c.beta1 >= 0 && c.beta1 < 1) || !(c.beta2 >= 0 && c.beta2 < 1) || !((float)c.eps > 0.f && c.eps < INFINITY))
    return MOE_ERR_INVALID_ARG;
  if (c.state_bits != 32 && c.state_bits != 8) return MOE_ERR_UNSUPPORTED;
  if (!device && (!(c.now.lr >= 0.f && c.now.lr < INFINITY) || c.now.step < 1)) return MOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(device) % 4 != 0) return MOE_ERR_INVALID_ARG;
  const bool eight = c.state_bits == 8;
  for (int k = 0; k < count; ++k) {
    const moe_adamw_tensor &t = tensors[k];
    if (t.n < 0 || !(t.weight_decay >= 0.f && t.weight_decay < INFINITY)) return MOE_ERR_INVALID_ARG;
    if (t.grad_dtype != MOE_F32 && t.grad_dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (t.n > (int64_t)kAdamChunk << 30) return MOE_ERR_UNSUPPORTED;
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v || (eight && (!t.m_scale || !t.v_scale))) return MOE_ERR_INVALID_ARG;
    const auto at = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
    if ((at(t.param) | at(t.copy) | at(t.grad) | at(t.m) | at(t.v)) % 16 != 0) return MOE_ERR_INVALID_ARG;
    if (eight && (at(t.m_scale) | at(t.v_scale)) % 4 != 0) return MOE_ERR_INVALID_ARG;
  }
  begin_launches();
  for (int k = 0; k < count;) {
    AdamArgs a{};
    a.index0 = k;
    int64_t groups = 0;
    for (; k < count && a.count < kAdamTensors; ++k) {
      const moe_adamw_tensor &t = tensors[k];
      const int64_t more = (t.n + kAdamChunk - 1) / kAdamChunk;
      if (groups + more > (int64_t)1 << 30) break;  // (the next launch: a tensor alone has at most that many)
      AdamTensor &x = a.tensor[a.count];
      x.param = t.param;
      x.copy = static_cast<bf16_t *>(t.copy);
      x.grad = t.grad;
      x.m = t.m;
      x.v = t.v;
      x.m_scale = t.m_scale;
      x.v_scale = t.v_scale;
      x.n = t.n;
      x.weight_decay = t.weight_decay;
      x.grad_bf16 = t.grad_dtype == MOE_BF16;
      a.first[a.count++] = (uint32_t)groups;
      groups += more;
      a.first[a.count] = (uint32_t)groups;
    }
    if (groups == 0) continue;
    a.beta1 = (float)c.beta1;
    a.beta2 = (float)c.beta2;
    a.new1 = (float)(1.0 - c.beta1);
    a.new2 = (float)(1.0 - c.beta2);
    a.eps = (float)c.eps;
    a.log_beta1 = (float)std::log(c.beta1);  // (beta 0: -inf, and 1 - beta^t is 1)
    a.log_beta2 = (float)std::log(c.beta2);
    a.now = c.now;
    a.device = device;
    if (eight)
      hipLaunchKernelGGL(adamw_kernel<true>, dim3((unsigned)groups), dim3(kAdamThreads), 0, (hipStream_t)stream, a);
    else
      hipLaunchKernelGGL(adamw_kernel<false>, dim3((unsigned)groups), dim3(kAdamThreads), 0, (hipStream_t)stream, a);
    const int rc = launch_status();
    if (rc != MOE_OK) return rc;
  }
  return MOE_OK;
}
