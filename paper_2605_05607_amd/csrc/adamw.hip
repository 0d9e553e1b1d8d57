// One AdamW step over a list of tensors: fp32 parameters (and a bf16 copy of them), both states in 32 bits or in 8.
//
//   g = grad_scale grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// States in 8 bits: blocks of 256 values, each E4M3 codes of value / scale with scale = largest magnitude times 1/448 (1 for an
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

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
constexpr int kAdamBlock = MOE_ADAMW_BLOCK;
constexpr int kAdamThreads = 256;
constexpr int kAdamTensors = 40;  // of one launch: their descriptions travel as kernel arguments
constexpr int64_t kAdamGroups = (1 << 24) - 1;        // workgroups of one launch (their threads are counted in 32 bits)
constexpr int64_t kAdamMost = kAdamGroups * 2048;     // values of a tensor: 3.4e10

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
  uint32_t first[kAdamTensors + 1];  // first chunk of every tensor (a workgroup for each)
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

// 1 - b^t for x = t log b, without the cancellation of small t: the exponential's series up to the eighth power (x > -1/2: what is
// left out is below 2^-26 of the result), else the difference.
__device__ __forceinline__ float one_less_power(float x) {
  float p = 1.0f / 40320;
  p = fmaf(p, x, 1.0f / 5040);
  p = fmaf(p, x, 1.0f / 720);
  p = fmaf(p, x, 1.0f / 120);
  p = fmaf(p, x, 1.0f / 24);
  p = fmaf(p, x, 1.0f / 6);
  p = fmaf(p, x, 0.5f);
  p = fmaf(p, x, 1.0f);
  return x > -0.5f ? -x * p : 1.0f - __expf(x);
}
__device__ __forceinline__ AdamStep step_numbers(const AdamArgs &a, const moe_adamw_device &now, const AdamTensor &x) {
  AdamStep s;
  s.beta1 = a.beta1;
  s.beta2 = a.beta2;
  s.new1 = a.new1;
  s.new2 = a.new2;
  s.eps = a.eps;
  s.keep = 1.0f - now.lr * x.weight_decay;
  s.rate = now.lr / one_less_power((float)(now.step - now.skipped) * a.log_beta1);
  s.root2 = 1.0f / sqrtf(one_less_power((float)(now.step - now.skipped) * a.log_beta2));
  s.grad_scale = now.grad_scale;
  return s;
}

// New m, v, sqrt(v) and parameter of one element.  The states' operations round one by one (no contraction, the correctly
// rounded square root), as do the scales (block_scale) and the quotients by them: where a state is held in codes, the last bit of a
// value can decide which code it gets, and this way the codes are those of the formulas evaluated in fp32 by anyone.
__device__ __forceinline__ void adam_element(const AdamStep &s, float g, float &p, float &m, float &v, float &root) {
  {
#pragma clang fp contract(off)
    g = g * s.grad_scale;
    m = s.beta1 * m + s.new1 * g;
    v = s.beta2 * v + s.new2 * g * g;
    root = sqrtf(v);  // (the instruction alone takes a subnormal v for 0, and eps may be less than its root)
  }
  p = fmaf(p, s.keep, -s.rate * m * __builtin_amdgcn_rcpf(fmaf(root, s.root2, s.eps)));
}

// E4M3 code of the magnitude of value / scale, rounded up where what is cut off exceeds the random bits (16, at the top of the 20 that
// are cut).  Times 2^-120, the formats' exponent fields agree and E4M3's subnormal values are fp32's, so the code is the top of the
// bit pattern throughout.  The quotient is the correctly rounded one, but where the remainder falls under fp32's range (blocks whose
// largest magnitude is below 2^-85) or the reciprocal is not (at most 33 of the 2^23 mantissas of a scale: all of them tried, with an
// instruction's estimate one step off to either side); there it may be an ulp off.
__device__ __forceinline__ uint32_t e4m3_stochastic(float v, float scale, float inv, uint32_t bits16) {
  const float a = fabsf(v), q0 = a * inv;
  const float q = fmaf(fmaf(-q0, scale, a), inv, q0);  // (as quotient(), without the sign)
  return (__float_as_uint(fminf(q * 0x1p-120f, 448.0f * 0x1p-120f)) + (bits16 << 4)) >> 20;
}

// The largest of a wave's values: neighbours, quarters and halves of a row of 16 lanes, then rows, by moves between lanes.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t max_of_lanes(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false));  // (0 where nothing comes in)
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_of_lanes<0xB1>(v);          // quad_perm 1 0 3 2
  v = max_of_lanes<0x4E>(v);          // quad_perm 2 3 0 1
  v = max_of_lanes<0x124>(v);         // row_ror 4
  v = max_of_lanes<0x128>(v);         // row_ror 8
  v = max_of_lanes<0x142, 0xA>(v);    // lane 15 of a row to the next (rows 1 and 3)
  v = max_of_lanes<0x143, 0xC>(v);    // lane 31 to rows 2 and 3
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Parameters, states and gradients pass with the non-temporal hint, for reads and writes: a step touches each once, and between two
// steps lies a whole pass over the model (25 M values with 32-bit states 132 -> 114 us, 302 M with 8-bit ones 891 -> 851; lists that
// the caches hold have the hint too, without a measurement of their own).  The bf16 copies, which the next kernels read, are written as
// usual.
template <typename V>
__device__ __forceinline__ V get(const V *p) { return __builtin_nontemporal_load(p); }
template <typename V>
__device__ __forceinline__ void put(V v, V *p) { __builtin_nontemporal_store(v, p); }

struct BlockScale {
  float scale, inv;
};
// The scale of the 256 values of a wave, from the largest bit pattern of their magnitudes (a NaN or an infinity gives a scale
// of NaN, so that the block shows it): one product with fp32's 1/448, which is part of the states' definition (a division gives
// another last bit in half of the blocks, and with it other codes).  Below 2^-100 a block counts as zero: the reciprocal of its scale is
// no normal number.  (Square roots of numbers in fp32 are 2^-75 and more, or 0.)
__device__ __forceinline__ BlockScale block_scale(uint32_t top) {
  top = wave_max(top);
  const bool finite = top < 0x7F800000u, some = top >= 0x0D800000u;
  const float scale = some ? __uint_as_float(top) * (1.0f / 448.0f) : 1.0f;
  const float r = __builtin_amdgcn_rcpf(scale);
  return {finite ? scale : __builtin_nanf(""), finite && some ? fmaf(fmaf(-scale, r, 1.0f), r, r) : 0.0f};
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void decode(uint32_t codes, float (&v)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  v[0] = lo[0];
  v[1] = lo[1];
  v[2] = hi[0];
  v[3] = hi[1];
}

// Four values that lie side by side, as they are read: the gradient in fp32 or (words 0 and 1) bf16, the states in fp32 or (word
// 0) codes with their block's scales.
template <bool EIGHT, bool BF16>
struct AdamQuad {
  f32x4 p;
  u32x4 g, m, v;
  float m_scale, v_scale;

  __device__ __forceinline__ void load(const AdamTensor &x, int64_t i, int64_t block) {
    p = get(reinterpret_cast<const f32x4 *>(x.param + i));
    if constexpr (BF16) {
      const u32x2 r = get(reinterpret_cast<const u32x2 *>(static_cast<const bf16_t *>(x.grad) + i));
      g[0] = r[0];
      g[1] = r[1];
    } else {
      g = get(reinterpret_cast<const u32x4 *>(static_cast<const float *>(x.grad) + i));
    }
    if constexpr (EIGHT) {
      m[0] = get(reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(x.m) + i));
      v[0] = get(reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(x.v) + i));
      m_scale = x.m_scale[block];
      v_scale = x.v_scale[block];
    } else {
      m = get(reinterpret_cast<const u32x4 *>(static_cast<const float *>(x.m) + i));
      v = get(reinterpret_cast<const u32x4 *>(static_cast<const float *>(x.v) + i));
    }
  }
  // the first `here` of the four (a tensor's end), zeros behind them
  __device__ __forceinline__ void load(const AdamTensor &x, int64_t i, int64_t block, int here) {
    p = f32x4{0.f, 0.f, 0.f, 0.f};
    g = m = v = u32x4{0u, 0u, 0u, 0u};
    m_scale = v_scale = 0.f;
    if (EIGHT) {
      m_scale = x.m_scale[block];
      v_scale = x.v_scale[block];
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      if (q >= here) continue;
      p[q] = x.param[i + q];
      if constexpr (BF16)
        g[q >> 1] |= (uint32_t)static_cast<const uint16_t *>(x.grad)[i + q] << (16 * (q & 1));
      else
        g[q] = static_cast<const uint32_t *>(x.grad)[i + q];
      if constexpr (EIGHT) {
        m[0] |= (uint32_t)static_cast<const uint8_t *>(x.m)[i + q] << (8 * q);
        v[0] |= (uint32_t)static_cast<const uint8_t *>(x.v)[i + q] << (8 * q);
      } else {
        m[q] = static_cast<const uint32_t *>(x.m)[i + q];
        v[q] = static_cast<const uint32_t *>(x.v)[i + q];
      }
    }
  }
  __device__ __forceinline__ float grad(int q) const {
    if constexpr (BF16) return __uint_as_float(q & 1 ? g[q >> 1] & 0xFFFF0000u : g[q >> 1] << 16);
    return __uint_as_float(g[q]);
  }

  // The step, in place: p, and m and v as they are stored (EIGHT: codes; the new scales go to memory).
  __device__ __forceinline__ void step(const AdamStep &s, const AdamTensor &x, int64_t i, int64_t block, uint32_t key) {
    float fm[4], fv[4], root[4];
    if constexpr (EIGHT) {
      decode(m[0], fm);
      decode(v[0], fv);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (EIGHT) {
        fm[q] *= m_scale;
        fv[q] *= v_scale;
        fv[q] *= fv[q];
      } else {
        fm[q] = __uint_as_float(m[q]);
        fv[q] = __uint_as_float(v[q]);
      }
      float fp = p[q];
      adam_element(s, grad(q), fp, fm[q], fv[q], root[q]);
      p[q] = fp;
    }
    if constexpr (!EIGHT) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        m[q] = __float_as_uint(fm[q]);
        v[q] = __float_as_uint(fv[q]);
      }
    } else {
      uint32_t top_m = 0u, top_v = 0u;  // (zeros behind the tensor's end)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        top_m = max(top_m, __float_as_uint(fm[q]) & 0x7FFFFFFFu);
        top_v = max(top_v, __float_as_uint(root[q]));  // (not negative; a NaN is above all in any case)
      }
      const BlockScale bm = block_scale(top_m), bv = block_scale(top_v);
      if ((threadIdx.x & 63) == 0) {
        x.m_scale[block] = bm.scale;
        x.v_scale[block] = bv.scale;
      }
      const uint32_t high = mix(key + (uint32_t)(i >> 32));
      m[0] = v[0] = 0u;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t h = mix(((uint32_t)i + q) ^ high);
        const uint32_t cm = e4m3_stochastic(fm[q], bm.scale, bm.inv, h & 0xFFFFu) | (__float_as_uint(fm[q]) >> 31 << 7);
        const uint32_t cv = e4m3_stochastic(root[q], bv.scale, bv.inv, h >> 16);
        m[0] |= cm << (8 * q);
        v[0] |= (root[q] > 0.f ? max(cv, 1u) : cv) << (8 * q);
      }
    }
  }

  __device__ __forceinline__ void store(const AdamTensor &x, int64_t i) const {
    put(p, reinterpret_cast<f32x4 *>(x.param + i));
    if (x.copy) *reinterpret_cast<bf16x4 *>(x.copy + i) = bf16x4{(bf16_t)p[0], (bf16_t)p[1], (bf16_t)p[2], (bf16_t)p[3]};
    if constexpr (EIGHT) {
      put((uint32_t)m[0], reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(x.m) + i));
      put((uint32_t)v[0], reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(x.v) + i));
    } else {
      put(m, reinterpret_cast<u32x4 *>(static_cast<float *>(x.m) + i));
      put(v, reinterpret_cast<u32x4 *>(static_cast<float *>(x.v) + i));
    }
  }
  __device__ __forceinline__ void store(const AdamTensor &x, int64_t i, int here) const {
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      if (q >= here) continue;
      x.param[i + q] = p[q];
      if (x.copy) x.copy[i + q] = (bf16_t)p[q];
      if constexpr (EIGHT) {
        static_cast<uint8_t *>(x.m)[i + q] = (uint8_t)(m[0] >> (8 * q));
        static_cast<uint8_t *>(x.v)[i + q] = (uint8_t)(v[0] >> (8 * q));
      } else {
        static_cast<uint32_t *>(x.m)[i + q] = m[q];
        static_cast<uint32_t *>(x.v)[i + q] = v[q];
      }
    }
  }
};

// PER blocks of 256 values for a wave, one behind the other; all are requested before the first is worked on.  32-bit
// states: two.  8-bit states, whose blocks take 350 vector instructions each: four where a launch has the values to fill the chip
// with that, else one (bf16 gradients and copies, 2^18 / 2^20 / 2^22 / 2^23 / 2^24 / 2^25 values: one block 3.5, 5.8, 15.8, 26.7, 51.5
// and 97.9 us, four 5.8, 7.8, 16.8, 27.2, 48.3 and 89.1; they cross between 2^23 and 2^24, and lists between the line and there lose 2 %
// at 2^23).
constexpr int kAdamFew = 1 << 22;
constexpr int64_t adam_chunk_values(int per) { return (int64_t)per * kAdamThreads * 4; }
template <bool EIGHT, bool BF16, int PER>
__device__ __forceinline__ void adam_chunk(const AdamArgs &a, const moe_adamw_device &now, const AdamTensor &x, int64_t begin,
                                           uint32_t key) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t first = begin + wave * PER * kAdamBlock;
  AdamQuad<EIGHT, BF16> quad[PER];
  if (PER > 1 && begin + adam_chunk_values(PER) <= x.n) {
#pragma unroll
    for (int b = 0; b < PER; ++b) quad[b].load(x, first + b * kAdamBlock + lane * 4, (first + b * kAdamBlock) / kAdamBlock);
    const AdamStep s = step_numbers(a, now, x);  // (while they are on their way)
#pragma unroll
    for (int b = 0; b < PER; ++b) {
      quad[b].step(s, x, first + b * kAdamBlock + lane * 4, (first + b * kAdamBlock) / kAdamBlock, key);
      quad[b].store(x, first + b * kAdamBlock + lane * 4);
    }
    return;
  }
#pragma unroll
  for (int b = 0; b < PER; ++b) {
    const int64_t at = first + b * kAdamBlock;  // (the same in a wave)
    if (at + kAdamBlock <= x.n) quad[b].load(x, at + lane * 4, at / kAdamBlock);
  }
  const AdamStep s = step_numbers(a, now, x);
#pragma unroll
  for (int b = 0; b < PER; ++b) {
    const int64_t at = first + b * kAdamBlock, i = at + lane * 4;
    if (at + kAdamBlock <= x.n) {
      quad[b].step(s, x, i, at / kAdamBlock, key);
      quad[b].store(x, i);
    } else if (at < x.n) {  // the tensor's last block
      const int here = (int)max((int64_t)0, min((int64_t)4, x.n - i));
      AdamQuad<EIGHT, BF16> one;
      if (here == 4) one.load(x, i, at / kAdamBlock); else one.load(x, i, at / kAdamBlock, here);
      one.step(s, x, i, at / kAdamBlock, key);
      if (here == 4) one.store(x, i); else one.store(x, i, here);
    }
  }
}

template <bool EIGHT, int PER>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamArgs a) {
  const moe_adamw_device now = a.device ? *a.device : a.now;
  if (!(fabsf(now.grad_scale) < INFINITY)) return;  // nothing is changed
  // Workgroups go to the XCDs in turn; sixteen neighbouring chunks at a time stay on one, whose pages and lines of scales are then its
  // own (302 M values, 8-bit states: 877 -> 822 us; 32-bit: 1572 -> 1493; 25 M and less: 0 to 2 %).
  uint32_t chunk = blockIdx.x;
  if ((chunk | 127u) < gridDim.x) chunk = (chunk & ~127u) + (chunk & 7u) * 16u + (chunk >> 3 & 15u);
  // the tensor of this chunk: a lane for each
  const int lane = threadIdx.x & 63;
  const int k = __builtin_amdgcn_readfirstlane(
      (int)__popcll(__ballot(lane + 1 < a.count && chunk >= a.first[min(lane + 1, kAdamTensors)])));
  const AdamTensor &x = a.tensor[k];
  const int64_t begin = (int64_t)(chunk - a.first[k]) * adam_chunk_values(PER);
  const uint32_t key = EIGHT ? mix(now.seed + mix((uint32_t)(now.step - now.skipped) + mix((uint32_t)(a.index0 + k) + 0x9E3779B9u))) : 0u;
  if (x.grad_bf16) adam_chunk<EIGHT, true, PER>(a, now, x, begin, key); else adam_chunk<EIGHT, false, PER>(a, now, x, begin, key);
}

}  // namespace moe355

using namespace moe355;

extern "C" int moe_adamw_step(const moe_adamw_config *config, const moe_adamw_tensor *tensors, int count,
                              const moe_adamw_device *device, void *stream) {
  if (!config || count < 0 || (count > 0 && !tensors)) return MOE_ERR_INVALID_ARG;
  const moe_adamw_config &c = *config;
  if (!(c.beta1 >= 0 && c.beta1 < 1) || !(c.beta2 >= 0 && c.beta2 < 1) || !((float)c.eps >= 0x1p-126f && c.eps < INFINITY))
    return MOE_ERR_INVALID_ARG;  // (the reciprocal of a subnormal eps leaves fp32, and a state of zeros would give 0 times infinity)
  if (c.state_bits != 32 && c.state_bits != 8) return MOE_ERR_UNSUPPORTED;
  if (!device && (!(c.now.lr >= 0.f && c.now.lr < INFINITY) || c.now.skipped < 0 || c.now.step <= c.now.skipped))
    return MOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(device) % 4 != 0) return MOE_ERR_INVALID_ARG;
  const bool eight = c.state_bits == 8;
  for (int k = 0; k < count; ++k) {
    const moe_adamw_tensor &t = tensors[k];
    if (t.n < 0 || !(t.weight_decay >= 0.f && t.weight_decay < INFINITY)) return MOE_ERR_INVALID_ARG;
    if (t.grad_dtype != MOE_F32 && t.grad_dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (t.n > kAdamMost) return MOE_ERR_UNSUPPORTED;
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
    int64_t values = 0;
    for (int i = k; i < std::min(count, k + kAdamTensors) && values <= kAdamFew; ++i) values += tensors[i].n;
    const int per = !eight ? 2 : values > kAdamFew ? 4 : 1;
    int64_t groups = 0;
    for (; k < count && a.count < kAdamTensors; ++k) {
      const moe_adamw_tensor &t = tensors[k];
      const int64_t more = (t.n + adam_chunk_values(per) - 1) / adam_chunk_values(per);
      if (groups + more > kAdamGroups) break;  // (the next launch: a tensor alone has at most that many)
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
    const auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kAdamThreads), 0, (hipStream_t)stream, a);
    };
    !eight ? launch(adamw_kernel<false, 2>) : per == 4 ? launch(adamw_kernel<true, 4>) : launch(adamw_kernel<true, 1>);
    const int rc = launch_status();
    if (rc != MOE_OK) return rc;
  }
  return MOE_OK;
}
