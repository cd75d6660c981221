// edp_loss.cuh -- what the kernels of the losses share: element types, the
// policy loss of one token, sums that keep the bits of more than fp32.
#pragma once

#include <cuda_fp16.h>

#include "edp_internal.cuh"

namespace edp {

constexpr unsigned kAllLanes = 0xffffffffu;
constexpr float kLn2 = 0.693147180559945309f;
constexpr double kLog2e = 1.442695040888963407;

template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) {
  return __bfloat162float(x);
}
template <>
__device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }

template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// 2^x to 2^-22, 0 below the smallest normal number.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

constexpr float kNegInf = -__builtin_huge_valf();

// The policy loss's constants, from an edp_policy_config.
struct PolicyRule {
  float low, high, dual;           // limits of the ratio; dual 0: none
  float ln_low, ln_high, ln_dual;  // and of its logarithm
  float kl_coef, entropy_coef, grad_scale;
  uint32_t kl;
};

// One token: its policy loss and divergence, the ratio, whether it is clipped,
// and the loss's derivative by logp (entropy apart), before weight and scale.
struct PolicyToken {
  float pg, kl, ratio, dlogp, old_kl;
  bool above, below;
};

// e^q - 1 - q and e^q - 1: below 1 the Taylor series, without the difference
// that would leave few bits of the first (relative error below 2^-23 for all q).
__device__ __forceinline__ float exp_less_line(float q, float e, float *em1) {
  float k;
  if (fabsf(q) < 1.f) {
    float p = 1.f / 6227020800.f;  // 1/13!
    p = fmaf(p, q, 1.f / 479001600.f);
    p = fmaf(p, q, 1.f / 39916800.f);
    p = fmaf(p, q, 1.f / 3628800.f);
    p = fmaf(p, q, 1.f / 362880.f);
    p = fmaf(p, q, 1.f / 40320.f);
    p = fmaf(p, q, 1.f / 5040.f);
    p = fmaf(p, q, 1.f / 720.f);
    p = fmaf(p, q, 1.f / 120.f);
    p = fmaf(p, q, 1.f / 24.f);
    p = fmaf(p, q, 1.f / 6.f);
    p = fmaf(p, q, 0.5f);
    k = q * q * p;
    *em1 = q + k;
  } else {
    *em1 = e - 1.f;
    k = *em1 - q;
  }
  return k;
}

__device__ __forceinline__ PolicyToken policy_token(const PolicyRule &c, float logp, float old,
                                                    float ref, bool has_ref, float adv) {
  PolicyToken o;
  const float d = logp - old;
  o.ratio = expf(d);
  float em1;
  o.old_kl = exp_less_line(d, o.ratio, &em1);
  // the limits act on the logarithm, whose difference of two fp32 numbers is
  // one rounding away from the numbers that the caller gave
  o.above = adv > 0.f && d > c.ln_high;
  const bool dual = adv < 0.f && d > c.ln_dual;
  o.below = dual || (adv < 0.f && d < c.ln_low);
  const float used = o.above ? c.high : dual ? c.dual : o.below ? c.low : o.ratio;
  // an advantage of 0 takes nothing from a ratio that overflowed
  o.pg = adv == 0.f && !isnan(d) ? 0.f : -used * adv;
  o.dlogp = o.above || o.below ? 0.f : o.pg;
  o.kl = 0.f;
  if (has_ref) {
    const float q = ref - logp;
    float g = 1.f;
    if (c.kl == EDP_KL_K1) {
      o.kl = -q;
    } else if (c.kl == EDP_KL_K2) {
      o.kl = 0.5f * q * q;
      g = -q;
    } else {
      o.kl = exp_less_line(q, expf(q), &em1);
      g = -em1;
    }
    if (c.kl_coef != 0.f) o.dlogp = fmaf(c.kl_coef, g, o.dlogp);
  }
  return o;
}


}  // namespace edp
