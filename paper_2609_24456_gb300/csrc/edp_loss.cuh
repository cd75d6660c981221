// edp_loss.cuh -- what the kernels of the losses share: element types, the
// policy loss of one token, sums that keep the bits of more than fp32, and the
// walk over a packed batch's tokens.
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
  df kl_both, less_entropy;        // both coefficients, the second negative
  uint32_t kl;
};

// e^q - 1 - q for |q| below 1: the Taylor series, whose first term left out is
// 2^-24 of the sum.
__device__ __forceinline__ float exp_less_line(float q) {
  float p = 1.f / 3628800.f;  // 1/10!
  p = fmaf(p, q, 1.f / 362880.f);
  p = fmaf(p, q, 1.f / 40320.f);
  p = fmaf(p, q, 1.f / 5040.f);
  p = fmaf(p, q, 1.f / 720.f);
  p = fmaf(p, q, 1.f / 120.f);
  p = fmaf(p, q, 1.f / 24.f);
  p = fmaf(p, q, 1.f / 6.f);
  p = fmaf(p, q, 0.5f);
  return q * q * p;
}
// The same for any q, and in em1 e^q - 1: from 1 on the difference loses at most
// two bits of e^q.
__device__ __forceinline__ float exp_less_line(float q, float *em1) {
  const float near = exp_less_line(q), e = ex2(q * (float)kLog2e) - 1.f;
  const bool far = !(fabsf(q) < 1.f);
  *em1 = far ? e : q + near;
  return far ? e - q : near;
}

// One token: its policy loss and divergence, the ratio less one, the divergence from
// the old policy, and the loss's derivative by logp (entropy apart), before weight
// and scale.  d = logp - old, q = ref - logp; with d, q and the advantage 0 all are 0
// but the derivative with EDP_KL_K1, whose divergence falls with logp everywhere.
struct PolicyToken {
  float pg, kl, ratio1, old_kl, dlogp;
  bool above, below;
};
enum class Kl { kNone, kK3, kOther };  // which estimator, as far as the code goes

// NEAR: |d| and |q| are below 1.
template <Kl KL, bool NEAR>
__device__ __forceinline__ PolicyToken policy_token(const PolicyRule &c, float d, float q,
                                                    float adv) {
  PolicyToken o;
  if (NEAR) {
    o.old_kl = exp_less_line(d);
    o.ratio1 = d + o.old_kl;
  } else {
    o.old_kl = exp_less_line(d, &o.ratio1);
  }
  const float r = o.ratio1 + 1.f;
  // the limits act on the logarithm, whose difference of two fp32 numbers is
  // one rounding away from the numbers that the caller gave
  const bool pos = adv > 0.f;
  const bool up = d > (pos ? c.ln_high : c.ln_dual), down = !pos && d < c.ln_low;
  const float used = up ? (pos ? c.high : c.dual) : down ? c.low : r;
  o.pg = -used * adv;
  // an advantage of 0 takes nothing from any ratio, one that overflowed among them
  if (!NEAR && adv == 0.f && !isnan(d)) o.pg = 0.f;
  o.dlogp = up || down ? 0.f : o.pg;
  o.above = up && pos;
  o.below = (up || down) && adv < 0.f;
  o.kl = 0.f;
  if (KL != Kl::kNone) {
    float g;  // minus the derivative
    if (KL == Kl::kK3) {
      if (NEAR) {
        o.kl = exp_less_line(q);
        g = q + o.kl;
      } else {
        o.kl = exp_less_line(q, &g);
      }
    } else if (c.kl == EDP_KL_K1) {
      o.kl = -q;
      g = -1.f;
    } else {
      o.kl = 0.5f * q * q;
      g = q;
    }
    // without the coefficient the divergence is reported alone, whatever it is
    if (c.kl_coef != 0.f) o.dlogp = fmaf(-c.kl_coef, g, o.dlogp);
  }
  return o;
}

// ---------------------------------------------------------------------------
// Sums in pairs of fp32 numbers: hi is the running sum, lo the sum of its
// rounding errors (Ogita, Rump and Oishi 2005, "Sum2").  About 46 bits, for 7
// operations a term; fp64 runs at a sixty-fourth of the fp32 rate here.  hi
// alone carries infinities and NaN.
// ---------------------------------------------------------------------------
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ void pair_add(Pair &a, float x) {
  const df s = two_sum(a.hi, x);
  a.hi = s.hi;
  a.lo = __fadd_rn(a.lo, s.lo);
}
__device__ __forceinline__ Pair pair_of(uint32_t n) {
  const float hi = (float)n;
  return {hi, (float)((long long)n - (long long)hi)};
}
__device__ __forceinline__ Pair pair_join(Pair a, Pair b) {
  const df s = two_sum(a.hi, b.hi);
  return {s.hi, __fadd_rn(__fadd_rn(a.lo, b.lo), s.lo)};
}
__device__ __forceinline__ df as_df(Pair a) {
  return isfinite(a.hi) ? quick_two_sum(a.hi, a.lo) : df{a.hi, 0.f};
}
__device__ __forceinline__ Pair pair_shfl_xor(Pair a, int o) {
  return {__shfl_xor_sync(kAllLanes, a.hi, o), __shfl_xor_sync(kAllLanes, a.lo, o)};
}
__device__ __forceinline__ Pair warp_join(Pair a) {
#pragma unroll
  for (int o = 16; o; o >>= 1) a = pair_join(a, pair_shfl_xor(a, o));
  return a;
}

// K sums of a warp's lanes at once, K a power of two: in each step a lane hands over
// half of the sums that it still has for as many of the other half.  Sum k ends in
// lanes k 32/K and on; the order is fixed.
template <int K>
__device__ __forceinline__ Pair warp_join_all(const Pair (&mine)[K]) {
  Pair v[K];
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = mine[k];
  const int lane = threadIdx.x & 31;
  int o = 16;
#pragma unroll
  for (int h = K / 2; h; h /= 2, o /= 2) {
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const Pair give = upper ? v[i] : v[i + h], keep = upper ? v[i + h] : v[i];
      v[i] = pair_join(keep, pair_shfl_xor(give, o));
    }
  }
#pragma unroll
  for (; o; o >>= 1) v[0] = pair_join(v[0], pair_shfl_xor(v[0], o));
  return v[0];
}

// K sums over the grid: the pairs of every thread of every CTA joined in a fixed
// order.  True in the last CTA to arrive, where total[] (shared) then holds them.
// part: [K][gridDim.x]; ticket: 0 before and after.
template <int NT, int K>
__device__ __forceinline__ bool grid_join(const Pair (&mine)[K], Pair *total, Pair *part,
                                          uint32_t *ticket) {
  static_assert(K <= NT / 32, "a warp per sum");
  __shared__ Pair red[K][NT / 32];
  __shared__ bool last;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  Pair v = warp_join_all(mine);
  if (lane % (32 / K) == 0) red[lane / (32 / K)][wid] = v;
  __syncthreads();
  v = Pair{0.f, 0.f};
  if (wid < K) {
    if (lane < NT / 32) v = red[wid][lane];
    v = warp_join(v);
  }
  if (gridDim.x == 1) {
    if (wid < K && lane == 0) total[wid] = v;
    __syncthreads();
    return true;
  }
  if (wid < K && lane == 0) {
    __stcg(reinterpret_cast<float2 *>(part) + (uint64_t)wid * gridDim.x + blockIdx.x,
           make_float2(v.hi, v.lo));
    __threadfence();
  }
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return false;
  __threadfence();
  if (wid < K) {
    v = Pair{0.f, 0.f};
    for (uint32_t b = lane; b < gridDim.x; b += 32) {
      const float2 x =
          __ldcg(reinterpret_cast<const float2 *>(part) + (uint64_t)wid * gridDim.x + b);
      v = pair_join(v, Pair{x.x, x.y});
    }
    v = warp_join(v);
    if (lane == 0) total[wid] = v;
  }
  if (threadIdx.x == 0) *ticket = 0u;
  __syncthreads();
  return true;
}

// ---------------------------------------------------------------------------
// A packed batch's tokens: a warp takes tiles of 128, 4 tokens per lane, and knows
// the sequence that each tile starts in.
// ---------------------------------------------------------------------------
constexpr uint32_t kTile = 128;

// The sequence of token t among lo .. hi - 1: the last one that starts at t or
// before (so an empty one holds none).
__device__ __forceinline__ uint32_t sequence_of(const uint64_t *off, uint32_t lo, uint32_t hi,
                                                uint64_t t) {
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (off[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}
// The same by a warp, 32 probes at a time: three rounds for 32,768 sequences.
__device__ __forceinline__ uint32_t sequence_of_warp(const uint64_t *off, uint32_t lo, uint32_t hi,
                                                     uint64_t t) {
  const uint32_t lane = threadIdx.x & 31;
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 31) / 32;  // probes lo + step, lo + 2 step, ...
    const uint32_t at = (uint32_t)min((uint64_t)lo + (uint64_t)(lane + 1) * step, (uint64_t)hi);
    const bool le = at < hi && off[at] <= t;
    const uint32_t k = __popc(__ballot_sync(kAllLanes, le));  // probes at or before t
    hi = (uint32_t)min((uint64_t)lo + (uint64_t)(k + 1) * step, (uint64_t)hi);
    lo += k * step;
  }
  return lo;
}

// A warp's place among the sequences, which only moves on.
struct SeqWalk {
  uint32_t q;     // the sequence
  uint64_t next;  // and where the one after it starts
  __device__ __forceinline__ void start(const uint64_t *off, uint32_t n, uint64_t t) {
    q = sequence_of_warp(off, 0, n, t);
    next = off[q + 1];
  }
  // to the sequence of token t: among the next 31 most often
  __device__ __forceinline__ void to(const uint64_t *off, uint32_t n, uint64_t t) {
    if (t < next) return;
    const uint64_t at = (uint64_t)q + 1 + (threadIdx.x & 31);
    const uint32_t k = __popc(__ballot_sync(kAllLanes, at < n && off[at] <= t));
    q = k < 32 ? q + k : sequence_of_warp(off, q + 32, n, t);
    next = off[q + 1];
  }
};

// Bytes that are not 0.
__device__ __forceinline__ uint32_t some_bytes(uint32_t x) {
  return __popc((((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) & 0x80808080u);
}

// Which of the tokens t .. t + 3 count, as bits; t is a multiple of 4.  first,
// end: the tokens that the sequences hold.
template <bool VEC>
__device__ __forceinline__ uint32_t token_bits(const TokenSet &s, uint64_t t, uint64_t first,
                                               uint64_t end) {
  if (t >= end) return 0;
  uint32_t bits = t + 4 <= end ? 15u : (1u << (uint32_t)(end - t)) - 1u;
  if (t < first) bits &= t + 4 <= first ? 0u : ~((1u << (uint32_t)(first - t)) - 1u);
  if (s.mask) {
    if (VEC && t + 4 <= s.n) {
      const uint32_t m = *reinterpret_cast<const uint32_t *>(s.mask + t);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!((m >> (8 * i)) & 0xffu)) bits &= ~(1u << i);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((bits >> i & 1u) && !s.mask[t + i]) bits &= ~(1u << i);
    }
  }
  if (s.target) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((bits >> i & 1u) && (uint32_t)s.target[t + i] >= s.vocab) bits &= ~(1u << i);
  }
  return bits;
}

struct Weighting {
  const float *sequence;             // SEQ_MEAN: each sequence's weight
  const unsigned long long *tokens;  // TOKEN_MEAN without norm: the divisor
  bool by_range;                     // the same where every token of the sequences counts
  float fixed;                       // otherwise: every weight
};

struct Range {
  uint64_t first, end;  // the tokens that the sequences hold
};
__device__ __forceinline__ Range token_range(const TokenSet &s) {
  if (!s.off) return {0, s.n};
  return {s.off[0], min(s.off[s.n_seq], s.n)};
}

// Up to so many tokens on average that its weight takes in, a row of logits counts them
// itself, beside its copy, in the place of one or two kernels before.  In a graph, with the
// kernels and without: 16 rows 14.0 and 11.5 us; of 32,003 columns, 515 rows in 16 sequences
// 28.3 and 27.1, in 4 28.3 and 28.6, with one mean over all 26.2 and 33.6; 1,000 rows in 16
// 45.4 and 46.1.  Over 8 to 1,000 rows of 4,096, 32,003 and 152,064 columns the rule is within
// 4% of the better one, but for means over 130 to 250 tokens of 4,096 columns (up to 22%).
constexpr uint64_t kFewTokens = 128;
constexpr uint64_t kFewRows = 1024;
// The scratch of a loss and what it is for.
struct Plan {
  Weighting w;
  float divisor;
  bool sequences;
  bool early;        // a kernel that counts tokens runs first
  Pair *part;        // sums of the policy loss's CTAs
  float *per_token;  // a number per token, where asked for
};
// Counts what the weights need, unless the batch's own CTA does (one_cta).
cudaError_t plan_weights(edp_ctx *c, const TokenSet &set, bool one_cta, bool per_token,
                         cudaStream_t s, Plan *p);
// The count that the loss would have set back to 0, after a launch that failed.
void forget_count(edp_ctx *c, const Plan &p, cudaStream_t s);

// What a row of logits weighs in a loss, by its token's place.
struct RowWeights {
  TokenSet set;
  bool count;                        // the row counts for itself (few rows), else:
  const float *sequence;             // each sequence's weight,
  const unsigned long long *tokens;  // or the divisor of all,
  float fixed;                       // or the weight of all
  float divisor;                     // by sequences: their number
};
__device__ __forceinline__ bool in_sequences(const RowWeights &w, uint64_t t) {
  return !w.set.off || (t >= w.set.off[0] && t < w.set.off[w.set.n_seq]);
}
// What row t of the sequences weighs, found by a warp.
__device__ __forceinline__ float row_weight(const RowWeights &w, uint64_t t) {
  const TokenSet &s = w.set;
  const bool by_sequence = s.reduce == EDP_REDUCE_SEQ_MEAN;
  if (!w.count) {
    if (w.sequence) return __ldcg(&w.sequence[sequence_of_warp(s.off, 0, (uint32_t)s.n_seq, t)]);
    return w.tokens ? 1.f / (float)__ldcg(w.tokens) : w.fixed;
  }
  uint64_t a = 0, b = s.n;
  if (s.off) {
    const uint32_t q = by_sequence ? sequence_of_warp(s.off, 0, (uint32_t)s.n_seq, t) : 0;
    a = s.off[q];
    b = min(s.off[by_sequence ? q + 1 : s.n_seq], s.n);
  }
  uint32_t n = 0;
#pragma unroll 2
  for (uint64_t i = (a & ~3ull) + 4 * (threadIdx.x & 31); i < b; i += 128)
    n += __popc(token_bits<false>(s, i, a, b));
  n = __reduce_add_sync(kAllLanes, n);
  return 1.f / ((by_sequence ? w.divisor : 1.f) * (float)n);
}

// Elements t .. t + 3 of an array of n; NaN-safe: what is beyond n is 0.
template <bool VEC>
__device__ __forceinline__ float4 load4(const float *p, uint64_t t, uint64_t n) {
  if (VEC && t + 4 <= n) return *reinterpret_cast<const float4 *>(p + t);
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (t < n) v.x = p[t];
  if (t + 1 < n) v.y = p[t + 1];
  if (t + 2 < n) v.z = p[t + 2];
  if (t + 3 < n) v.w = p[t + 3];
  return v;
}
template <bool VEC>
__device__ __forceinline__ void store4(float *p, uint64_t t, uint64_t n, float4 v) {
  if (VEC && t + 4 <= n) {
    *reinterpret_cast<float4 *>(p + t) = v;
    return;
  }
  if (t < n) p[t] = v.x;
  if (t + 1 < n) p[t + 1] = v.y;
  if (t + 2 < n) p[t + 2] = v.z;
  if (t + 3 < n) p[t + 3] = v.w;
}

}  // namespace edp
