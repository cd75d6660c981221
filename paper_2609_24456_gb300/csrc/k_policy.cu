// k_policy.cu -- the clipped policy loss over the tokens of a packed batch, with
// its gradients by the log-probabilities and the entropies.
//
// One pass over the tokens (16 to 32 bytes each), in chunks of 4 per thread, so
// that sequences of any lengths load the CTAs alike.  A token's weight needs the
// number of tokens that count, in the batch or in its sequence: a pass over the
// mask (1 byte a token) counts them per chunk first, and a chunk adds up those
// of the sequences that reach into it from outside.  A batch of one chunk
// counts for itself and is one launch.
#include <cmath>

#include "edp_loss.cuh"

namespace edp {

cudaError_t launch_policy_rows(edp_ctx *ctx, const Logits &z, const PolicyRule &rule,
                               const float *weight, const PolicyTokens &p, float *logp,
                               float *entropy, void *dz, uint64_t dstride, cudaStream_t s);

namespace {

constexpr int kThreads = 512;      // a chunk of 2,048 tokens
constexpr int kSmallThreads = 1024;  // a batch of up to 4,096 tokens, in one CTA
constexpr int kSums = 7;  // pg, kl, entropy; ratio, old kl; clipped above, below

struct Weighting {
  const uint32_t *chunk;              // tokens that count, per chunk
  const unsigned long long *tokens;   // and in all
  bool by_mask;   // SEQ_MEAN: sequences' tokens are counted, not their lengths
  bool by_total;  // TOKEN_MEAN: the divisor is *tokens
  float fixed;    // otherwise, but for SEQ_MEAN: every weight
  float divisor;  // SEQ_MEAN: sequences
};

struct Range {
  uint64_t first, end;  // the tokens that the sequences hold
};
__device__ __forceinline__ Range token_range(const TokenSet &s) {
  if (!s.off) return {0, s.n};
  return {s.off[0], min(s.off[s.n_seq], s.n)};
}

template <int NT>
__device__ __forceinline__ uint32_t cta_sum(uint32_t v, uint32_t *red) {
  v = __reduce_add_sync(kAllLanes, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  uint32_t x = (threadIdx.x & 31) < NT / 32 ? red[threadIdx.x & 31] : 0;
  return __reduce_add_sync(kAllLanes, x);
}

// Tokens that count, per chunk, and their total.
template <bool VEC>
__global__ void __launch_bounds__(kThreads)
k_token_counts(TokenSet s, uint32_t *chunk, unsigned long long *total) {
  __shared__ uint32_t red[kThreads / 32];
  pdl_wait();
  pdl_launch();
  const Range r = token_range(s);
  uint32_t sum = 0;
  for (uint64_t c = blockIdx.x; c * 4 * kThreads < s.n; c += gridDim.x) {
    const uint32_t bits = token_bits<VEC>(s, (c * kThreads + threadIdx.x) * 4, r.first, r.end);
    if (chunk) {
      const uint32_t n = cta_sum<kThreads>(__popc(bits), red);
      if (threadIdx.x == 0) chunk[c] = n;
    } else {
      sum += __popc(bits);
    }
  }
  if (chunk) return;
  sum = cta_sum<kThreads>(sum, red);
  if (threadIdx.x == 0 && sum) atomicAdd(total, (unsigned long long)sum);
}

// Weights of a chunk's tokens, where each sequence has its own.
template <int NT>
struct ChunkWeights {
  uint32_t pre[NT];   // tokens that count before a thread's, shifted by 4, and its bits
  uint32_t red[NT / 32];
  uint32_t lo, hi;    // the sequences of the chunk's first and last token
  uint32_t before, after;  // tokens of lo before the chunk, of hi after it

  // tokens that count among the chunk's first x
  __device__ __forceinline__ uint32_t upto(uint32_t x) const {
    if (x >= 4u * NT) return (pre[NT - 1] >> 4) + __popc(pre[NT - 1] & 15u);
    const uint32_t p = pre[x >> 2];
    return (p >> 4) + __popc(p & ((1u << (x & 3u)) - 1u));
  }

  template <bool VEC>
  __device__ __forceinline__ void fill(const TokenSet &s, const Weighting &w, const Range &r,
                                       uint64_t t0, uint32_t bits) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    constexpr uint64_t C = 4ull * NT;
    __syncthreads();  // the chunk before is done with
    if (wid < 2) {
      const uint64_t t = wid == 0 ? t0 : min(t0 + C, r.end) - 1;
      const uint32_t q = sequence_of_warp(s.off, (uint32_t)s.n_seq, t);
      if (lane == 0) (wid == 0 ? lo : hi) = q;
    }
    if (w.by_mask) {
      uint32_t n = __popc(bits), incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(kAllLanes, incl, o);
        if (lane >= o) incl += y;
      }
      if (lane == 31) red[wid] = incl;
      __syncthreads();
      const uint32_t x = lane < wid ? red[lane] : 0;
      pre[threadIdx.x] = ((__reduce_add_sync(kAllLanes, x) + incl - n) << 4) | bits;
    }
    __syncthreads();
    if (!w.by_mask) return;
    // of the sequence that comes in from the left and of the one that goes on to
    // the right: the chunks that they fill, and the part of the one at their end
    const uint64_t a = s.off[lo], b = min(s.off[hi + 1], r.end);
    uint32_t left = 0, right = 0;
    const uint64_t c = t0 / C;
    if (a < t0) {
      const uint64_t ca = a / C;
      for (uint64_t k = ca + 1 + threadIdx.x; k < c; k += NT) left += __ldcg(&w.chunk[k]);
      left += __popc(token_bits<VEC>(s, ca * C + 4 * threadIdx.x, max(a, r.first), r.end));
    }
    if (b > t0 + C) {
      const uint64_t cb = (b - 1) / C;
      for (uint64_t k = c + 1 + threadIdx.x; k < cb; k += NT) right += __ldcg(&w.chunk[k]);
      right += __popc(token_bits<VEC>(s, cb * C + 4 * threadIdx.x, r.first, b));
    }
    left = __reduce_add_sync(kAllLanes, left);
    right = __reduce_add_sync(kAllLanes, right);
    if (threadIdx.x == 0) before = after = 0;
    __syncthreads();
    if (lane == 0 && left) atomicAdd(&before, left);
    if (lane == 0 && right) atomicAdd(&after, right);
    __syncthreads();
  }

  // weights of a thread's tokens t .. t + 3
  __device__ __forceinline__ void get(const TokenSet &s, const Weighting &w, const Range &r,
                                      uint64_t t0, uint64_t t, uint32_t bits, float (&out)[4]) {
    constexpr uint64_t C = 4ull * NT;
    uint32_t q = 0;
    uint64_t end = 0;
    float each = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      out[i] = 0.f;
      if (!(bits >> i & 1u)) continue;
      if (t + i >= end) {
        q = sequence_of(s.off, end ? q : lo, hi + 1, t + i);
        const uint64_t a = s.off[q];
        end = min(s.off[q + 1], r.end);
        uint64_t n = end - a;
        if (w.by_mask) {
          n = upto((uint32_t)(end - t0 < C ? end - t0 : C)) - upto(a > t0 ? (uint32_t)(a - t0) : 0u);
          if (a < t0) n += before;
          if (end > t0 + C) n += after;
        }
        each = 1.f / (w.divisor * (float)n);
      }
      out[i] = each;
    }
  }
};

enum class Weights { kFixed, kSequence, kGiven };

// What the tokens weigh where all weigh the same; n: those of the one chunk, if
// there is only one.
__device__ __forceinline__ float same_weight(const Weighting &w, uint32_t n, bool one) {
  if (!w.by_total) return w.fixed;
  const unsigned long long k = one ? n : __ldcg(w.tokens);
  return 1.f / (float)k;
}

// The weights alone, for the form from logits.
template <bool VEC>
__global__ void __launch_bounds__(kThreads)
k_token_weights(TokenSet s, Weighting w, bool sequences, float *out) {
  __shared__ ChunkWeights<kThreads> cw;
  pdl_wait();
  pdl_launch();
  const Range r = token_range(s);
  for (uint64_t t0 = (uint64_t)blockIdx.x * 4 * kThreads; t0 < s.n;
       t0 += (uint64_t)gridDim.x * 4 * kThreads) {
    const uint64_t t = t0 + 4 * threadIdx.x;
    const uint32_t bits = token_bits<VEC>(s, t, r.first, r.end);
    float v[4] = {};
    if (sequences) {
      if (t0 < r.end) {
        cw.fill<VEC>(s, w, r, t0, bits);
        cw.get(s, w, r, t0, t, bits, v);
      }
    } else {
      const bool one = s.n <= 4 * kThreads;
      const float f = same_weight(w, one ? cta_sum<kThreads>(__popc(bits), cw.red) : 0u, one);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = bits >> i & 1u ? f : 0.f;
    }
    store4<VEC>(out, t, s.n, make_float4(v[0], v[1], v[2], v[3]));
  }
}

// The policy loss of every token, its gradients and the batch's sums.
template <int NT, Weights W, bool VEC>
__global__ void __launch_bounds__(NT, 1536 / NT)
k_policy(TokenSet s, PolicyTokens p, PolicyRule rule, Weighting w, const float *given, float *loss,
         float *dlogp, float *dentropy, Pair *part, Ctrl *ctrl) {
  __shared__ ChunkWeights<W == Weights::kSequence ? NT : 32> cw;
  __shared__ uint32_t red[NT / 32];
  __shared__ Pair total[kSums + 1];
  pdl_wait();
  Pair sum[kSums + 1];
#pragma unroll
  for (int k = 0; k <= kSums; ++k) sum[k] = Pair{0.f, 0.f};
  const Range r = token_range(s);
  for (uint64_t t0 = (uint64_t)blockIdx.x * 4 * NT; t0 < s.n;
       t0 += (uint64_t)gridDim.x * 4 * NT) {
    const uint64_t t = t0 + 4 * threadIdx.x;
    const float4 lp = load4<VEC>(p.logp, t, s.n), od = load4<VEC>(p.old_logp, t, s.n);
    const float4 ad = load4<VEC>(p.adv, t, s.n);
    float4 rf = make_float4(0.f, 0.f, 0.f, 0.f), en = rf;
    if (p.ref_logp) rf = load4<VEC>(p.ref_logp, t, s.n);
    if (p.entropy) en = load4<VEC>(p.entropy, t, s.n);
    uint32_t bits;
    float wt[4];
    if (W == Weights::kGiven) {
      const float4 g = load4<VEC>(given, t, s.n);
      wt[0] = g.x, wt[1] = g.y, wt[2] = g.z, wt[3] = g.w;
      bits = (g.x != 0.f) | (g.y != 0.f) << 1 | (g.z != 0.f) << 2 | (g.w != 0.f) << 3;
    } else {
      bits = token_bits<VEC>(s, t, r.first, r.end);
      if (W == Weights::kSequence) {
        wt[0] = wt[1] = wt[2] = wt[3] = 0.f;
        if (t0 < r.end) {
          cw.template fill<VEC>(s, w, r, t0, bits);
          cw.get(s, w, r, t0, t, bits, wt);
        }
      } else {
        const bool one = NT == kSmallThreads;
        const float f = same_weight(w, one && w.by_total ? cta_sum<NT>(__popc(bits), red) : 0u,
                                    one);
        wt[0] = wt[1] = wt[2] = wt[3] = f;
      }
    }
    const float l4[4] = {lp.x, lp.y, lp.z, lp.w}, o4[4] = {od.x, od.y, od.z, od.w};
    const float a4[4] = {ad.x, ad.y, ad.z, ad.w}, r4[4] = {rf.x, rf.y, rf.z, rf.w};
    const float e4[4] = {en.x, en.y, en.z, en.w};
    float g4[4], h4[4], add[5] = {};
    uint32_t above = 0, below = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g4[i] = h4[i] = 0.f;
      if (!(bits >> i & 1u)) continue;
      const PolicyToken o =
          policy_token(rule, l4[i], o4[i], r4[i], p.ref_logp != nullptr, a4[i]);
      const float by = rule.grad_scale * wt[i];
      g4[i] = by * o.dlogp;
      h4[i] = -by * rule.entropy_coef;
      add[0] = fmaf(wt[i], o.pg, add[0]);
      add[1] = fmaf(wt[i], o.kl, add[1]);
      add[2] = fmaf(wt[i], e4[i], add[2]);
      add[3] += o.ratio;
      add[4] += o.old_kl;
      above += o.above;
      below += o.below;
    }
#pragma unroll
    for (int k = 0; k < 5; ++k) pair_add(sum[k], add[k]);
    pair_add(sum[5], (float)above);
    pair_add(sum[6], (float)below);
    pair_add(sum[7], (float)__popc(bits));
    if (dlogp) store4<VEC>(dlogp, t, s.n, make_float4(g4[0], g4[1], g4[2], g4[3]));
    if (dentropy) store4<VEC>(dentropy, t, s.n, make_float4(h4[0], h4[1], h4[2], h4[3]));
  }
  if (!grid_join<NT, kSums + 1>(sum, total, part, &ctrl->loss_ticket)) return;
  if (threadIdx.x == 0) {
    double v[kSums + 1];
    for (int k = 0; k <= kSums; ++k) v[k] = pair_value(total[k]);
    const double n = v[7] > 0.0 ? v[7] : 1.0;
    loss[0] = (float)(v[0] + (rule.kl_coef != 0.f ? (double)rule.kl_coef * v[1] : 0.0) -
                      (rule.entropy_coef != 0.f ? (double)rule.entropy_coef * v[2] : 0.0));
    loss[1] = (float)v[0];
    loss[2] = (float)v[1];
    loss[3] = (float)v[2];
    loss[4] = (float)(v[5] / n);
    loss[5] = (float)(v[6] / n);
    loss[6] = (float)(v[3] / n);
    loss[7] = (float)(v[4] / n);
    ctrl->loss_tokens = 0;
  }
}

PolicyRule policy_rule(const edp_policy_config &c) {
  PolicyRule r;
  r.low = (float)(1.0 - c.clip_low);
  r.high = (float)(1.0 + c.clip_high);
  r.dual = (float)c.dual_clip;
  r.ln_low = (float)std::log1p(-c.clip_low);
  r.ln_high = (float)std::log1p(c.clip_high);
  r.ln_dual = c.dual_clip > 0.0 ? (float)std::log(c.dual_clip) : __builtin_huge_valf();
  r.kl_coef = (float)c.kl_coef;
  r.entropy_coef = (float)c.entropy_coef;
  r.grad_scale = (float)c.grad_scale;
  r.kl = c.kl;
  return r;
}

template <typename... P>
bool aligned_to(uintptr_t bytes, P... p) {
  return (((uintptr_t)p | ...) & (bytes - 1)) == 0;
}

// Chunks, at most `per_sm` CTAs per SM.
unsigned chunk_grid(const edp_ctx *c, uint64_t n, int threads, unsigned per_sm) {
  const uint64_t chunks = (n + 4ull * threads - 1) / (4ull * threads);
  const uint64_t most = (uint64_t)per_sm * (uint64_t)c->coop_sms;
  return (unsigned)(chunks < most ? chunks : most);
}

// The scratch of a call and what it is for.
struct Plan {
  Weighting w;
  bool sequences, counts, vec;
  Pair *part;
  uint32_t *chunk;
  float *weight, *entropy;
};

cudaError_t make_plan(edp_ctx *c, const TokenSet &set, bool vec, bool one_chunk, bool weights,
                      bool entropy, cudaStream_t s, Plan *p) {
  p->vec = vec;
  p->sequences = set.reduce == EDP_REDUCE_SEQ_MEAN;
  const bool chosen = set.mask || set.target;
  p->w = Weighting{};
  p->w.by_mask = p->sequences && chosen;
  p->w.by_total = set.reduce == EDP_REDUCE_TOKEN_MEAN && !(set.norm > 0.0);
  p->w.divisor = (float)(set.norm > 0.0 ? set.norm : (double)set.n_seq);
  p->w.fixed = set.reduce == EDP_REDUCE_TOKEN_MEAN ? (float)(1.0 / set.norm)
                                                   : 1.f / p->w.divisor;
  p->counts = !one_chunk && (p->w.by_mask || p->w.by_total);
  const size_t part = ((size_t)(kSums + 1) * 3 * c->coop_sms * sizeof(Pair) + 15) & ~(size_t)15;
  const uint64_t chunks = (set.n + 4 * kThreads - 1) / (4 * kThreads);
  const size_t chunk = p->w.by_mask ? (chunks * sizeof(uint32_t) + 15) & ~(size_t)15 : 0;
  const size_t row = (set.n * sizeof(float) + 15) & ~(size_t)15;
  void *blk = nullptr;
  const cudaError_t e =
      ctx_scratch(c, part + chunk + row * ((size_t)weights + (size_t)entropy), s, &blk);
  if (e != cudaSuccess) return e;
  uint8_t *b = (uint8_t *)blk;
  p->part = (Pair *)b;
  p->chunk = p->w.by_mask ? (uint32_t *)(b + part) : nullptr;
  p->weight = (float *)(b + part + chunk);
  p->entropy = (float *)(b + part + chunk + (weights ? row : 0));
  p->w.chunk = p->chunk;
  p->w.tokens = &c->ctrl->loss_tokens;
  return cudaSuccess;
}

cudaError_t launch_counts(edp_ctx *c, const TokenSet &set, const Plan &p, cudaStream_t s) {
  if (!p.counts) return cudaSuccess;
  auto kern = p.vec ? k_token_counts<true> : k_token_counts<false>;
  return launch_pdl(kern, dim3(chunk_grid(c, set.n, kThreads, 4)), dim3(kThreads), s, set, p.chunk,
                    &c->ctrl->loss_tokens);
}

template <Weights W>
cudaError_t launch_policy(edp_ctx *c, const TokenSet &set, const PolicyTokens &t,
                          const PolicyRule &rule, const Plan &p, bool small, const float *given,
                          float *loss, float *dlogp, float *dentropy, cudaStream_t s) {
  if (small) {
    auto kern = p.vec ? k_policy<kSmallThreads, W, true> : k_policy<kSmallThreads, W, false>;
    return launch_pdl(kern, dim3(1), dim3(kSmallThreads), s, set, t, rule, p.w, given, loss, dlogp,
                      dentropy, p.part, c->ctrl);
  }
  auto kern = p.vec ? k_policy<kThreads, W, true> : k_policy<kThreads, W, false>;
  return launch_pdl(kern, dim3(chunk_grid(c, set.n, kThreads, 3)), dim3(kThreads), s, set, t, rule,
                    p.w, given, loss, dlogp, dentropy, p.part, c->ctrl);
}

}  // namespace

cudaError_t launch_policy_loss(edp_ctx *c, const edp_policy_config &cfg, const TokenSet &set,
                               const PolicyTokens &t, float *loss, float *dlogp,
                               float *dentropy, cudaStream_t s) {
  const bool vec = aligned_to(16, t.logp, t.old_logp, t.ref_logp, t.adv, t.entropy, dlogp,
                              dentropy) && aligned_to(4, set.mask);
  const bool small = set.n <= 4 * kSmallThreads;
  Plan p;
  cudaError_t e = make_plan(c, set, vec, small, false, false, s, &p);
  if (e != cudaSuccess) return e;
  e = launch_counts(c, set, p, s);
  if (e != cudaSuccess) return e;
  const PolicyRule rule = policy_rule(cfg);
  return p.sequences ? launch_policy<Weights::kSequence>(c, set, t, rule, p, small, nullptr, loss,
                                                         dlogp, dentropy, s)
                     : launch_policy<Weights::kFixed>(c, set, t, rule, p, small, nullptr, loss,
                                                      dlogp, dentropy, s);
}

cudaError_t launch_policy_loss_logits(edp_ctx *c, const edp_policy_config &cfg,
                                      const TokenSet &set, const PolicyTokens &t,
                                      const Logits &z, float *loss, float *logp, float *entropy,
                                      void *dz, uint64_t dstride, cudaStream_t s) {
  const bool vec = aligned_to(16, t.old_logp, t.ref_logp, t.adv, logp, entropy) &&
                   aligned_to(4, set.mask);
  const bool own_entropy = !entropy && cfg.entropy_coef > 0.0;
  Plan p;
  cudaError_t e = make_plan(c, set, vec, set.n <= 4 * kThreads, true, own_entropy, s, &p);
  if (e != cudaSuccess) return e;
  if (own_entropy) entropy = p.entropy;
  e = launch_counts(c, set, p, s);
  if (e != cudaSuccess) return e;
  auto kern = vec ? k_token_weights<true> : k_token_weights<false>;
  e = launch_pdl(kern, dim3(chunk_grid(c, set.n, kThreads, 3)), dim3(kThreads), s, set, p.w,
                 p.sequences, p.weight);
  if (e != cudaSuccess) return e;
  const PolicyRule rule = policy_rule(cfg);
  e = launch_policy_rows(c, z, rule, p.weight, t, logp, entropy, dz, dstride, s);
  if (e != cudaSuccess) return e;
  PolicyTokens q = t;
  q.logp = logp;
  q.entropy = entropy;
  return launch_policy<Weights::kGiven>(c, set, q, rule, p, set.n <= 4 * kSmallThreads, p.weight,
                                        loss, nullptr, nullptr, s);
}

}  // namespace edp
