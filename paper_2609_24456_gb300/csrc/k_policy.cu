// k_policy.cu -- the clipped policy loss over the tokens of a packed batch, with
// its gradients by the log-probabilities and the entropies.
//
// One pass over the tokens (16 to 32 bytes each).  Each CTA has a run of them, its
// warps take tiles of 128 in turn, without barriers, whatever the sequences'
// lengths.  A token's weight needs the number of tokens that count, in the batch
// or in its sequence: the mask (1 byte a token) is counted by blocks of 512
// first, and a warp per sequence makes its weight from the blocks inside it and
// the bytes at its ends.  A batch of up to 4,096 tokens is one CTA that counts for
// itself, in one launch.
//
// 8,192 sequences of 128 to 4,096 tokens, masked, with a reference (17.3 M tokens of 21
// bytes, weights by sequence): 80 us, 4.5 TB/s; the floor is 54 us.  What bounds it:
// issue (about 100 instructions a token, half of them selections and comparisons of the
// clipping and the masks, at 2.8 of 4 a cycle from 32 warps of 64 registers, up to 72 bytes
// of them spilled), then the two launches before it (5 us).
// Two CTAs of 512 threads per SM; 85 us with three of 384, 94 with five of 256, 91 with
// the next tile loaded ahead (80 registers, spilled).  fp64 sums, or a search for each
// token's sequence, as in the first kernel: 521 us.
#include <cmath>
#include <type_traits>

#include "edp_loss.cuh"

namespace edp {

cudaError_t launch_policy_rows(edp_ctx *ctx, const Logits &z, const PolicyRule &rule,
                               const RowWeights &w, const PolicyTokens &p, float *logp,
                               float *entropy, void *dz, uint64_t dstride, bool early,
                               cudaStream_t s);

namespace {

constexpr int kThreads = 512;
constexpr int kPerSm = 2;  // CTAs of k_policy, in one wave
constexpr int kSmallThreads = 1024;  // a batch of up to 4,096 tokens, in one CTA
constexpr uint32_t kBlock = 512;     // tokens counted together
constexpr int kSums = 8;  // pg, kl, entropy; ratio - 1, old kl; clipped above, below; tokens
// Tiles between two additions to the sums: 32 tokens a lane in fp32, 2^-19 of their sum at
// the worst.
constexpr int kFlush = 8;

template <int NT>
__device__ __forceinline__ uint32_t cta_sum(uint32_t v, uint32_t *red) {
  v = __reduce_add_sync(kAllLanes, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  const uint32_t x = (threadIdx.x & 31) < NT / 32 ? red[threadIdx.x & 31] : 0;
  return __reduce_add_sync(kAllLanes, x);
}

// Tokens that count in t .. t + 15.
template <bool VEC>
__device__ __forceinline__ uint32_t count16(const TokenSet &s, uint64_t t, const Range &r) {
  if (VEC && s.mask && !s.target && t >= r.first && t + 16 <= r.end) {
    const uint4 m = *reinterpret_cast<const uint4 *>(s.mask + t);
    return some_bytes(m.x) + some_bytes(m.y) + some_bytes(m.z) + some_bytes(m.w);
  }
  uint32_t n = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) n += __popc(token_bits<VEC>(s, t + 4 * k, r.first, r.end));
  return n;
}

// Tokens that count, by blocks (a warp each) or in all.
template <bool VEC>
__global__ void __launch_bounds__(kThreads)
k_token_counts(TokenSet s, uint32_t *block, unsigned long long *total) {
  __shared__ uint32_t red[kThreads / 32];
  pdl_wait();
  pdl_launch();
  const Range r = token_range(s);
  const int lane = threadIdx.x & 31;
  const uint64_t step = (uint64_t)gridDim.x * (kThreads / 32);
  uint32_t sum = 0;
  for (uint64_t b = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
       b * kBlock < s.n; b += step) {
    const uint32_t n = count16<VEC>(s, b * kBlock + 16 * lane, r);
    if (block) {
      const uint32_t all = __reduce_add_sync(kAllLanes, n);
      if (lane == 0) block[b] = all;
    }
    sum += n;
  }
  if (block) return;
  sum = cta_sum<kThreads>(sum, red);
  if (threadIdx.x == 0 && sum) atomicAdd(total, (unsigned long long)sum);
}

// Tokens that count among [a, b), below a block's worth, by a warp.
__device__ __forceinline__ uint32_t count_few(const TokenSet &s, uint64_t a, uint64_t b) {
  uint32_t n = 0;
#pragma unroll 4
  for (uint64_t t = a + (threadIdx.x & 31); t < b; t += 32)
    n += (!s.mask || s.mask[t]) && (!s.target || (uint32_t)s.target[t] < s.vocab);
  return n;
}

// Each sequence's weight, 1 / (divisor tokens); block: NULL where every token counts.
__global__ void __launch_bounds__(kThreads)
k_sequence_weights(TokenSet s, const uint32_t *block, float divisor, float *weight) {
  // behind k_token_counts, which waited for all that came before this call, what comes
  // after this kernel may start at once and read what it does not wait for
  if (block) pdl_launch();
  pdl_wait();
  if (!block) pdl_launch();
  const int lane = threadIdx.x & 31;
  const uint64_t step = (uint64_t)gridDim.x * (kThreads / 32);
  for (uint64_t q = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); q < s.n_seq;
       q += step) {
    const uint64_t a = s.off[q], b = min(s.off[q + 1], s.n);
    uint64_t n = b > a ? b - a : 0;
    if (block && n) {
      const uint64_t ka = (a + kBlock - 1) / kBlock, kb = b / kBlock;  // whole blocks
      uint32_t some = 0;
      if (ka >= kb) {
        some = count_few(s, a, b);
      } else {
        for (uint64_t k = ka + lane; k < kb; k += 32) some += __ldcg(&block[k]);
        some += count_few(s, a, ka * kBlock) + count_few(s, kb * kBlock, b);
      }
      // a lane's count fits 32 bits up to 2^37 tokens (2 TB), the sequence's need not
      n = ((uint64_t)__reduce_add_sync(kAllLanes, some >> 16) << 16) +
          __reduce_add_sync(kAllLanes, some & 0xffffu);
    }
    if (lane == 0) weight[q] = n ? 1.f / (divisor * (float)n) : 0.f;
  }
}

// Sequences' counts in a batch of one CTA: a prefix over its tokens.
template <int NT>
struct OneCta {
  uint32_t pre[NT];  // tokens that count before a thread's, shifted by 4, and its bits
  uint32_t red[NT / 32];

  // tokens that count among the first x
  __device__ __forceinline__ uint32_t upto(uint32_t x) const {
    if (x >= 4u * NT) return (pre[NT - 1] >> 4) + __popc(pre[NT - 1] & 15u);
    const uint32_t p = pre[x >> 2];
    return (p >> 4) + __popc(p & ((1u << (x & 3u)) - 1u));
  }
  __device__ __forceinline__ void fill(uint32_t bits) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t n = __popc(bits);
    uint32_t incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(kAllLanes, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) red[wid] = incl;
    __syncthreads();
    const uint32_t x = lane < wid ? red[lane] : 0;
    pre[threadIdx.x] = ((__reduce_add_sync(kAllLanes, x) + incl - n) << 4) | bits;
    __syncthreads();
  }
};

// What the tokens of a lane, t .. t + 3, weigh.  q0, q1: the sequences of the tile's
// first and last token.
template <typename F>
__device__ __forceinline__ void sequence_weights(const TokenSet &s, uint64_t end, uint64_t t,
                                                 uint32_t bits, uint32_t q0, uint32_t q1, F of,
                                                 float (&w)[4]) {
  uint32_t q = q0;
  uint64_t next = 0;
  float each = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = 0.f;
    if (!(bits >> i & 1u)) continue;
    if (t + i >= next) {
      q = sequence_of(s.off, q, q1 + 1, t + i);
      next = s.off[q + 1];
      each = of(q, s.off[q], min(next, end));
    }
    w[i] = each;
  }
}

// The policy loss of every token, its gradients and the batch's sums.  SEQ: a weight
// for each sequence.  NT == kSmallThreads: one CTA, which counts for itself.
template <int NT, bool SEQ, bool VEC, Kl KL>
__global__ void __launch_bounds__(NT, NT == kSmallThreads ? 1 : kPerSm)
k_policy(TokenSet s, PolicyTokens p, PolicyRule rule, Weighting w, float divisor, float *loss,
         float *dlogp, float *dentropy, Pair *part, bool early, Ctrl *ctrl) {
  constexpr bool kOne = NT == kSmallThreads;
  constexpr uint32_t kWarps = NT / 32;
  __shared__ OneCta<kOne ? NT : 32> one;
  __shared__ Pair total[kSums];
  // early: the kernel before is of this call and waited, itself or the one before it,
  // for all that came before; it writes logp and entropy (one CTA) or the weights alone
  if (!early) pdl_wait();
  bool waited = !early;
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const Range r = token_range(s);
  float fixed = w.fixed;
  Pair sum[kSums];
#pragma unroll
  for (int k = 0; k < kSums; ++k) sum[k] = Pair{0.f, 0.f};
  float add[5] = {};
  uint32_t above = 0, below = 0, tokens = 0;
  auto flush = [&] {
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      pair_add(sum[k], add[k]);
      add[k] = 0.f;
    }
  };
  // the CTA's tokens c0 .. c0 + cn - 1, in tiles in turn by its warps; places
  // within them are 32-bit numbers.  Tiles below `whole` count but for the mask.
  const uint64_t tiles = (s.n + kTile - 1) / kTile;
  const uint64_t c0 = blockIdx.x * ((tiles + gridDim.x - 1) / gridDim.x) * kTile;
  const uint64_t c1 = min(s.n, c0 + (tiles + gridDim.x - 1) / gridDim.x * kTile);
  const uint32_t cn = kOne ? 4 * NT : c1 > c0 ? (uint32_t)(c1 - c0) : 0;
  const uint32_t whole = VEC && !s.target && c0 >= r.first && r.end > c0
                             ? (uint32_t)min((uint64_t)cn, r.end - c0) : 0;
  const float *lpc = p.logp + c0, *odc = p.old_logp + c0, *adc = p.adv + c0;
  const float *rfc = p.ref_logp + c0, *enc = p.entropy + c0;
  const uint8_t *mc = s.mask + c0;
  struct Tile {
    float4 lp, od, ad, rf, en;
    uint32_t m;  // a byte per token, 0: it does not count
  };
  const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
  auto load = [&](uint32_t i) {
    Tile x;
    const uint32_t e = i + 4 * lane;
    x.rf = x.en = none;
    if (i + kTile <= whole) {
      if (!kOne) x.lp = *reinterpret_cast<const float4 *>(lpc + e);
      x.od = *reinterpret_cast<const float4 *>(odc + e);
      x.ad = *reinterpret_cast<const float4 *>(adc + e);
      if (KL != Kl::kNone) x.rf = *reinterpret_cast<const float4 *>(rfc + e);
      if (!kOne && p.entropy) x.en = *reinterpret_cast<const float4 *>(enc + e);
      x.m = s.mask ? *reinterpret_cast<const uint32_t *>(mc + e) : 0xffffffffu;
    } else {
      const uint64_t t = c0 + e;
      if (!kOne) x.lp = load4<VEC>(p.logp, t, s.n);
      x.od = load4<VEC>(p.old_logp, t, s.n);
      x.ad = load4<VEC>(p.adv, t, s.n);
      if (KL != Kl::kNone) x.rf = load4<VEC>(p.ref_logp, t, s.n);
      if (!kOne && p.entropy) x.en = load4<VEC>(p.entropy, t, s.n);
      const uint32_t bits = token_bits<VEC>(s, t, r.first, r.end);
      x.m = (bits & 1u) | (bits & 2u) << 7 | (bits & 4u) << 14 | (bits & 8u) << 21;
    }
    return x;
  };
  SeqWalk walk;
  // where the walk's sequence and the one after it end in the CTA's tokens, and
  // their weights
  uint32_t next = 0, after = 0;
  float here = 0.f, there = 0.f;
  bool known = false;
  auto place = [&](uint64_t t) {
    return t > c0 ? (uint32_t)min(t - c0, (uint64_t)cn + kTile) : 0u;
  };
  const uint32_t share = (cn / kTile + kWarps - 1 + (cn % kTile != 0)) / kWarps * kTile;
  const uint32_t stop = (uint32_t)min((uint64_t)cn, (uint64_t)(wid + 1) * share);
  uint32_t i = wid * share;
#pragma unroll 1
  while (i < stop) {
   const uint32_t group = min(stop, i + kFlush * kTile);
#pragma unroll 1
   for (; i < group; i += kTile) {
    Tile x = load(i);
    if (!kOne && !waited) {
      pdl_wait();
      waited = true;
    }
    bool b[4];  // which of the lane's tokens count
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = x.m & (0xffu << (8 * k));
    auto bits = [&] { return b[0] | b[1] << 1 | b[2] << 2 | b[3] << 3; };
    float wt[4];
    if (kOne && SEQ) {
      one.fill(bits());
      sequence_weights(s, r.end, c0 + i + 4 * lane, bits(), 0, (uint32_t)s.n_seq - 1,
                       [&](uint32_t, uint64_t a, uint64_t b) {
                         return 1.f / (divisor * (float)(one.upto((uint32_t)b) -
                                                         one.upto((uint32_t)a)));
                       }, wt);
    } else if (SEQ) {
      const uint32_t n = (uint32_t)s.n_seq;
      if (c0 + i >= r.end) {
        wt[0] = wt[1] = wt[2] = wt[3] = 0.f;
      } else {
        if (i >= next) {  // on to the sequence of the tile's first token
          if (known && after > i) {
            ++walk.q;
            next = after;
            here = there;
          } else {
            if (known) {
              walk.next = c0 + next;
              walk.to(s.off, n, c0 + i);
            } else {
              walk.start(s.off, n, c0 + i);
            }
            next = place(walk.next);
            here = __ldcg(&w.sequence[walk.q]);
          }
          known = true;
          // and what will be wanted at its end
          after = walk.q + 1 < n ? place(s.off[walk.q + 2]) : next;
          there = walk.q + 1 < n ? __ldcg(&w.sequence[walk.q + 1]) : 0.f;
        }
        wt[0] = wt[1] = wt[2] = wt[3] = here;
        if (i + kTile > next) {
          if (i + kTile <= after || c0 + after >= r.end) {  // two sequences
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (i + 4 * lane + k >= next) wt[k] = there;
          } else {
            SeqWalk to = walk;
            to.next = c0 + next;
            to.to(s.off, n, min(c0 + i + kTile, r.end) - 1);
            sequence_weights(s, r.end, c0 + i + 4 * lane, bits(), walk.q, to.q,
                             [&](uint32_t q, uint64_t, uint64_t) {
                               return __ldcg(&w.sequence[q]);
                             }, wt);
          }
        }
      }
    } else {
      if (w.by_range) fixed = r.end > r.first ? 1.f / (float)(r.end - r.first) : 0.f;
      if (!kOne && w.tokens) fixed = 1.f / (float)max(__ldcg(w.tokens), 1ull);
      if (kOne && w.tokens) fixed = 1.f / (float)max(cta_sum<NT>(__popc(bits()), one.red), 1u);
      wt[0] = wt[1] = wt[2] = wt[3] = fixed;
    }
    if (kOne) {
      if (!waited) pdl_wait();
      waited = true;
      x.lp = load4<VEC>(p.logp, c0 + i + 4 * lane, s.n);
      if (p.entropy) x.en = load4<VEC>(p.entropy, c0 + i + 4 * lane, s.n);
    }
    // what does not count is 0 from here on, whatever it held, and so is its gradient
    const float l4[4] = {x.lp.x, x.lp.y, x.lp.z, x.lp.w};
    const float o4[4] = {x.od.x, x.od.y, x.od.z, x.od.w};
    const float a4[4] = {x.ad.x, x.ad.y, x.ad.z, x.ad.w};
    const float r4[4] = {x.rf.x, x.rf.y, x.rf.z, x.rf.w};
    const float e4[4] = {x.en.x, x.en.y, x.en.z, x.en.w};
    float g4[4], d4[4], q4[4], adv4[4], most = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      d4[k] = b[k] ? l4[k] - o4[k] : 0.f;
      q4[k] = KL != Kl::kNone && b[k] ? r4[k] - l4[k] : 0.f;
      adv4[k] = b[k] ? a4[k] : 0.f;
      most = fmaxf(most, fabsf(d4[k]));
      if (KL == Kl::kK3) most = fmaxf(most, fabsf(q4[k]));
    }
    auto take = [&](auto near) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const PolicyToken o =
            policy_token<KL, decltype(near)::value>(rule, d4[k], q4[k], adv4[k]);
        g4[k] = b[k] ? rule.grad_scale * wt[k] * o.dlogp : 0.f;
        add[0] = fmaf(wt[k], o.pg, add[0]);
        if (KL != Kl::kNone) add[1] = fmaf(wt[k], o.kl, add[1]);
        add[3] += o.ratio1;
        add[4] += o.old_kl;
        above += o.above;
        below += o.below;
      }
    };
    if (__any_sync(kAllLanes, most >= 1.f)) take(std::false_type{});
    else take(std::true_type{});
    if (p.entropy) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (b[k]) add[2] = fmaf(wt[k], e4[k], add[2]);
    }
    tokens += some_bytes(x.m);
    auto store = [&](float *out, float4 v) {
      if (i + kTile <= whole) *reinterpret_cast<float4 *>(out + c0 + i + 4 * lane) = v;
      else store4<VEC>(out, c0 + i + 4 * lane, s.n, v);
    };
    if (dlogp) store(dlogp, make_float4(g4[0], g4[1], g4[2], g4[3]));
    if (dentropy) {
      const float h = -rule.grad_scale * rule.entropy_coef;
      store(dentropy, make_float4(b[0] ? h * wt[0] : 0.f, b[1] ? h * wt[1] : 0.f,
                                  b[2] ? h * wt[2] : 0.f, b[3] ? h * wt[3] : 0.f));
    }
   }
   flush();
  }
  if (!waited) pdl_wait();  // a warp without tokens: before the CTA's sums go out
  sum[5] = pair_of(above);
  sum[6] = pair_of(below);
  sum[7] = pair_of(tokens);
  if (!grid_join<NT, kSums>(sum, total, part, &ctrl->loss_ticket)) return;
  // an output per thread, in pairs: fp64 divisions one after another cost a microsecond
  if (threadIdx.x < 8) {
    const uint32_t k = threadIdx.x;
    const float n = total[7].hi + total[7].lo;
    if (k == 0) {
      df l = as_df(total[0]);
      if (rule.kl_coef != 0.f) l = df_add(l, df_mul(as_df(total[1]), rule.kl_both));
      if (rule.entropy_coef != 0.f) l = df_add(l, df_mul(as_df(total[2]), rule.less_entropy));
      // pairs lose infinities, plain numbers do not
      loss[0] = isfinite(l.hi) ? l.hi
                : total[0].hi + (rule.kl_coef != 0.f ? rule.kl_coef * total[1].hi : 0.f) -
                      (rule.entropy_coef != 0.f ? rule.entropy_coef * total[2].hi : 0.f);
      ctrl->loss_tokens = 0;
    } else if (k < 4) {
      loss[k] = as_df(total[k - 1]).hi;
    } else {
      const int from = k == 4 ? 5 : k == 5 ? 6 : k == 6 ? 3 : 4;
      const float mean = n > 0.f ? as_df(total[from]).hi / n : 0.f;
      loss[k] = k == 6 && n > 0.f ? 1.f + mean : mean;
    }
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
  auto both = [](double v) {
    const float hi = (float)v;
    return df{hi, (float)(v - (double)hi)};
  };
  r.kl_both = both(c.kl_coef);
  r.less_entropy = both(-c.entropy_coef);
  return r;
}

template <typename... P>
bool aligned_to(uintptr_t bytes, P... p) {
  return (((uintptr_t)p | ...) & (bytes - 1)) == 0;
}

unsigned at_most(uint64_t want, uint64_t most) {
  return (unsigned)(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace

cudaError_t plan_weights(edp_ctx *c, const TokenSet &set, bool one_cta, bool per_token,
                         cudaStream_t s, Plan *p) {
  const uint64_t sms = (uint64_t)c->coop_sms;
  p->sequences = set.reduce == EDP_REDUCE_SEQ_MEAN;
  p->divisor = (float)(set.norm > 0.0 ? set.norm : (double)set.n_seq);
  const bool chosen = set.mask || set.target;
  const bool mean = set.reduce == EDP_REDUCE_TOKEN_MEAN && !(set.norm > 0.0);
  const bool by_total = mean && chosen;
  p->w = Weighting{};
  p->w.fixed = 1.f / p->divisor;
  p->w.by_range = mean && !chosen;
  const bool blocks = p->sequences && chosen && !one_cta;
  p->early = !one_cta && (blocks || by_total);
  size_t at = 0;
  auto take = [&](bool want, uint64_t bytes) {
    const size_t a = at;
    if (want) at += (bytes + 15) & ~(size_t)15;
    return a;
  };
  const size_t part = take(true, kSums * kPerSm * sms * sizeof(Pair));
  const size_t weight = take(p->sequences && !one_cta, set.n_seq * sizeof(float));
  const size_t block = take(blocks, (set.n + kBlock - 1) / kBlock * sizeof(uint32_t));
  const size_t own = take(per_token, set.n * sizeof(float));
  void *blk = nullptr;
  cudaError_t e = ctx_scratch(c, at, s, &blk);
  if (e != cudaSuccess) return e;
  uint8_t *b = (uint8_t *)blk;
  p->part = (Pair *)(b + part);
  p->per_token = (float *)(b + own);
  if (by_total) p->w.tokens = &c->ctrl->loss_tokens;
  if (one_cta) return cudaSuccess;
  const unsigned warps = kThreads / 32;
  if (blocks || by_total) {
    auto kern = aligned_to(16, set.mask) ? k_token_counts<true> : k_token_counts<false>;
    const uint64_t want = (set.n + kBlock * warps - 1) / (kBlock * warps);
    e = launch_pdl(kern, dim3(at_most(want, 4 * sms)), dim3(kThreads), s, set,
                   blocks ? (uint32_t *)(b + block) : nullptr, &c->ctrl->loss_tokens);
    if (e != cudaSuccess) return e;
  }
  if (p->sequences) {
    p->w.sequence = (float *)(b + weight);
    e = launch_pdl(k_sequence_weights, dim3(at_most((set.n_seq + warps - 1) / warps, 4 * sms)),
                   dim3(kThreads), s, set,
                   blocks ? (const uint32_t *)(b + block) : nullptr, p->divisor,
                   (float *)(b + weight));
  }
  return e;
}

void forget_count(edp_ctx *c, const Plan &p, cudaStream_t s) {
  if (p.w.tokens) cudaMemsetAsync(&c->ctrl->loss_tokens, 0, sizeof c->ctrl->loss_tokens, s);
}

namespace {

template <bool VEC>
cudaError_t launch_policy(edp_ctx *c, const TokenSet &set, const PolicyTokens &t,
                          const PolicyRule &rule, const Plan &p, bool one_cta, bool early,
                          float *loss, float *dlogp, float *dentropy, cudaStream_t s) {
  auto go = [&](auto kern, unsigned grid, int threads) {
    return launch_pdl(kern, dim3(grid), dim3(threads), s, set, t, rule, p.w, p.divisor, loss,
                      dlogp, dentropy, p.part, early, c->ctrl);
  };
  const uint64_t want = (set.n + 4 * kThreads - 1) / (4 * kThreads);
  const unsigned grid = at_most(want, (uint64_t)kPerSm * (uint64_t)c->coop_sms);
  auto kind = [&](auto kl) {
    constexpr Kl KL = decltype(kl)::value;
    if (one_cta)
      return p.sequences ? go(k_policy<kSmallThreads, true, VEC, KL>, 1, kSmallThreads)
                         : go(k_policy<kSmallThreads, false, VEC, KL>, 1, kSmallThreads);
    return p.sequences ? go(k_policy<kThreads, true, VEC, KL>, grid, kThreads)
                       : go(k_policy<kThreads, false, VEC, KL>, grid, kThreads);
  };
  if (!t.ref_logp) return kind(std::integral_constant<Kl, Kl::kNone>{});
  return rule.kl == EDP_KL_K3 ? kind(std::integral_constant<Kl, Kl::kK3>{})
                              : kind(std::integral_constant<Kl, Kl::kOther>{});
}

}  // namespace

cudaError_t launch_policy_loss(edp_ctx *c, const edp_policy_config &cfg, const TokenSet &set,
                               const PolicyTokens &t, float *loss, float *dlogp,
                               float *dentropy, cudaStream_t s) {
  const bool one_cta = set.n <= 4 * kSmallThreads;
  Plan p;
  cudaError_t e = plan_weights(c, set, one_cta, false, s, &p);
  if (e != cudaSuccess) return e;
  const bool vec = aligned_to(16, t.logp, t.old_logp, t.ref_logp, t.adv, t.entropy, dlogp,
                              dentropy) && aligned_to(4, set.mask);
  const PolicyRule rule = policy_rule(cfg);
  e = vec ? launch_policy<true>(c, set, t, rule, p, one_cta, p.early, loss, dlogp, dentropy, s)
          : launch_policy<false>(c, set, t, rule, p, one_cta, p.early, loss, dlogp, dentropy, s);
  if (e != cudaSuccess) forget_count(c, p, s);
  return e;
}

cudaError_t launch_policy_loss_logits(edp_ctx *c, const edp_policy_config &cfg,
                                      const TokenSet &set, const PolicyTokens &t,
                                      const Logits &z, float *loss, float *logp, float *entropy,
                                      void *dz, uint64_t dstride, cudaStream_t s) {
  const bool own_entropy = !entropy && cfg.entropy_coef > 0.0;
  Plan p;
  const uint64_t means = set.reduce == EDP_REDUCE_SEQ_MEAN ? set.n_seq : 1;
  const bool few = set.n <= kFewRows && set.n <= kFewTokens * means;
  cudaError_t e = plan_weights(c, set, few, own_entropy, s, &p);
  if (e != cudaSuccess) return e;
  if (own_entropy) entropy = p.per_token;
  const PolicyRule rule = policy_rule(cfg);
  const bool counted = p.sequences || p.w.tokens;
  const RowWeights w{set, few && counted, p.w.sequence, p.w.tokens, p.w.fixed, p.divisor};
  e = launch_policy_rows(c, z, rule, w, t, logp, entropy, dz, dstride, p.early, s);
  if (e != cudaSuccess) {
    forget_count(c, p, s);
    return e;
  }
  PolicyTokens q = t;
  q.logp = logp;
  q.entropy = entropy;
  const bool one_cta = set.n <= 4 * kSmallThreads;
  const bool vec = aligned_to(16, t.old_logp, t.ref_logp, t.adv, logp, entropy) &&
                   aligned_to(4, set.mask);
  e = vec ? launch_policy<true>(c, set, q, rule, p, one_cta, one_cta, loss, nullptr, nullptr, s)
          : launch_policy<false>(c, set, q, rule, p, one_cta, one_cta, loss, nullptr, nullptr, s);
  if (e != cudaSuccess) forget_count(c, p, s);
  return e;
}

}  // namespace edp
