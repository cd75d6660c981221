// k_loss.cu -- losses over the tokens of a packed batch, with their gradients:
// the clipped policy loss, the preference loss over pairs of sequences and the
// balance loss of a router.
#include <cmath>

#include "edp_loss.cuh"

namespace edp {

cudaError_t launch_policy_rows(edp_ctx *ctx, const Logits &z, const PolicyRule &rule,
                               const float *weight, const PolicyTokens &p, float *logp,
                               float *entropy, void *dz, uint64_t dstride, cudaStream_t s);

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ df warp_add(df v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const df b{__shfl_xor_sync(kAllLanes, v.hi, o), __shfl_xor_sync(kAllLanes, v.lo, o)};
    v = df_add(v, b);
  }
  return v;
}
// df_add, whose corrections are NaN where a sum is infinite.
__device__ __forceinline__ double df_value(df v) {
  return isfinite(v.hi) ? (double)v.hi + (double)v.lo : (double)v.hi;
}

// The sequence of token t: the last s with off[s] <= t (so an empty one holds
// none); t is in [off[0], off[n]).
__device__ __forceinline__ uint64_t sequence_of(const uint64_t *off, uint64_t n, uint64_t t) {
  uint64_t lo = 0, hi = n;  // off[lo] <= t < off[hi]
  while (hi - lo > 1) {
    const uint64_t mid = (lo + hi) / 2;
    if (off[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ bool counts(const TokenSet &s, uint64_t t) {
  if (s.mask && !s.mask[t]) return false;
  if (s.target && (uint32_t)s.target[t] >= s.vocab) return false;
  return !s.off || (t >= s.off[0] && t < s.off[s.n_seq]);
}

// Tokens that count in each sequence, a warp each (cnt), or in the batch (total).
__global__ void __launch_bounds__(kThreads)
k_count(TokenSet s, uint32_t *cnt, unsigned long long *total) {
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & 31;
  if (cnt) {
    const uint64_t step = (uint64_t)gridDim.x * kWarps;
    for (uint64_t q = (uint64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); q < s.n_seq; q += step) {
      uint32_t n = 0;
      const uint64_t end = min(s.off[q + 1], s.n);
      for (uint64_t t = s.off[q] + lane; t < end; t += 32) n += counts(s, t);
      n = __reduce_add_sync(kAllLanes, n);
      if (lane == 0) cnt[q] = n;
    }
    return;
  }
  uint32_t n = 0;
  for (uint64_t t = (uint64_t)blockIdx.x * kThreads + threadIdx.x; t < s.n;
       t += (uint64_t)gridDim.x * kThreads)
    n += counts(s, t);
  n = __reduce_add_sync(kAllLanes, n);
  if (lane == 0 && n) atomicAdd(total, (unsigned long long)n);
}

__device__ __forceinline__ float token_weight(const TokenSet &s, const uint32_t *cnt,
                                              const unsigned long long *total, uint64_t t) {
  if (!counts(s, t)) return 0.f;
  const float seqs = s.norm > 0.0 ? (float)s.norm : (float)s.n_seq;
  if (s.reduce == EDP_REDUCE_TOKEN_MEAN)
    return 1.f / (s.norm > 0.0 ? (float)s.norm : (float)*total);
  if (s.reduce == EDP_REDUCE_SEQ_SUM) return 1.f / seqs;
  return 1.f / (seqs * (float)cnt[sequence_of(s.off, s.n_seq, t)]);
}

__global__ void __launch_bounds__(kThreads)
k_token_weights(TokenSet s, const uint32_t *cnt, const unsigned long long *total, float *w) {
  pdl_wait();
  pdl_launch();
  for (uint64_t t = (uint64_t)blockIdx.x * kThreads + threadIdx.x; t < s.n;
       t += (uint64_t)gridDim.x * kThreads)
    w[t] = token_weight(s, cnt, total, t);
}

constexpr int kPolicySums = 8;  // pg, kl, entropy; above, below, ratio, old kl; tokens

// Adds K sums of every CTA, in the order of the CTAs: true in the last one, whose
// thread 0 then has the totals.  ticket: 0 before and after.
template <int K>
__device__ __forceinline__ bool grid_sums(const df (&mine)[K], double (&total)[K], double *part,
                                          uint32_t *ticket) {
  __shared__ double red[kWarps][K];
  __shared__ bool last;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const double v = df_value(warp_add(mine[k]));
    if (lane == 0) red[wid][k] = v;
  }
  __syncthreads();
  if (threadIdx.x < K) {
    double v = 0.0;
    for (int w = 0; w < kWarps; ++w) v += red[w][threadIdx.x];
    part[(uint64_t)blockIdx.x * K + threadIdx.x] = v;
    __threadfence();
  }
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return false;
  __threadfence();
  // each warp a run of CTAs, lanes in turn; joined in that order
  double acc[K];
#pragma unroll
  for (int k = 0; k < K; ++k) acc[k] = 0.0;
  for (uint32_t b = threadIdx.x; b < gridDim.x; b += kThreads)
#pragma unroll
    for (int k = 0; k < K; ++k) acc[k] += __ldcg(&part[(uint64_t)b * K + k]);
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int o = 16; o; o >>= 1) acc[k] += __shfl_xor_sync(kAllLanes, acc[k], o);
    if (lane == 0) red[wid][k] = acc[k];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      total[k] = 0.0;
      for (int w = 0; w < kWarps; ++w) total[k] += red[w][k];
    }
    *ticket = 0u;
  }
  return true;
}

// The policy loss of every token, its gradients and the batch's sums.  w: the
// tokens' weights, or NULL: found here.
__global__ void __launch_bounds__(kThreads)
k_policy(TokenSet s, PolicyTokens p, PolicyRule rule, const uint32_t *cnt, const float *w,
         float *loss, float *dlogp, float *dentropy, double *part, Ctrl *ctrl) {
  pdl_wait();
  df sum[kPolicySums];
#pragma unroll
  for (int k = 0; k < kPolicySums; ++k) sum[k] = df{0.f, 0.f};
  for (uint64_t t = (uint64_t)blockIdx.x * kThreads + threadIdx.x; t < s.n;
       t += (uint64_t)gridDim.x * kThreads) {
    const float wt = w ? w[t] : token_weight(s, cnt, &ctrl->loss_tokens, t);
    float g = 0.f, h = 0.f;
    if (wt != 0.f) {
      const PolicyToken o = policy_token(rule, p.logp[t], p.old_logp[t],
                                         p.ref_logp ? p.ref_logp[t] : 0.f, p.ref_logp != nullptr,
                                         p.adv[t]);
      const float by = rule.grad_scale * wt;
      g = by * o.dlogp;
      h = -by * rule.entropy_coef;
      sum[0] = df_add_f(sum[0], wt * o.pg);
      sum[1] = df_add_f(sum[1], wt * o.kl);
      if (p.entropy) sum[2] = df_add_f(sum[2], wt * p.entropy[t]);
      sum[3] = df_add_f(sum[3], o.above ? 1.f : 0.f);
      sum[4] = df_add_f(sum[4], o.below ? 1.f : 0.f);
      sum[5] = df_add_f(sum[5], o.ratio);
      sum[6] = df_add_f(sum[6], o.old_kl);
      sum[7] = df_add_f(sum[7], 1.f);
    }
    if (dlogp) dlogp[t] = g;
    if (dentropy) dentropy[t] = h;
  }
  double all[kPolicySums];
  if (!grid_sums(sum, all, part, &ctrl->loss_ticket) || threadIdx.x) return;
  const double n = all[7] > 0.0 ? all[7] : 1.0;
  loss[0] = (float)(all[0] + (rule.kl_coef != 0.f ? (double)rule.kl_coef * all[1] : 0.0) -
                    (rule.entropy_coef != 0.f ? (double)rule.entropy_coef * all[2] : 0.0));
  loss[1] = (float)all[0];
  loss[2] = (float)all[1];
  loss[3] = (float)all[2];
  for (int k = 4; k < 8; ++k) loss[k] = (float)(all[k - 1] / n);
  ctrl->loss_tokens = 0;
}

// ---- preference loss -----------------------------------------------------------

struct PrefRule {
  double beta, smooth, margin, norm, grad_scale;
  uint32_t kind, average;
};
// Gradients by a sequence's sum, as whole numbers of 2^-20 and of 2^-62: whole
// numbers add up in any order to the same.
struct SeqGrad {
  unsigned long long hi, lo;
};
constexpr double kHiUnit = 1.0 / 1048576.0;                 // 2^-20
constexpr double kLoUnit = 1.0 / 4611686018427387904.0;     // 2^-62
constexpr double kGradMost = 4194304.0;                     // 2^22

__device__ __forceinline__ void grad_add(SeqGrad *g, uint32_t *bad, double v) {
  if (!(fabs(v) < kGradMost)) {
    *bad = 1u;  // every writer writes the same
    return;
  }
  const double h = rint(v / kHiUnit);
  const double l = rint((v - h * kHiUnit) / kLoUnit);
  if (h != 0.0) atomicAdd(&g->hi, (unsigned long long)(long long)h);
  if (l != 0.0) atomicAdd(&g->lo, (unsigned long long)(long long)l);
}

// u of each sequence (a warp each) in fp64, its token count; the gradients cleared.
__global__ void __launch_bounds__(kThreads)
k_seq_ratio(TokenSet s, const float *logp, const float *ref, uint32_t average, double *u,
            uint32_t *cnt, SeqGrad *grad, uint32_t *bad, float *ratio) {
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & 31;
  const uint64_t step = (uint64_t)gridDim.x * kWarps;
  for (uint64_t q = (uint64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); q < s.n_seq; q += step) {
    df v{0.f, 0.f};
    uint32_t n = 0;
    const uint64_t end = min(s.off[q + 1], s.n);
    for (uint64_t t = s.off[q] + lane; t < end; t += 32)
      if (!s.mask || s.mask[t]) {
        v = df_add_f(v, logp[t]);
        if (ref) v = df_add_f(v, -ref[t]);
        ++n;
      }
    n = __reduce_add_sync(kAllLanes, n);
    double x = df_value(warp_add(v));
    if (average) x = n ? x / (double)n : 0.0;
    if (lane == 0) {
      u[q] = x;
      cnt[q] = n;
      grad[q] = SeqGrad{0, 0};
      bad[q] = 0;
      if (ratio) ratio[q] = (float)x;
    }
  }
}

__global__ void __launch_bounds__(kThreads)
k_pairs(PrefRule r, const int64_t *pair, uint32_t n_pair, uint64_t n_seq, const double *u,
        SeqGrad *grad, uint32_t *bad, float *loss, float *pair_loss, double *part, Ctrl *ctrl) {
  pdl_wait();
  df sum[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = df{0.f, 0.f};
  for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < n_pair; i += gridDim.x * kThreads) {
    const int64_t c = pair[2 * (uint64_t)i], x = pair[2 * (uint64_t)i + 1];
    float l = 0.f;
    if ((uint64_t)c >= n_seq || (uint64_t)x >= n_seq) {
      flag(ctrl, DEVERR_INDEX, (unsigned long long)((uint64_t)c >= n_seq ? c : x));
    } else {
      const double h = u[c] - u[x], d = r.beta * h - r.margin;
      double g;  // by u of the chosen
      if (r.kind == EDP_PREF_LOGISTIC) {
        const float df32 = (float)d, e = expf(-fabsf(df32));
        const float tail = log1pf(e);  // -ln s(|d|)
        const float up = tail + fmaxf(-df32, 0.f), down = tail + fmaxf(df32, 0.f);
        const float s = (float)r.smooth;
        l = s == 0.f ? up : fmaf(1.f - s, up, s * down);
        // 1 - e - s(d) = s(-d) - e
        const double sd = (double)(df32 > 0.f ? e / (1.f + e) : 1.f / (1.f + e));
        g = -r.beta * (sd - r.smooth);
      } else if (r.kind == EDP_PREF_HINGE) {
        l = (float)fmax(1.0 - d, 0.0);
        if (isnan(d)) l = (float)d;
        g = d < 1.0 ? -r.beta : 0.0;
      } else {
        const double y = h - 1.0 / (2.0 * r.beta);
        l = (float)(y * y);
        g = 2.0 * y;
      }
      if (isnan(d)) g = d;
      grad_add(&grad[c], &bad[c], g);
      grad_add(&grad[x], &bad[x], -g);
      sum[0] = df_add_f(sum[0], l);
      sum[1] = df_add_f(sum[1], h > 0.0 ? 1.f : 0.f);
      sum[2] = df_add(sum[2], df_split(r.beta * u[c]));
      sum[3] = df_add(sum[3], df_split(r.beta * u[x]));
    }
    if (pair_loss) pair_loss[i] = l;
  }
  pdl_launch();
  double all[4];
  if (!grid_sums(sum, all, part, &ctrl->loss_ticket) || threadIdx.x) return;
  loss[0] = (float)(all[0] / r.norm);
  for (int k = 1; k < 4; ++k) loss[k] = (float)(all[k] / (double)n_pair);
}

__global__ void __launch_bounds__(kThreads)
k_pref_grad(TokenSet s, PrefRule r, const uint32_t *cnt, const SeqGrad *grad, const uint32_t *bad,
            float *dlogp) {
  pdl_wait();
  pdl_launch();
  for (uint64_t t = (uint64_t)blockIdx.x * kThreads + threadIdx.x; t < s.n;
       t += (uint64_t)gridDim.x * kThreads) {
    float g = 0.f;
    if (counts(s, t)) {
      const uint64_t q = sequence_of(s.off, s.n_seq, t);
      double v = (double)(long long)grad[q].hi * kHiUnit + (double)(long long)grad[q].lo * kLoUnit;
      v *= r.grad_scale / (r.norm * (r.average ? (double)cnt[q] : 1.0));
      g = bad[q] ? __int_as_float(0x7fc00000) : (float)v;
    }
    dlogp[t] = g;
  }
}

// ---- balance loss ----------------------------------------------------------------

constexpr uint32_t kMaxExperts = 1024;
constexpr double kProbUnit = 1.0 / 1099511627776.0;  // 2^-40

// Sums that are whole numbers, so that the order of the adds does not matter.
struct BalanceSums {
  unsigned long long tokens;
  uint32_t bad, pad;  // a row was NaN
  unsigned long long prob[kMaxExperts];  // in units of 2^-40
};

__global__ void __launch_bounds__(kThreads)
k_expert_counts(const int32_t *sel, uint32_t top, const uint8_t *mask, uint64_t rows, uint32_t E,
                unsigned long long *counts, BalanceSums *sums, Ctrl *ctrl) {
  __shared__ uint32_t hist[kMaxExperts];
  __shared__ uint32_t tokens;
  pdl_wait();
  pdl_launch();
  for (uint32_t e = threadIdx.x; e < E; e += kThreads) hist[e] = 0;
  if (threadIdx.x == 0) tokens = 0;
  __syncthreads();
  for (uint64_t t = (uint64_t)blockIdx.x * kThreads + threadIdx.x; t < rows;
       t += (uint64_t)gridDim.x * kThreads) {
    if (mask && !mask[t]) continue;
    atomicAdd(&tokens, 1u);
    for (uint32_t k = 0; k < top; ++k) {
      const int32_t e = sel[t * top + k];
      if (e < 0) continue;
      if ((uint32_t)e < E) atomicAdd(&hist[e], 1u);
      else flag(ctrl, DEVERR_INDEX, (unsigned long long)e);
    }
  }
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < E; e += kThreads)
    if (hist[e]) atomicAdd(&counts[e], (unsigned long long)hist[e]);
  if (threadIdx.x == 0 && tokens) atomicAdd(&sums->tokens, (unsigned long long)tokens);
}

// A warp per row, EPL experts per lane.
template <typename T, int EPL>
__global__ void __launch_bounds__(kThreads)
k_balance(const T *z, uint64_t rows, uint64_t stride, uint32_t E, const uint8_t *mask,
          uint32_t top, const unsigned long long *counts, BalanceSums *sums, double coef,
          double grad_scale, float *loss, float *prob, T *dz, uint64_t dstride, Ctrl *ctrl) {
  __shared__ unsigned long long acc[kMaxExperts];
  __shared__ bool last;
  pdl_wait();
  const int lane = threadIdx.x & 31;
  for (uint32_t e = threadIdx.x; e < E; e += kThreads) acc[e] = 0;
  __syncthreads();
  const double N = (double)max(sums->tokens, 1ull);
  const double per = (double)E / ((double)top * N);  // f_e = counts[e] * per
  const float scale = (float)(grad_scale * coef / N);
  float f[EPL], ps[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const uint32_t e = lane + 32 * i;
    f[i] = e < E ? (float)((double)counts[e] * per) : 0.f;
    ps[i] = 0.f;
  }
  bool bad = false;
  for (uint64_t t = (uint64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); t < rows;
       t += (uint64_t)gridDim.x * kWarps) {
    const bool use = !mask || mask[t];
    float y[EPL], s = 0.f, fp = 0.f, m = kNegInf;
    if (use) {
      bool nan = false;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        const uint32_t e = lane + 32 * i;
        y[i] = e < E ? to_f32(z[t * stride + e]) : kNegInf;
        m = fmaxf(m, y[i]);
        nan |= isnan(y[i]);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAllLanes, m, o));
      if (m == kNegInf && !__any_sync(kAllLanes, nan)) {
        if (lane == 0) flag(ctrl, DEVERR_ROW, t);
        m = 0.f;  // every p is 0
      }
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        y[i] = ex2((y[i] - m) * (float)kLog2e);
        s += y[i];
        fp = fmaf(y[i], f[i], fp);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        s += __shfl_xor_sync(kAllLanes, s, o);
        fp += __shfl_xor_sync(kAllLanes, fp, o);
      }
      const float inv = s == 0.f ? 0.f : 1.f / s;
      fp *= inv;
      bad |= !isfinite(inv);
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        y[i] *= inv;
        ps[i] += y[i];
      }
    }
    if (dz) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        const uint32_t e = lane + 32 * i;
        if (e < E) dz[t * dstride + e] = from_f32<T>(use ? scale * y[i] * (f[i] - fp) : 0.f);
      }
    }
  }
  if (bad) atomicExch(&sums->bad, 1u);
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const uint32_t e = lane + 32 * i;
    if (e < E && isfinite(ps[i]))
      atomicAdd(&acc[e], (unsigned long long)__double2ull_rn((double)ps[i] / kProbUnit));
  }
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < E; e += kThreads)
    if (acc[e]) atomicAdd(&sums->prob[e], acc[e]);
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(&ctrl->loss_ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  __shared__ double red[kThreads];
  const bool nan = __ldcg(&sums->bad) != 0;
  double v = 0.0;
  for (uint32_t e = threadIdx.x; e < E; e += kThreads) {
    const double p = nan ? (double)__int_as_float(0x7fc00000)
                         : (double)__ldcg(&sums->prob[e]) * kProbUnit / N;
    if (prob) prob[e] = (float)p;
    v += (double)counts[e] * per * p;
  }
  red[threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < kThreads; ++i) v += red[i];
  loss[0] = (float)(coef * v);
  ctrl->loss_ticket = 0;
}

uint64_t blocks_of(const edp_ctx *c, uint64_t items, uint64_t each) {
  const uint64_t b = (items + each - 1) / each, most = 8ull * (uint64_t)c->coop_sms;
  return b < 1 ? 1 : b > most ? most : b;
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

// Scratch in turn, each part on a 16-byte boundary.
struct Carve {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t a = at;
    at += (bytes + 15) & ~(size_t)15;
    return a;
  }
};

bool counts_sequences(const TokenSet &s) { return s.reduce == EDP_REDUCE_SEQ_MEAN; }
bool counts_tokens(const TokenSet &s) {
  return s.reduce == EDP_REDUCE_TOKEN_MEAN && !(s.norm > 0.0);
}

cudaError_t launch_counts(edp_ctx *c, const TokenSet &s, uint32_t *cnt, cudaStream_t st) {
  if (counts_sequences(s))
    return launch_pdl(k_count, dim3((unsigned)blocks_of(c, s.n_seq, kWarps)), dim3(kThreads), st, s,
                      cnt, (unsigned long long *)nullptr);
  if (counts_tokens(s))
    return launch_pdl(k_count, dim3((unsigned)blocks_of(c, s.n, 4 * kThreads)), dim3(kThreads), st,
                      s, (uint32_t *)nullptr, &c->ctrl->loss_tokens);
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_policy_loss(edp_ctx *c, const edp_policy_config &cfg, const TokenSet &set,
                               const PolicyTokens &p, float *loss, float *dlogp,
                               float *dentropy, cudaStream_t s) {
  const uint64_t grid = blocks_of(c, set.n, 4 * kThreads);
  Carve k;
  const size_t part = k.take(grid * kPolicySums * sizeof(double));
  const size_t cnt = k.take(counts_sequences(set) ? set.n_seq * sizeof(uint32_t) : 0);
  void *blk = nullptr;
  cudaError_t e = ctx_scratch(c, k.at, s, &blk);
  if (e != cudaSuccess) return e;
  uint8_t *b = (uint8_t *)blk;
  e = launch_counts(c, set, (uint32_t *)(b + cnt), s);
  if (e != cudaSuccess) return e;
  return launch_pdl(k_policy, dim3((unsigned)grid), dim3(kThreads), s, set, p, policy_rule(cfg),
                    (const uint32_t *)(b + cnt), (const float *)nullptr, loss, dlogp, dentropy,
                    (double *)(b + part), c->ctrl);
}

cudaError_t launch_policy_loss_logits(edp_ctx *c, const edp_policy_config &cfg,
                                      const TokenSet &set, const PolicyTokens &p,
                                      const Logits &z, float *loss, float *logp, float *entropy,
                                      void *dz, uint64_t dstride, cudaStream_t s) {
  const uint64_t grid = blocks_of(c, set.n, 4 * kThreads);
  const bool own_entropy = !entropy && cfg.entropy_coef > 0.0;
  Carve k;
  const size_t part = k.take(grid * kPolicySums * sizeof(double));
  const size_t cnt = k.take(counts_sequences(set) ? set.n_seq * sizeof(uint32_t) : 0);
  const size_t w = k.take(set.n * sizeof(float));
  const size_t ent = k.take(own_entropy ? set.n * sizeof(float) : 0);
  void *blk = nullptr;
  cudaError_t e = ctx_scratch(c, k.at, s, &blk);
  if (e != cudaSuccess) return e;
  uint8_t *b = (uint8_t *)blk;
  float *weight = (float *)(b + w);
  if (own_entropy) entropy = (float *)(b + ent);
  const PolicyRule rule = policy_rule(cfg);
  e = launch_counts(c, set, (uint32_t *)(b + cnt), s);
  if (e != cudaSuccess) return e;
  e = launch_pdl(k_token_weights, dim3((unsigned)blocks_of(c, set.n, kThreads)), dim3(kThreads), s,
                 set, (const uint32_t *)(b + cnt),
                 (const unsigned long long *)&c->ctrl->loss_tokens, weight);
  if (e != cudaSuccess) return e;
  e = launch_policy_rows(c, z, rule, weight, p, logp, entropy, dz, dstride, s);
  if (e != cudaSuccess) return e;
  PolicyTokens q = p;
  q.logp = logp;
  q.entropy = entropy;
  return launch_pdl(k_policy, dim3((unsigned)grid), dim3(kThreads), s, set, q, rule,
                    (const uint32_t *)nullptr, (const float *)weight, loss, (float *)nullptr,
                    (float *)nullptr, (double *)(b + part), c->ctrl);
}

cudaError_t launch_preference_loss(edp_ctx *c, const edp_preference_config &cfg,
                                   const TokenSet &set, const float *logp, const float *ref,
                                   const int64_t *pair, uint32_t n_pair, float *loss,
                                   float *ratio, float *pair_loss, float *dlogp,
                                   cudaStream_t s) {
  const uint64_t grid = blocks_of(c, n_pair, kThreads);
  Carve k;
  const size_t part = k.take(grid * 4 * sizeof(double));
  const size_t u = k.take(set.n_seq * sizeof(double));
  const size_t grad = k.take(set.n_seq * sizeof(SeqGrad));
  const size_t cnt = k.take(set.n_seq * sizeof(uint32_t));
  const size_t bad = k.take(set.n_seq * sizeof(uint32_t));
  void *blk = nullptr;
  cudaError_t e = ctx_scratch(c, k.at, s, &blk);
  if (e != cudaSuccess) return e;
  uint8_t *b = (uint8_t *)blk;
  const PrefRule rule{cfg.beta, cfg.label_smoothing, cfg.margin,
                      cfg.norm > 0.0 ? cfg.norm : (double)n_pair, cfg.grad_scale, cfg.kind,
                      cfg.average};
  e = launch_pdl(k_seq_ratio, dim3((unsigned)blocks_of(c, set.n_seq, kWarps)), dim3(kThreads), s,
                 set, logp, ref, cfg.average, (double *)(b + u), (uint32_t *)(b + cnt),
                 (SeqGrad *)(b + grad), (uint32_t *)(b + bad), ratio);
  if (e != cudaSuccess) return e;
  e = launch_pdl(k_pairs, dim3((unsigned)grid), dim3(kThreads), s, rule, pair, n_pair, set.n_seq,
                 (const double *)(b + u), (SeqGrad *)(b + grad), (uint32_t *)(b + bad), loss,
                 pair_loss, (double *)(b + part), c->ctrl);
  if (e != cudaSuccess || !dlogp) return e;
  return launch_pdl(k_pref_grad, dim3((unsigned)blocks_of(c, set.n, 4 * kThreads)), dim3(kThreads),
                    s, set, rule, (const uint32_t *)(b + cnt), (const SeqGrad *)(b + grad),
                    (const uint32_t *)(b + bad), dlogp);
}

namespace {
template <typename T>
cudaError_t balance_as(edp_ctx *c, const Logits &z, uint32_t top, double coef, double grad_scale,
                       float *loss, const int64_t *counts, float *prob, void *dz,
                       uint64_t dstride, BalanceSums *sums, cudaStream_t s) {
  auto go = [&](auto kern) {
    const uint64_t b = blocks_of(c, z.rows, 4 * kWarps);
    return launch_pdl(kern, dim3((unsigned)b), dim3(kThreads), s, (const T *)z.z, z.rows,
                      z.stride, z.vocab, z.mask, top, (const unsigned long long *)counts, sums,
                      coef, grad_scale, loss, prob, (T *)dz, dstride, c->ctrl);
  };
  if (z.vocab <= 32) return go(k_balance<T, 1>);
  if (z.vocab <= 64) return go(k_balance<T, 2>);
  if (z.vocab <= 128) return go(k_balance<T, 4>);
  if (z.vocab <= 256) return go(k_balance<T, 8>);
  if (z.vocab <= 512) return go(k_balance<T, 16>);
  return go(k_balance<T, 32>);
}
}  // namespace

cudaError_t launch_balance_loss(edp_ctx *c, const Logits &z, const int32_t *sel, uint32_t top,
                                double coef, double grad_scale, float *loss, int64_t *counts,
                                float *prob, void *dz, uint64_t dstride, cudaStream_t s) {
  void *blk = nullptr;
  cudaError_t e = ctx_scratch(c, sizeof(BalanceSums), s, &blk);
  if (e != cudaSuccess) return e;
  BalanceSums *sums = (BalanceSums *)blk;
  e = cudaMemsetAsync(sums, 0, sizeof *sums, s);
  if (e != cudaSuccess) return e;
  e = cudaMemsetAsync(counts, 0, z.vocab * sizeof(int64_t), s);
  if (e != cudaSuccess) return e;
  // both plainly: what they wait for is a memory operation
  const uint64_t b = blocks_of(c, z.rows, kThreads);
  k_expert_counts<<<dim3((unsigned)b), dim3(kThreads), 0, s>>>(
      sel, top, z.mask, z.rows, z.vocab, (unsigned long long *)counts, sums, c->ctrl);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  switch (z.dtype) {
    case EDP_BF16:
      return balance_as<__nv_bfloat16>(c, z, top, coef, grad_scale, loss, counts, prob, dz,
                                       dstride, sums, s);
    case EDP_F16:
      return balance_as<__half>(c, z, top, coef, grad_scale, loss, counts, prob, dz, dstride,
                                sums, s);
    default:
      return balance_as<float>(c, z, top, coef, grad_scale, loss, counts, prob, dz, dstride, sums,
                               s);
  }
}

}  // namespace edp
