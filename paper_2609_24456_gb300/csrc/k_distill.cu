// k_distill.cu -- the distillation loss of rows of logits against a teacher's lists, and
// the gradient of the logits.
//
// The teacher gives up to 128 tokens of a row with their log-probabilities, and with
// `rest` the logarithm of what all other tokens have together.  The student's
// distribution q = softmax(z / T) falls into the same classes, q_i of an entry and q_r of
// all else, and the loss is a divergence f(p, q) between the classes.  For a token j of
// class b, with f' the derivatives by q and G = sum_b q_b f'_b,
//   dz_j = (q_j / T) (f'_b - G)
//   sum p ln(p/q):                    q f' = -p             G = -P, P = sum of all p
//   sum q ln(q/p):                    f' = ln(q/p) + 1      G = loss + 1
//   B sum p ln(p/m) + A sum q ln(q/m),
//     m = B p + A q, A = 1 - B:       f' = A ln(q/m)        G = A sum q ln(q/m)
// so that every token outside of the list has the same factor of its 2^y.
//
// q_r = 1 - sum q_i would lose what it is of when the list holds nearly all: the entries
// are taken out of the row (set to -infinity in shared memory) before its sums, which then
// are those of the rest, relative to its own maximum; the entries join them afterwards.
#include <cmath>

#include "edp_rows.cuh"

namespace edp {
namespace {

constexpr int kThreads = 384;
// CTAs per SM, which bound the registers: as many as parts of 76 KB allow
constexpr int kCtas = 3;
enum class Rest { kGrad, kZero, kCareful };

struct DistillRule {
  uint32_t kind;
  float beta, alpha, ln_beta, ln_alpha;  // of the mixture: the teacher's share, the student's
  float inv_tt;                          // 1 / the teacher's temperature
  float grad_scale;
};
struct TeacherLists {
  const int32_t *ids;
  const float *value, *rest;
  uint32_t top;
};

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kAllLanes, x, o));
  return x;
}
__device__ __forceinline__ float warp_add(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kAllLanes, x, o);
  return x;
}
// ln(e^a + e^b)
__device__ __forceinline__ float log_add(float a, float b) {
  return fmaxf(a, b) + log1pf(expf(-fabsf(a - b)));
}
// weight log, 0 without weight whatever the logarithm
__device__ __forceinline__ float weigh(float weight, float log) {
  return weight == 0.f ? 0.f : weight * log;
}

// A row's entries over a warp's lanes, E each: entry k = lane + 32 i.  id < 0: none.
template <int E>
struct Entries {
  int32_t id[E];
  float lp[E], z[E];  // the teacher's log-probability, the student's logit
};

// What the classes give: the loss, the factor of 2^y of the tokens outside of the list
// (before `by`), and each entry's gradient (before `by`) in the place of its logit.
struct Classes {
  float loss, outside;
};
template <int E>
__device__ __forceinline__ Classes classes(const DistillRule &r, Entries<E> &e, bool has_rest,
                                           float lpr, const RowSum &rest, float M, float c,
                                           float inv_t) {
  const float left = rest.m == kNegInf ? rest.s : rest.s * ex2((rest.m - M) * c);
  float S = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) S += e.id[i] >= 0 ? ex2((e.z[i] - M) * c) : 0.f;
  S = warp_add(S) + left;
  const float ln = logf(S), inv = 1.f / S;
  const float qr = left * inv;
  const float lqr = rest.s == 0.f ? kNegInf : (rest.m - M) * inv_t + logf(rest.s) - ln;
  const float pr = has_rest ? expf(lpr) : 0.f;
  Classes o;
  if (r.kind == EDP_DISTILL_FORWARD) {
    float l = 0.f, P = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e.id[i] >= 0) {
        const float p = expf(e.lp[i]);
        l += weigh(p, e.lp[i] - ((e.z[i] - M) * inv_t - ln));
        P += p;
      }
    o.loss = warp_add(l) + weigh(pr, lpr - lqr);
    P = warp_add(P) + pr;
    o.outside = fmaf(P, qr, -pr);
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e.id[i] >= 0) e.z[i] = fmaf(P, ex2((e.z[i] - M) * c) * inv, -expf(e.lp[i]));
  } else if (r.kind == EDP_DISTILL_REVERSE) {
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e.id[i] >= 0) {
        const float q = ex2((e.z[i] - M) * c) * inv;
        const float d = (e.z[i] - M) * inv_t - ln - e.lp[i];
        l += weigh(q, d);
        e.z[i] = q;
        e.lp[i] = d;
      }
    o.loss = warp_add(l) + weigh(qr, lqr - lpr);
    o.outside = weigh(qr, lqr - lpr - o.loss);
#pragma unroll
    for (int i = 0; i < E; ++i) e.z[i] = weigh(e.z[i], e.lp[i] - o.loss);
  } else {
    float l = 0.f, g = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e.id[i] >= 0) {
        const float lp = e.lp[i], lq = (e.z[i] - M) * inv_t - ln;
        const float q = ex2((e.z[i] - M) * c) * inv;
        const float lm = log_add(lp + r.ln_beta, lq + r.ln_alpha);
        l += weigh(r.beta * expf(lp), lp - lm);
        g += weigh(r.alpha * q, lq - lm);
        e.z[i] = q;
        e.lp[i] = lq - lm;
      }
    const float lmr = log_add(lpr + r.ln_beta, lqr + r.ln_alpha);
    g = warp_add(g) + weigh(r.alpha * qr, lqr - lmr);
    o.loss = warp_add(l) + weigh(r.beta * pr, lpr - lmr) + g;
    o.outside = weigh(qr, fmaf(r.alpha, lqr - lmr, -g));
#pragma unroll
    for (int i = 0; i < E; ++i) e.z[i] = weigh(e.z[i], fmaf(r.alpha, e.lp[i], -g));
  }
  o.outside = rest.s == 0.f ? 0.f : o.outside / rest.s;
  return o;
}

// The weighted loss of a row, from one CTA of each row; the last of them adds up all
// rows in a fixed order and leaves the counters at 0.
__device__ __forceinline__ void conclude(float weighted, float *per_row, float *loss,
                                         Ctrl *ctrl) {
  constexpr int NW = kThreads / 32;
  __shared__ Pair sums[NW];
  __shared__ bool last;
  if (threadIdx.x == 0) {
    last = true;
    if (gridDim.x > 1) {
      __stcg(per_row + blockIdx.x, weighted);
      __threadfence();
      last = atomicAdd(&ctrl->loss_ticket, 1u) == gridDim.x - 1;
    } else {
      loss[0] = weighted;
    }
  }
  if (gridDim.x == 1) {
    if (threadIdx.x == 0) ctrl->loss_tokens = 0;
    return;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  Pair a{0.f, 0.f};
  for (uint32_t i = threadIdx.x; i < gridDim.x; i += kThreads) pair_add(a, __ldcg(per_row + i));
  a = warp_join(a);
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  if (lane == 0) sums[wid] = a;
  __syncthreads();
  if (wid) return;
  a = warp_join(lane < NW ? sums[lane] : Pair{0.f, 0.f});
  if (lane == 0) {
    loss[0] = as_df(a).hi;
    ctrl->loss_ticket = 0;
    ctrl->loss_tokens = 0;
  }
}

// A cluster of gridDim.y CTAs per row, each with its part in shared memory.
template <typename T, bool BACK, int E>
__global__ void __launch_bounds__(kThreads, kCtas)
k_distill(RowArgs a, RowWeights weights, bool by_range, TeacherLists lists, DistillRule rule,
          float *loss, float *row_loss, float *per_row, void *dz, uint64_t dstride, bool early,
          Ctrl *ctrl) {
  constexpr int NT = kThreads;
  constexpr bool F = kFused<T>;
  using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
  extern __shared__ uint4 resident[];
  __shared__ RowSum red[NT / 32];
  __shared__ float4 parts[2][8];  // what the cluster's CTAs send: m, S, weight, list's maximum
  __shared__ RowGrad grad;
  __shared__ Rest rest;
  __shared__ unsigned long long bar, sent[2];
  const uint64_t t = blockIdx.x;
  const uint32_t part = blockIdx.y, np = gridDim.y;
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 1);
    for (int k = 0; k < 2; ++k) {
      mbar_init(&sent[k], 1);
      mbar_arrive_tx(&sent[k], np * sizeof(float4));
    }
    mbar_init_fence();
  }
  __syncthreads();
  // early: the kernel before is of this call, waited for all that came before it and
  // writes the weights alone
  if (!early) pdl_wait();
  pdl_launch();
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  T *d = reinterpret_cast<T *>(dz) + t * dstride + first;
  if ((a.mask && !a.mask[t]) || !in_sequences(weights, t)) {
    if (BACK) part_zero<T, NT>(d, n);
    if (early) pdl_wait();  // so that what waits for this kernel finds the weights
    if (part) return;
    if (row_loss && threadIdx.x == 0) row_loss[t] = 0.f;
    conclude(0.f, per_row, loss, ctrl);
    return;  // the whole cluster
  }
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride, *p = row + first;
  // the part keeps its place within 16 bytes
  T *held = reinterpret_cast<T *>(resident) + ((uintptr_t)p & 15u) / sizeof(T);
  const Span<T> sp(p, n);
  if (threadIdx.x == 0 && sp.vecs) {
    mbar_arrive_tx(&bar, sp.vecs * 16);
    bulk_load(held + sp.head, p + sp.head, sp.vecs * 16, &bar, policy_normal());
  }
  if (threadIdx.x < sp.head + sp.tail) {
    const uint32_t i =
        threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * Vec16<T>::kN;
    held[i] = p[i];
  }
  if (np > 1) cluster_started();
  // The first warp's, beside the copy: the row's weight, the list and its logits (those of
  // other parts too, before a CTA can have written its gradient there).
  float w = 0.f, lpr = 0.f;
  int32_t strange = -1;  // an id >= vocab
  Entries<E> e;
  if (early) pdl_wait();
  if (wid == 0) {
    const uint64_t at = t * lists.top;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const uint32_t k = lane + 32 * i;
      e.id[i] = k < lists.top ? lists.ids[at + k] : -1;
      e.lp[i] = k < lists.top ? lists.value[at + k] : kNegInf;
    }
    if (lists.rest) lpr = lists.rest[t];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if (e.lp[i] == kNegInf) e.id[i] = -1;
      if (e.id[i] >= 0 && (uint32_t)e.id[i] >= a.vocab) {
        strange = e.id[i];
        e.id[i] = -1;
      }
      e.z[i] = e.id[i] >= 0 ? to_f32(row[e.id[i]]) : kNegInf;
    }
    if (by_range) {
      const Range r = token_range(weights.set);
      w = 1.f / (float)(r.end - r.first);
    } else {
      w = row_weight(weights, t);
    }
    if (!lists.rest) {  // the list's own softmax
      float m = kNegInf, s = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (e.id[i] >= 0) m = fmaxf(m, e.lp[i]);
      m = warp_max(m);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        e.lp[i] = (e.lp[i] - m) * rule.inv_tt;
        s += e.id[i] >= 0 ? expf(e.lp[i]) : 0.f;
      }
      const float ln = logf(warp_add(s));
#pragma unroll
      for (int i = 0; i < E; ++i) e.lp[i] -= ln;
    }
  }
  if (sp.vecs && !mbar_wait(&bar, 0, kRowWaitNs)) {
    if (threadIdx.x == 0) flag(ctrl, DEVERR_TIMEOUT, t);
    mbar_wait(&bar, 0, kRowWaitNs);  // bounded: the copy lands before the CTA ends
  }
  __syncthreads();
  bool twice = false;
  if (wid == 0) {
    // Each entry leaves its number in its place and looks whether it is still there.
    Bits *place = reinterpret_cast<Bits *>(held);
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e.id[i] >= 0 && (uint32_t)e.id[i] - first < n)
        place[(uint32_t)e.id[i] - first] = (Bits)(lane + 32 * i);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e.id[i] >= 0 && (uint32_t)e.id[i] - first < n)
        twice |= place[(uint32_t)e.id[i] - first] != (Bits)(lane + 32 * i);
    twice = __any_sync(kAllLanes, twice);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e.id[i] >= 0 && (uint32_t)e.id[i] - first < n)
        held[(uint32_t)e.id[i] - first] = from_f32<T>(kNegInf);
  }
  __syncthreads();
  float weighted = 0.f;
  // The first warp joins the CTA's sums, gives them to the cluster's other CTAs and
  // takes theirs, and makes of all what the part's gradient needs.
  auto finish = [&](auto fused, int round) {
    constexpr bool FUSED = decltype(fused)::value;
    RowSum sum = warp_sum<T, FUSED, lanes_for(NT / 32)>(
        lane < NT / 32 ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, a.c);
    bool whole = true;
    float M = kNegInf;  // of the list, then of the row
#pragma unroll
    for (int i = 0; i < E; ++i) M = fmaxf(M, e.z[i]);
    M = warp_max(M);
    if (np > 1) {
      // The weight (negative: a token twice) and the list's maximum go along so that the
      // message leaves after they were read: once it is there, the row's first CTA may set
      // the count behind the weight back, and others write gradients over the list's logits.
      const float4 mine = make_float4(__shfl_sync(kAllLanes, sum.m, 0),
                                      __shfl_sync(kAllLanes, sum.s, 0), twice ? -w : w, M);
      if (lane < np) send_float4(&parts[round][part], mine, &sent[round], lane);
      if (!mbar_wait(&sent[round], 0, kRowWaitNs)) {
        if (lane == 0) flag(ctrl, DEVERR_TIMEOUT, t);
        whole = mbar_wait(&sent[round], 0, kRowWaitNs);  // none of them comes after the end
      }
      whole = __all_sync(kAllLanes, whole);
      const float4 x = lane < np ? parts[round][lane] : make_float4(kNegInf, 0.f, 0.f, 0.f);
      twice = __any_sync(kAllLanes, signbit(x.z));
      sum = warp_sum<T, FUSED, 8>(RowSum{x.x, x.y, 0.f}, a.c);
      sum = {__shfl_sync(kAllLanes, sum.m, 0), __shfl_sync(kAllLanes, sum.s, 0), 0.f};
    } else {
      sum = {__shfl_sync(kAllLanes, sum.m, 0), __shfl_sync(kAllLanes, sum.s, 0), 0.f};
    }
    if (FUSED) sum = exact_sums<T>(sum, a.c);
    if (FUSED && !sums_hold(sum.m, a.c)) {
      if (lane == 0) rest = Rest::kCareful;
      return;
    }
    M = fmaxf(M, sum.m);
    bool nan = sum.s != sum.s;
#pragma unroll
    for (int i = 0; i < E; ++i) nan |= e.z[i] != e.z[i];
    nan = __any_sync(kAllLanes, nan);
    const bool none = M == kNegInf && !nan;  // no token has a probability
    const uint32_t wrong = __ballot_sync(kAllLanes, strange >= 0);
    if (part == 0) {
      if (strange >= 0 && lane == __ffs(wrong) - 1)
        flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)strange);
      if (lane == 0 && twice) flag(ctrl, DEVERR_TWICE, t);
      if (lane == 0 && none) flag(ctrl, DEVERR_ROW, t);
    }
    const bool zero = none || wrong || twice || !whole;
    const Classes o = classes<E>(rule, e, lists.rest != nullptr, lpr, sum, M, a.c, a.inv_t);
    const float by = rule.grad_scale * w * a.inv_t;
#pragma unroll
    for (int i = 0; i < E; ++i) e.z[i] *= by;
    weighted = zero ? 0.f : w * o.loss;
    if (lane) return;
    if (part == 0 && row_loss) row_loss[t] = zero ? 0.f : o.loss;
    rest = zero ? Rest::kZero : Rest::kGrad;
    // without a finite logit outside of the list there is no maximum to be relative to, and
    // each 2^y is 0
    grad.m = sum.m == kNegInf ? 0.f : sum.m;
    grad.a = by * o.outside;
    grad.b = grad.at = 0.f;
  };
  RowSum sum = warp_sum<T, F>(part_sum<T, false, F, NT>(held, n, a.c), a.c);
  if (lane == 0) red[wid] = sum;
  if (np > 1) cluster_wait();  // every CTA has started, so that its shared memory is there
  __syncthreads();
  if (wid == 0) finish(std::integral_constant<bool, F>{}, 0);
  __syncthreads();
  if (F && rest == Rest::kCareful) {  // rare: again, the careful way
    sum = warp_sum<T, false>(part_sum<T, false, false, NT>(held, n, a.c), a.c);
    if (lane == 0) red[wid] = sum;
    __syncthreads();
    if (wid == 0) finish(std::false_type{}, 1);
    __syncthreads();
  }
  if (BACK) {
    if (rest == Rest::kZero) {
      part_zero<T, NT>(d, n);
    } else {
      part_grad_any<T, false, NT>(held, d, n, n, grad, a.c);
      __syncthreads();  // before the entries take their places
      if (wid == 0) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (e.id[i] >= 0 && (uint32_t)e.id[i] - first < n)
            d[(uint32_t)e.id[i] - first] = from_f32<T>(e.z[i]);
      }
    }
  }
  if (part == 0) conclude(weighted, per_row, loss, ctrl);
}

}  // namespace

cudaError_t launch_distill_loss(edp_ctx *ctx, const edp_distill_config &cfg, const TokenSet &set,
                                const Logits &z, const int32_t *ids, const float *value,
                                uint32_t top, const float *rest, float *loss, float *row_loss,
                                void *dz, uint64_t dstride, cudaStream_t s) {
  Plan p;
  const uint64_t means = set.reduce == EDP_REDUCE_SEQ_MEAN ? set.n_seq : 1;
  const bool few = set.n <= kFewRows && set.n <= kFewTokens * means;
  cudaError_t e = plan_weights(ctx, set, few, true, s, &p);
  if (e != cudaSuccess) return e;
  const bool counted = p.sequences || p.w.tokens;
  const RowWeights w{set, few && counted, p.w.sequence, p.w.tokens, p.w.fixed, p.divisor};
  const TeacherLists lists{ids, value, rest, top};
  DistillRule rule;
  rule.kind = cfg.kind;
  rule.beta = (float)cfg.beta;
  rule.alpha = (float)(1.0 - cfg.beta);
  rule.ln_beta = (float)std::log(cfg.beta);
  rule.ln_alpha = (float)std::log1p(-cfg.beta);
  rule.inv_tt = (float)(1.0 / cfg.teacher_temperature);
  rule.grad_scale = (float)cfg.grad_scale;
  e = by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    uint32_t parts = row_parts(ctx, z, 2);
    while (parts < 8 && part_bytes(z, parts) > kResidentPart) parts *= 2;
    // few rows: smaller parts, so that the last of them are a small share
    while (parts < 8 && z.rows * parts < 8ull * ctx->coop_sms && part_bytes(z, parts) > kLeastPart)
      parts *= 2;
    auto go = [&](auto kern) {
      const cudaError_t err = cudaFuncSetAttribute(
          kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kResidentMost);
      if (err != cudaSuccess) return err;
      return launch_rows(kern, z.rows, parts, true, kThreads, part_bytes(z, parts), s,
                         row_args(z), w, p.w.by_range, lists, rule, loss, row_loss, p.per_token,
                         dz, dstride, p.early, ctx->ctrl);
    };
    auto wide = [&](auto entries) {
      constexpr int E = decltype(entries)::value;
      return dz ? go(k_distill<T, true, E>) : go(k_distill<T, false, E>);
    };
    if (top <= 32) return wide(std::integral_constant<int, 1>{});
    if (top <= 64) return wide(std::integral_constant<int, 2>{});
    return wide(std::integral_constant<int, 4>{});
  });
  if (e != cudaSuccess) forget_count(ctx, p, s);
  return e;
}

}  // namespace edp
