// k_logits.cu -- from logits to log-probabilities and back: the
// log-probability and entropy of each row's target, the gradient of the
// logits, and both in one pass with the policy loss between them.
//
// With z the row, T the temperature and m = max z, everything is in powers of
// two: y_j = (z_j - m) log2(e) / T, S = sum 2^y_j, U = sum 2^y_j y_j, so that
//   logp = (z_t - m) / T - ln S,  H = ln S - ln2 U / S,  p_j = 2^y_j / S.
// One pass keeps (m, S, U) per thread; a larger maximum rescales S and U.  Two
// elements at a time where the instructions allow (F2), since the pass is as much
// bound by issue as by memory: 11 instructions an element (two roundings for the
// logarithm, one element each) read 8,192 rows of 152,064 bfloat16 logits, a tenth of
// them masked, in 389 us, 7 of them in 324 us.
//
// What bounds each now, at 6.69 TB/s of measured copy:
//   log-probabilities, 8,192 x 152,064 bf16      324 us   335 us to read them: memory
//   gradient with entropy, 4,096 x 152,064 bf16  349 us   354 us to read and write: memory
//   gradient, 777 x 32,003 f16                    21 us   14.9 us: 1,554 CTAs, 2.6 waves, each
//                                                         of which loads once and then stores
//   both with the policy loss, 8,192 x 152,064   784 us   707 us to read and write once
//   one row of 152,064                           3.8 us   in a graph: launch, one round
//                                                         trip to memory, the cluster's join

#include "edp_rows.cuh"

namespace edp {
namespace {

// A cluster of gridDim.y CTAs per row (1, 2, 4 or 8), each a part of it.
template <typename T, bool ENT>
__global__ void __launch_bounds__(kRowThreads)
k_token_logprob(RowArgs a, float *logp, float *entropy, float *stats, Ctrl *ctrl) {
  __shared__ RowSum red[kRowWarps];
  __shared__ RowSum parts[8];
  __shared__ RowSum whole;
  pdl_wait();
  pdl_launch();
  const uint64_t t = blockIdx.x;
  const uint32_t part = blockIdx.y, np = gridDim.y;
  const Row kind = row_kind(a.target, a.mask, t, a.vocab);
  if (kind != Row::kUse) {
    if (part == 0 && threadIdx.x == 0) {
      logp[t] = 0.f;
      if (entropy) entropy[t] = 0.f;
      if (stats) stats[2 * t] = stats[2 * t + 1] = 0.f;
      if (kind == Row::kBad) flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)a.target[t]);
    }
    return;  // the whole cluster
  }
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
  if (np > 1) cluster_started();
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  constexpr bool F = kFused<T>;
  RowSum sum = cta_join<T, F>(part_sum<T, ENT, F>(row + first, n, a.c), a.c, red);
  if (np > 1) {
    cluster_wait();  // every CTA has started, so that its shared memory is there
    if (threadIdx.x == 0) cg::this_cluster().map_shared_rank(parts, 0)[part] = sum;
    cluster_arrive();
    cluster_wait();
    if (part) return;
    if (threadIdx.x < 32)
      sum = warp_sum<T, F, 8>(threadIdx.x < np ? parts[threadIdx.x] : RowSum{kNegInf, 0.f, 0.f},
                              a.c);
  }
  if (F) {
    if (threadIdx.x == 0) whole = exact_sums<T>(sum, a.c);
    __syncthreads();
    sum = whole;
    if (!sums_hold(sum.m, a.c))  // rare: one CTA, the careful way
      sum = cta_join<T, false>(part_sum<T, ENT, false>(row, a.vocab, a.c), a.c, red);
  }
  if (threadIdx.x == 0) {
    const RowOut o = row_out(sum, to_f32(row[a.target[t]]), a.inv_t);
    if (o.s == 0.f) flag(ctrl, DEVERR_ROW, t);
    logp[t] = o.logp;
    if (entropy) entropy[t] = o.entropy;
    if (stats) {
      stats[2 * t] = o.m;
      stats[2 * t + 1] = o.s;
    }
  }
}

template <typename T, bool ENT>
__global__ void __launch_bounds__(kRowThreads)
k_token_logprob_grad(RowArgs a, const float *stats, const float *entropy, const float *dlogp,
                     const float *dentropy, void *dz, uint64_t dstride, Ctrl *ctrl) {
  pdl_wait();
  pdl_launch();
  const uint64_t t = blockIdx.x;
  uint32_t first, n;
  row_part(a.vocab, blockIdx.y, gridDim.y, &first, &n);
  T *d = reinterpret_cast<T *>(dz) + t * dstride;
  const Row kind = row_kind(a.target, a.mask, t, a.vocab);
  const float s = kind == Row::kUse ? stats[2 * t + 1] : 0.f;
  if (s == 0.f) {
    if (kind == Row::kBad && blockIdx.y == 0 && threadIdx.x == 0)
      flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)a.target[t]);
    part_zero(d + first, n);
    return;
  }
  const RowGrad g = row_grad(stats[2 * t], s, ENT ? entropy[t] : 0.f, dlogp[t],
                             ENT ? dentropy[t] : 0.f, a.inv_t);
  part_grad_any<T, ENT>(reinterpret_cast<const T *>(a.z) + t * a.stride + first, d + first, n,
                        (uint32_t)a.target[t] - first, g, a.c);
}

// The policy loss's derivative by a row's log-probability, before weight and scale.
__device__ __forceinline__ float row_policy(const PolicyRule &rule, float logp, float old,
                                            bool has_ref, float ref, float adv) {
  const float d = logp - old;
  if (!has_ref) return policy_token<Kl::kNone, false>(rule, d, 0.f, adv).dlogp;
  const float q = ref - logp;
  return rule.kl == EDP_KL_K3 ? policy_token<Kl::kK3, false>(rule, d, q, adv).dlogp
                              : policy_token<Kl::kOther, false>(rule, d, q, adv).dlogp;
}

// Log-probability, policy gradient and the logits' gradient of a row, by a
// cluster of gridDim.y CTAs, with the logits read twice: for rows whose parts do
// not fit shared memory (k_policy_resident).
template <typename T, bool ENT>
__global__ void __launch_bounds__(kRowThreads)
k_policy_rows(RowArgs a, RowWeights weights, const float *old_logp, const float *ref_logp,
              const float *adv, PolicyRule rule, float *logp, float *entropy, void *dz,
              uint64_t dstride, Ctrl *ctrl) {
  __shared__ RowSum red[kRowWarps];
  __shared__ RowSum parts[8];
  __shared__ RowSum whole;
  pdl_wait();
  pdl_launch();
  const uint64_t t = blockIdx.x;
  const uint32_t part = blockIdx.y, np = gridDim.y;
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  T *d = reinterpret_cast<T *>(dz) + t * dstride;
  const Row kind = row_kind(a.target, a.mask, t, a.vocab);
  if (kind != Row::kUse || !in_sequences(weights, t)) {
    if (part == 0 && threadIdx.x == 0) {
      logp[t] = 0.f;
      if (entropy) entropy[t] = 0.f;
      if (kind == Row::kBad)
        flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)a.target[t]);
    }
    part_zero(d + first, n);
    return;  // the whole cluster
  }
  const float w = row_weight(weights, t);
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
  const uint32_t target = (uint32_t)a.target[t];
  const float zt = to_f32(row[target]);
  if (np > 1) cluster_started();
  constexpr bool F = kFused<T>;
  RowSum sum = cta_join<T, F>(part_sum<T, ENT, F>(row + first, n, a.c), a.c, red);
  if (np > 1) cluster_wait();  // every CTA has started, so that its shared memory is there
  // also: every CTA has read the target before one overwrites it
  sum = exact_sums<T>(cluster_join<T, F>(sum, a.c, part, np, parts, &whole), a.c);
  if (F && !sums_hold(sum.m, a.c)) {  // rare: every CTA the whole row, the careful way
    __syncthreads();
    sum = cta_join<T, false>(part_sum<T, ENT, false>(row, a.vocab, a.c), a.c, red);
    if (threadIdx.x == 0) whole = sum;
    __syncthreads();
    sum = whole;
    if (np > 1) {  // before one of them overwrites its part
      cluster_arrive();
      cluster_wait();
    }
  }
  const RowOut o = row_out(sum, zt, a.inv_t);
  if (part == 0 && threadIdx.x == 0) {
    if (o.s == 0.f) flag(ctrl, DEVERR_ROW, t);
    logp[t] = o.logp;
    if (entropy) entropy[t] = o.entropy;
  }
  if (o.s == 0.f) {
    part_zero(d + first, n);
    return;
  }
  const float by = rule.grad_scale * w;
  const RowGrad g = row_grad(o.m, o.s, ENT ? o.entropy : 0.f,
                             by * row_policy(rule, o.logp, old_logp[t], ref_logp != nullptr,
                                             ref_logp ? ref_logp[t] : 0.f, adv[t]),
                             ENT ? -by * rule.entropy_coef : 0.f, a.inv_t);
  part_grad_any<T, ENT>(row + first, d + first, n, target - first, g, a.c);
}

// The same with each CTA's part of the row in shared memory: read from memory once,
// its gradient written once.  The part comes by a bulk copy; the CTAs of other rows
// on the SM (two beside it) take turns with it at waiting, computing and storing.  8,192 rows
// of 152,064 bfloat16 logits: 784 us, 1,012 with the logits read twice.  Parts of 76 KB
// (4 CTAs) and 384 threads; 842 us with 38 KB and 256 threads, 806 with 76 KB and 256,
// 809 with 512, 875 with 101 KB and 512.  The CTAs' sums travel as messages, each
// counted on an mbarrier of its receiver (841 us; 914 with barriers of the cluster, whose
// release waits for all of a CTA's writes).
constexpr int kResidentThreads = 384;
// CTAs per SM, which bound the registers (56 and 40): as many as parts of 76 KB allow of
// the 16-bit forms, whose two ways spill at 40 (f16 without entropy, 4,096 rows of 152,064:
// 412 us, 379 at 54); fp32 has one way, and where its parts are small more CTAs (515 rows
// of 32,003: 37.0 us, 41.3 with 3).
template <typename T>
constexpr int kResidentCtas = kFused<T> ? 3 : 4;
enum class Rest { kGrad, kZero, kCareful };

template <typename T, bool ENT>
__global__ void __launch_bounds__(kResidentThreads, kResidentCtas<T>)
k_policy_resident(RowArgs a, RowWeights weights, const float *old_logp, const float *ref_logp,
                  const float *adv, PolicyRule rule, float *logp, float *entropy, void *dz,
                  uint64_t dstride, bool early, Ctrl *ctrl) {
  constexpr int NT = kResidentThreads;
  constexpr bool F = kFused<T>;
  extern __shared__ uint4 resident[];
  __shared__ RowSum red[NT / 32];
  __shared__ float4 parts[2][8];  // what the cluster's CTAs send: m, S, U, the target's logit
  __shared__ RowGrad grad;
  __shared__ Rest rest;
  __shared__ unsigned long long bar, sent[2];
  const uint64_t t = blockIdx.x;
  const uint32_t part = blockIdx.y, np = gridDim.y;
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
  const Row kind = row_kind(a.target, a.mask, t, a.vocab);
  if (kind != Row::kUse || !in_sequences(weights, t)) {
    if (part == 0 && threadIdx.x == 0) {
      logp[t] = 0.f;
      if (entropy) entropy[t] = 0.f;
      if (kind == Row::kBad)
        flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)a.target[t]);
    }
    part_zero<T, NT>(d, n);
    if (early) pdl_wait();  // so that what waits for this kernel finds the weights
    return;  // the whole cluster
  }
  const T *p = reinterpret_cast<const T *>(a.z) + t * a.stride + first;
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
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const uint32_t at = (uint32_t)a.target[t] - first;  // beyond n: not in this part
  float w = 0.f, old = 0.f, ref = 0.f, ad = 0.f;      // the first warp's, beside the copy
  if (early) pdl_wait();
  if (wid == 0) {
    w = row_weight(weights, t);
    old = old_logp[t];
    if (ref_logp) ref = ref_logp[t];
    ad = adv[t];
  }
  if (sp.vecs && !mbar_wait(&bar, 0, kRowWaitNs)) {
    if (threadIdx.x == 0) flag(ctrl, DEVERR_TIMEOUT, t);
    mbar_wait(&bar, 0, kRowWaitNs);  // bounded: the copy lands before the CTA ends
  }
  __syncthreads();
  // The first warp joins the CTA's sums, gives them to the cluster's other CTAs and
  // takes theirs, and makes of all what the part's gradient needs.
  auto finish = [&](auto fused, int round) {
    constexpr bool FUSED = decltype(fused)::value;
    RowSum sum = warp_sum<T, FUSED, NT / 32 <= 8 ? 8 : NT / 32 <= 16 ? 16 : 32>(
        lane < NT / 32 ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, a.c);
    float zt = at < n ? to_f32(held[at]) : 0.f;
    bool whole = true;
    if (np > 1) {
      const float4 mine = make_float4(__shfl_sync(kAllLanes, sum.m, 0),
                                      __shfl_sync(kAllLanes, sum.s, 0),
                                      __shfl_sync(kAllLanes, sum.u, 0), zt);
      if (lane < np) send_float4(&parts[round][part], mine, &sent[round], lane);
      if (!mbar_wait(&sent[round], 0, kRowWaitNs)) {
        if (lane == 0) flag(ctrl, DEVERR_TIMEOUT, t);
        whole = mbar_wait(&sent[round], 0, kRowWaitNs);  // none of them comes after the end
      }
      const float4 x = lane < np ? parts[round][lane] : make_float4(kNegInf, 0.f, 0.f, 0.f);
      zt = __shfl_sync(kAllLanes, x.w, owner_of(a.vocab, (uint32_t)a.target[t], np));
      sum = warp_sum<T, FUSED, 8>(RowSum{x.x, x.y, x.z}, a.c);
    }
    if (FUSED) sum = exact_sums<T>(sum, a.c);
    if (FUSED && !sums_hold(sum.m, a.c)) {
      if (lane == 0) rest = Rest::kCareful;
      return;
    }
    if (lane) return;
    const RowOut o = whole ? row_out(sum, zt, a.inv_t) : RowOut{0.f, 0.f, 0.f, 0.f};
    if (part == 0) {
      if (o.s == 0.f) flag(ctrl, DEVERR_ROW, t);
      logp[t] = o.logp;
      if (entropy) entropy[t] = o.entropy;
    }
    rest = o.s == 0.f ? Rest::kZero : Rest::kGrad;
    const float by = rule.grad_scale * w;
    grad = row_grad(o.m, o.s, ENT ? o.entropy : 0.f,
                    by * row_policy(rule, o.logp, old, ref_logp != nullptr, ref, ad),
                    ENT ? -by * rule.entropy_coef : 0.f, a.inv_t);
  };
  RowSum sum = warp_sum<T, F>(part_sum<T, ENT, F, NT>(held, n, a.c), a.c);
  if (lane == 0) red[wid] = sum;
  if (np > 1) cluster_wait();  // every CTA has started, so that its shared memory is there
  __syncthreads();
  if (wid == 0) finish(std::integral_constant<bool, F>{}, 0);
  __syncthreads();
  if (F && rest == Rest::kCareful) {  // rare: again, the careful way
    sum = warp_sum<T, false>(part_sum<T, ENT, false, NT>(held, n, a.c), a.c);
    if (lane == 0) red[wid] = sum;
    __syncthreads();
    if (wid == 0) finish(std::false_type{}, 1);
    __syncthreads();
  }
  if (rest == Rest::kZero) part_zero<T, NT>(d, n);
  else part_grad_any<T, ENT, NT>(held, d, n, at, grad, a.c);
}

}  // namespace

cudaError_t launch_token_logprob(edp_ctx *ctx, const Logits &z, float *logp, float *entropy,
                                 float *stats, cudaStream_t s) {
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    auto kern = entropy ? k_token_logprob<T, true> : k_token_logprob<T, false>;
    return launch_rows(kern, z.rows, row_parts(ctx, z, 2), true, kRowThreads, 0, s, row_args(z), logp,
                       entropy, stats, ctx->ctrl);
  });
}

cudaError_t launch_token_logprob_grad(edp_ctx *ctx, const Logits &z, const float *stats,
                                      const float *entropy, const float *dlogp,
                                      const float *dentropy, void *dz, uint64_t dstride,
                                      cudaStream_t s) {
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    auto kern = entropy ? k_token_logprob_grad<T, true> : k_token_logprob_grad<T, false>;
    return launch_rows(kern, z.rows, row_parts(ctx, z, 16), false, kRowThreads, 0, s, row_args(z),
                       stats, entropy, dlogp, dentropy, dz, dstride, ctx->ctrl);
  });
}

cudaError_t launch_policy_rows(edp_ctx *ctx, const Logits &z, const PolicyRule &rule,
                               const RowWeights &w, const PolicyTokens &p, float *logp,
                               float *entropy, void *dz, uint64_t dstride, bool early,
                               cudaStream_t s) {
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    uint32_t parts = row_parts(ctx, z, 2);
    while (parts < 8 && part_bytes(z, parts) > kResidentPart) parts *= 2;
    // few rows: smaller parts, so that the last of them are a small share
    while (parts < 8 && z.rows * parts < 8ull * ctx->coop_sms && part_bytes(z, parts) > kLeastPart)
      parts *= 2;
    const size_t bytes = part_bytes(z, parts);
    if (bytes > kResidentMost)
      return launch_rows(entropy ? k_policy_rows<T, true> : k_policy_rows<T, false>, z.rows, parts,
                         true, kRowThreads, 0, s, row_args(z), w, p.old_logp, p.ref_logp, p.adv,
                         rule, logp, entropy, dz, dstride, ctx->ctrl);
    auto kern = entropy ? k_policy_resident<T, true> : k_policy_resident<T, false>;
    const cudaError_t e = cudaFuncSetAttribute(
        kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kResidentMost);
    if (e != cudaSuccess) return e;
    return launch_rows(kern, z.rows, parts, true, kResidentThreads, bytes, s, row_args(z), w,
                       p.old_logp, p.ref_logp, p.adv, rule, logp, entropy, dz, dstride, early,
                       ctx->ctrl);
  });
}

}  // namespace edp
