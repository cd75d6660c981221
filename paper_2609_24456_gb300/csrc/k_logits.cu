// k_logits.cu -- from logits to log-probabilities and back: the
// log-probability and entropy of each row's target, the gradient of the
// logits, and both in one pass with the policy loss between them.
//
// With z the row, T the temperature and m = max z, everything is in powers of
// two: y_j = (z_j - m) log2(e) / T, S = sum 2^y_j, U = sum 2^y_j y_j, so that
//   logp = (z_t - m) / T - ln S,  H = ln S - ln2 U / S,  p_j = 2^y_j / S.
// One pass keeps (m, S, U) per thread; a larger maximum rescales S and U.
#include <cooperative_groups.h>

#include "edp_loss.cuh"

namespace cg = cooperative_groups;

namespace edp {
namespace {

constexpr int kRowThreads = 512;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kUnroll = 4;  // 16-byte loads in flight per thread

constexpr float kNoLog = -1e4f;  // stands for logarithms whose power of 2 is 0 in fp32

// Running maximum and sums of a part of a row.
struct RowSum {
  float m, s, u;
};

__device__ __forceinline__ RowSum row_join(RowSum a, RowSum b, float c) {
  const float m = fmaxf(a.m, b.m);
  if (m == kNegInf) return {m, a.s + b.s, a.u + b.u};  // NaN among them stays
  const float da = a.m == kNegInf ? 0.f : (a.m - m) * c;
  const float db = b.m == kNegInf ? 0.f : (b.m - m) * c;
  const float fa = ex2(da), fb = ex2(db);
  // 2^(y + d) (y + d): a part whose factor underflowed has no product either
  const float ua = fa > 0.f ? fa * fmaf(da, a.s, a.u) : 0.f;
  const float ub = fb > 0.f ? fb * fmaf(db, b.s, b.u) : 0.f;
  return {m, fmaf(fa, a.s, fb * b.s), ua + ub};
}

// N elements of one thread.
template <bool ENT, int N>
__device__ __forceinline__ void row_take(RowSum &a, const float (&v)[N], float c) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
  if (m > a.m) {
    if (a.m != kNegInf) {
      const float d = (a.m - m) * c, f = ex2(d);
      if (ENT) a.u = f > 0.f ? f * fmaf(d, a.s, a.u) : 0.f;
      a.s *= f;
    }
    a.m = m;
  }
  const float mm = a.m == kNegInf ? 0.f : a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = (v[i] - mm) * c;
    const float e = ex2(y);
    a.s += e;
    // -infinity has no product
    if (ENT) a.u = fmaf(e, fmaxf(y, kNoLog), a.u);
  }
}

template <typename T>
struct Vec16 {
  static constexpr int kN = 16 / sizeof(T);
  __device__ static __forceinline__ void unpack(const uint4 &w, float (&v)[kN]) {
    const T *x = reinterpret_cast<const T *>(&w);
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = to_f32(x[i]);
  }
  __device__ static __forceinline__ uint4 pack(const float (&v)[kN]) {
    uint4 w;
    T *x = reinterpret_cast<T *>(&w);
#pragma unroll
    for (int i = 0; i < kN; ++i) x[i] = from_f32<T>(v[i]);
    return w;
  }
};

// Elements [0, n) at p as those before the first 16-byte boundary, vectors, rest.
template <typename T>
struct Span {
  uint32_t head, vecs, tail;
  __device__ __forceinline__ Span(const T *p, uint32_t n) {
    head = min(n, (uint32_t)((16u - ((uint32_t)(uintptr_t)p & 15u)) & 15u) / (uint32_t)sizeof(T));
    vecs = (n - head) / Vec16<T>::kN;
    tail = n - head - vecs * Vec16<T>::kN;
  }
};

template <typename T, bool ENT>
__device__ __forceinline__ RowSum part_sum(const T *p, uint32_t n, float c) {
  constexpr int N = Vec16<T>::kN;
  RowSum a{kNegInf, 0.f, 0.f};
  const Span<T> sp(p, n);
  if (threadIdx.x < sp.head + sp.tail) {
    const uint32_t i = threadIdx.x < sp.head ? threadIdx.x
                                             : threadIdx.x + sp.vecs * N;
    const float v[1] = {to_f32(p[i])};
    row_take<ENT, 1>(a, v, c);
  }
  const uint4 *q = reinterpret_cast<const uint4 *>(p + sp.head);
  uint32_t i = threadIdx.x;
  for (; i + (kUnroll - 1) * kRowThreads < sp.vecs; i += kUnroll * kRowThreads) {
    uint4 w[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) w[k] = q[i + k * kRowThreads];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      float v[N];
      Vec16<T>::unpack(w[k], v);
      row_take<ENT, N>(a, v, c);
    }
  }
  for (; i < sp.vecs; i += kRowThreads) {
    float v[N];
    Vec16<T>::unpack(q[i], v);
    row_take<ENT, N>(a, v, c);
  }
  return a;
}

// The CTA's sum, in thread 0; joined by lanes and warps in a fixed order.
__device__ __forceinline__ RowSum cta_join(RowSum a, float c, RowSum *red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const RowSum b{__shfl_down_sync(kAllLanes, a.m, o), __shfl_down_sync(kAllLanes, a.s, o),
                   __shfl_down_sync(kAllLanes, a.u, o)};
    a = row_join(a, b, c);
  }
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  if (lane == 0) red[wid] = a;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < kRowWarps; ++w) a = row_join(a, red[w], c);
  return a;
}

// The part of a row that CTA `part` of `parts` takes, as whole vectors' worth.
__device__ __forceinline__ void row_part(uint32_t vocab, uint32_t part, uint32_t parts,
                                         uint32_t *first, uint32_t *n) {
  const uint32_t each = (((vocab + parts - 1) / parts) + 7u) & ~7u;
  const uint64_t lo = min((uint64_t)part * each, (uint64_t)vocab);
  *first = (uint32_t)lo;
  *n = (uint32_t)min((uint64_t)each, vocab - lo);
}

enum class Row { kSkip, kBad, kUse };
__device__ __forceinline__ Row row_kind(const int32_t *target, const uint8_t *mask, uint64_t t,
                                        uint32_t vocab) {
  if (mask && !mask[t]) return Row::kSkip;
  const int32_t x = target[t];
  return x < 0 ? Row::kSkip : (uint32_t)x >= vocab ? Row::kBad : Row::kUse;
}

struct RowOut {
  float logp, entropy, m, s;
};
// What the whole row's sum says (S = 0: no distribution).
__device__ __forceinline__ RowOut row_out(const RowSum &a, float zt, float inv_t) {
  if (a.m == kNegInf && !(a.s != a.s)) return {0.f, 0.f, 0.f, 0.f};
  const float ln = logf(a.s);
  return {(zt - a.m) * inv_t - ln, ln - kLn2 * (a.u / a.s), a.m, a.s};
}

// The two halves of a barrier of the cluster (all of whose CTAs are resident, so
// that each arrives without waiting for another).
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct RowArgs {
  const void *z;
  uint64_t stride;
  uint32_t vocab;
  const int32_t *target;
  const uint8_t *mask;
  float c, inv_t;  // log2(e) / T and 1 / T
};

// A cluster of gridDim.y CTAs per row (1, 2, 4 or 8), each a part of it.
template <typename T, bool ENT>
__global__ void __launch_bounds__(kRowThreads)
k_token_logprob(RowArgs a, float *logp, float *entropy, float *stats, Ctrl *ctrl) {
  __shared__ RowSum red[kRowWarps];
  __shared__ RowSum parts[8];
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
  if (np > 1) cluster_arrive();
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  RowSum sum = cta_join(part_sum<T, ENT>(row + first, n, a.c), a.c, red);
  if (np > 1) {
    cluster_wait();  // every CTA has started, so that its shared memory is there
    if (threadIdx.x == 0) cg::this_cluster().map_shared_rank(parts, 0)[part] = sum;
    cluster_arrive();
    cluster_wait();
    if (part) return;
    if (threadIdx.x == 0)
      for (uint32_t k = 1; k < np; ++k) sum = row_join(sum, parts[k], a.c);
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

// Gradient of a part of a row.  dz_j = (1/T) (g [j = t] - p_j (g + h (ln p_j + H)))
// = p_j (A + B y_j) off the target, with ln p_j = ln2 y_j - ln S.
struct RowGrad {
  float m, inv_s, ga, gb;  // A and B, signed
  float at;                // added at the target
};
__device__ __forceinline__ RowGrad row_grad(float m, float s, float entropy, float g, float h,
                                            float inv_t) {
  RowGrad r;
  r.m = m;
  r.inv_s = 1.f / s;
  r.ga = -inv_t * (g + h * (entropy - logf(s)));
  r.gb = -inv_t * h * kLn2;
  r.at = inv_t * g;
  return r;
}
template <bool ENT>
__device__ __forceinline__ float grad_of(float z, const RowGrad &g, float c) {
  const float y = (z - g.m) * c;
  const float p = ex2(y) * g.inv_s;
  return p * (ENT ? fmaf(g.gb, fmaxf(y, kNoLog), g.ga) : g.ga);
}

template <typename T, bool ENT>
__device__ __forceinline__ void part_grad(const T *p, T *d, uint32_t first, uint32_t n,
                                          uint32_t target, const RowGrad &g, float c) {
  constexpr int N = Vec16<T>::kN;
  p += first;
  d += first;
  const uint32_t at = target - first;  // beyond n: not in this part
  const float zt = at < n ? to_f32(p[at]) : 0.f;
  __syncthreads();  // the target is read before it is overwritten (in place)
  if ((((uintptr_t)p ^ (uintptr_t)d) & 15u) == 0) {
    const Span<T> sp(p, n);
    if (threadIdx.x < sp.head + sp.tail) {
      const uint32_t i = threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * N;
      d[i] = from_f32<T>(grad_of<ENT>(to_f32(p[i]), g, c));
    }
    const uint4 *q = reinterpret_cast<const uint4 *>(p + sp.head);
    uint4 *o = reinterpret_cast<uint4 *>(d + sp.head);
    uint32_t i = threadIdx.x;
    for (; i + (kUnroll - 1) * kRowThreads < sp.vecs; i += kUnroll * kRowThreads) {
      uint4 w[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) w[k] = q[i + k * kRowThreads];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        float v[N];
        Vec16<T>::unpack(w[k], v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = grad_of<ENT>(v[e], g, c);
        o[i + k * kRowThreads] = Vec16<T>::pack(v);
      }
    }
    for (; i < sp.vecs; i += kRowThreads) {
      float v[N];
      Vec16<T>::unpack(q[i], v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = grad_of<ENT>(v[e], g, c);
      o[i] = Vec16<T>::pack(v);
    }
  } else {
    for (uint32_t i = threadIdx.x; i < n; i += kRowThreads)
      d[i] = from_f32<T>(grad_of<ENT>(to_f32(p[i]), g, c));
  }
  if (at < n) {
    __syncthreads();
    if (threadIdx.x == 0) d[at] = from_f32<T>(grad_of<ENT>(zt, g, c) + g.at);
  }
}

template <typename T>
__device__ __forceinline__ void part_zero(T *d, uint32_t n) {
  constexpr int N = Vec16<T>::kN;
  const Span<T> sp(d, n);
  if (threadIdx.x < sp.head + sp.tail)
    d[threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * N] = from_f32<T>(0.f);
  uint4 *o = reinterpret_cast<uint4 *>(d + sp.head);
  for (uint32_t i = threadIdx.x; i < sp.vecs; i += kRowThreads) o[i] = make_uint4(0, 0, 0, 0);
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
  part_grad<T, ENT>(reinterpret_cast<const T *>(a.z) + t * a.stride, d, first, n,
                    (uint32_t)a.target[t], g, a.c);
}

// What row t weighs in the policy loss, found by a warp; 0 outside the sequences.
__device__ __forceinline__ float row_weight(const RowWeights &w, uint64_t t) {
  if (w.off && (t < w.off[0] || t >= w.off[w.n_seq])) return 0.f;
  if (w.sequence) return __ldcg(&w.sequence[sequence_of_warp(w.off, 0, w.n_seq, t)]);
  return w.tokens ? 1.f / (float)__ldcg(w.tokens) : w.fixed;
}

// The policy loss's derivative by a row's log-probability, before weight and scale.
__device__ __forceinline__ float row_policy(const PolicyRule &rule, float logp, float old,
                                            const float *ref, float adv) {
  const float d = logp - old;
  if (!ref) return policy_token<Kl::kNone, false>(rule, d, 0.f, adv).dlogp;
  const float q = *ref - logp;
  return rule.kl == EDP_KL_K3 ? policy_token<Kl::kK3, false>(rule, d, q, adv).dlogp
                              : policy_token<Kl::kOther, false>(rule, d, q, adv).dlogp;
}

// Log-probability, policy gradient and the logits' gradient of a row, by a
// cluster of gridDim.y CTAs.
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
  const float w = kind == Row::kUse ? row_weight(weights, t) : 0.f;
  if (w == 0.f) {
    if (part == 0 && threadIdx.x == 0) {
      logp[t] = 0.f;
      if (entropy) entropy[t] = 0.f;
      if (kind == Row::kBad)
        flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)a.target[t]);
    }
    part_zero(d + first, n);
    return;  // the whole cluster
  }
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
  const uint32_t target = (uint32_t)a.target[t];
  const float zt = to_f32(row[target]);
  if (np > 1) cluster_arrive();
  RowSum sum = cta_join(part_sum<T, ENT>(row + first, n, a.c), a.c, red);
  if (np > 1) {
    cluster_wait();  // every CTA has started, so that its shared memory is there
    if (threadIdx.x == 0)
      for (uint32_t k = 0; k < np; ++k)
        cg::this_cluster().map_shared_rank(parts, k)[part] = sum;
    cluster_arrive();  // also: every CTA has read the target before one overwrites it
    cluster_wait();
    if (threadIdx.x == 0) {
      sum = parts[0];
      for (uint32_t k = 1; k < np; ++k) sum = row_join(sum, parts[k], a.c);
    }
  }
  if (threadIdx.x == 0) whole = sum;
  __syncthreads();
  const RowOut o = row_out(whole, zt, a.inv_t);
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
                             by * row_policy(rule, o.logp, old_logp[t],
                                             ref_logp ? ref_logp + t : nullptr, adv[t]),
                             ENT ? -by * rule.entropy_coef : 0.f, a.inv_t);
  part_grad<T, ENT>(row, d, first, n, target, g, a.c);
}

RowArgs row_args(const Logits &z) {
  RowArgs a;
  a.z = z.z;
  a.stride = z.stride;
  a.vocab = z.vocab;
  a.target = z.target;
  a.mask = z.mask;
  a.c = (float)(kLog2e / z.temperature);
  a.inv_t = (float)(1.0 / z.temperature);
  return a;
}

// CTAs per row: one for at least two waves of rows, else so many (up to 8, a
// portable cluster) that the chip has work, each with two vectors per thread.
uint32_t row_parts(const edp_ctx *c, const Logits &z) {
  const uint64_t size = z.dtype == EDP_F32 ? 4 : 2;
  const uint64_t least = (uint64_t)kRowThreads * 32 / size;
  uint32_t p = 1;
  while (p < 8 && z.rows * p < 2ull * c->coop_sms && z.vocab >= 2 * p * least) p *= 2;
  return p;
}

template <typename... KArgs, typename... Args>
cudaError_t launch_rows(void (*kern)(KArgs...), uint64_t rows, uint32_t parts, bool cluster,
                        cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)rows, parts);
  cfg.blockDim = dim3(kRowThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = parts;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster && parts > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

// f(T{}) for the logits' type.
template <typename F>
cudaError_t by_type(uint32_t dtype, F f) {
  switch (dtype) {
    case EDP_BF16: return f(__nv_bfloat16{});
    case EDP_F16: return f(__half{});
    default: return f(float{});
  }
}

}  // namespace

cudaError_t launch_token_logprob(edp_ctx *ctx, const Logits &z, float *logp, float *entropy,
                                 float *stats, cudaStream_t s) {
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    auto kern = entropy ? k_token_logprob<T, true> : k_token_logprob<T, false>;
    return launch_rows(kern, z.rows, row_parts(ctx, z), true, s, row_args(z), logp, entropy, stats,
                       ctx->ctrl);
  });
}

cudaError_t launch_token_logprob_grad(edp_ctx *ctx, const Logits &z, const float *stats,
                                      const float *entropy, const float *dlogp,
                                      const float *dentropy, void *dz, uint64_t dstride,
                                      cudaStream_t s) {
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    auto kern = entropy ? k_token_logprob_grad<T, true> : k_token_logprob_grad<T, false>;
    return launch_rows(kern, z.rows, row_parts(ctx, z), false, s, row_args(z), stats, entropy,
                       dlogp, dentropy, dz, dstride, ctx->ctrl);
  });
}

cudaError_t launch_policy_rows(edp_ctx *ctx, const Logits &z, const PolicyRule &rule,
                               const RowWeights &w, const PolicyTokens &p, float *logp,
                               float *entropy, void *dz, uint64_t dstride, cudaStream_t s) {
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    auto kern = entropy ? k_policy_rows<T, true> : k_policy_rows<T, false>;
    return launch_rows(kern, z.rows, row_parts(ctx, z), true, s, row_args(z), w, p.old_logp,
                       p.ref_logp, p.adv, rule, logp, entropy, dz, dstride, ctx->ctrl);
  });
}

}  // namespace edp
