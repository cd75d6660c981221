// edp_rows.cuh -- what the kernels over rows of logits share: vectors as pairs of fp32
// numbers, a row's maximum and sums of exponentials over lanes, warps, CTAs and
// clusters, the gradient of a part of a row, parts in shared memory, and launches.
#pragma once

#include <cooperative_groups.h>

#include <type_traits>

#include "edp_loss.cuh"

namespace edp {

namespace cg = cooperative_groups;

constexpr int kRowThreads = 512;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kUnroll = 4;  // 16-byte loads in flight per thread

constexpr float kNoLog = -1e4f;  // stands for logarithms whose power of 2 is 0 in fp32

// The difference z - m and its product with c cost an instruction more than one
// fused z c - (m c), whose rounding of m c is the same for all of a row and is
// taken out at its end.  What is taken out grows with m c: a 16-bit row with |m c|
// beyond kFusedMost (a largest logit of 181,704 at temperature 1, of 182 at 0.001)
// goes the careful way, as fp32 rows do.  Up to there the rounding is at most 2^-7.
constexpr float kFusedMost = 262144.f;
template <typename T>
constexpr bool kFused = sizeof(T) == 2;

// Two fp32 numbers in a 64-bit register: both in one instruction, each rounded as
// on its own.
struct F2 {
  unsigned long long v;
  __device__ __forceinline__ F2() {}
  __device__ __forceinline__ F2(float x, float y) {
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
  }
  __device__ __forceinline__ explicit F2(float x) : F2(x, x) {}
  __device__ __forceinline__ float x() const {
    float a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
    return a;
  }
  __device__ __forceinline__ float y() const {
    float a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
    return b;
  }
};
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 ex2_both(F2 a) { return F2(ex2(a.x()), ex2(a.y())); }

// A 16-byte vector as pairs of fp32 numbers.
template <typename T>
struct Vec16 {
  static constexpr int kN = 16 / sizeof(T), kPairs = kN / 2;
  __device__ static __forceinline__ F2 pair(const uint4 &w, int i) {
    const T *x = reinterpret_cast<const T *>(&w);
    return F2(to_f32(x[2 * i]), to_f32(x[2 * i + 1]));
  }
  __device__ static __forceinline__ void set(uint4 &w, int i, F2 v) {
    T *x = reinterpret_cast<T *>(&w);
    x[2 * i] = from_f32<T>(v.x());
    x[2 * i + 1] = from_f32<T>(v.y());
  }
  // NaN apart
  __device__ static __forceinline__ float max(const uint4 &w) {
    float m = to_f32(reinterpret_cast<const T *>(&w)[0]);
#pragma unroll
    for (int i = 1; i < kN; ++i) m = fmaxf(m, to_f32(reinterpret_cast<const T *>(&w)[i]));
    return m;
  }
};
template <typename T2>
__device__ __forceinline__ float max_of_pairs(const uint4 &w) {
  const T2 *x = reinterpret_cast<const T2 *>(&w);
  const T2 m = __hmax2(__hmax2(x[0], x[1]), __hmax2(x[2], x[3]));
  return fmaxf(to_f32(m.x), to_f32(m.y));
}
template <>
__device__ __forceinline__ float Vec16<__nv_bfloat16>::max(const uint4 &w) {
  return max_of_pairs<__nv_bfloat162>(w);
}
template <>
__device__ __forceinline__ float Vec16<__half>::max(const uint4 &w) {
  return max_of_pairs<__half2>(w);
}
template <>
__device__ __forceinline__ F2 Vec16<__nv_bfloat16>::pair(const uint4 &w, int i) {
  const uint32_t x = (&w.x)[i];
  return F2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
template <>
__device__ __forceinline__ void Vec16<__nv_bfloat16>::set(uint4 &w, int i, F2 v) {
  (&w.x)[i] = pack_bf16x2(v.x(), v.y());
}
template <>
__device__ __forceinline__ void Vec16<__half>::set(uint4 &w, int i, F2 v) {
  const __half2 h = __floats2half2_rn(v.x(), v.y());
  (&w.x)[i] = *reinterpret_cast<const uint32_t *>(&h);
}

// Logarithms of a row relative to its maximum m.
template <typename T, bool FUSED>
struct RowLog {
  float c, less;  // y = z c - less, or (z - less) c
  __device__ __forceinline__ RowLog(float m, float c_) : c(c_) {
    // a part with low numbers or -infinity alone is taken relative to the lowest maximum
    // that the fused form has, so that its sums stay finite (they go over as they are to
    // a row whose maximum is there or higher; another row goes the careful way)
    if (FUSED) less = fmaxf(m * c, -kFusedMost);
    else less = m == kNegInf ? 0.f : m;
  }
  __device__ __forceinline__ float of(float z) const {
    return FUSED ? fmaf(z, c, -less) : (z - less) * c;
  }
  __device__ __forceinline__ F2 of(F2 z) const {
    return FUSED ? fma2(z, F2(c), F2(-less)) : (z + F2(-less)) * F2(c);
  }
  // what takes logarithms relative to `from` to these
  __device__ __forceinline__ float shift(const RowLog &from) const {
    return FUSED ? from.less - less : (from.less - less) * c;
  }
};

// -infinity has no product with its 0, nor has a logarithm that overflows once it is
// scaled: a number whose power of 2 is 0 all the same stands for them, in bfloat16
// before the logarithm (two at a time), else after.  kLowLogit is so low that at any
// temperature 2^(z c) is 0 beside every maximum of the fused form, and so high that an
// entropy gradient's product with it is finite up to a dentropy of 8e26 T^2.
constexpr float kLowLogit = -4e11f;
template <typename T, bool FUSED>
__device__ __forceinline__ uint4 finite_words(uint4 w) {
  if constexpr (FUSED && std::is_same<T, __nv_bfloat16>::value) {
    const __nv_bfloat162 low = __float2bfloat162_rn(kLowLogit);
    __nv_bfloat162 *x = reinterpret_cast<__nv_bfloat162 *>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __hmax2_nan(x[i], low);
  }
  return w;
}
template <typename T, bool FUSED>
__device__ __forceinline__ F2 finite_log(F2 y) {
  if constexpr (FUSED && std::is_same<T, __nv_bfloat16>::value) return y;
  return F2(fmaxf(y.x(), kNoLog), fmaxf(y.y(), kNoLog));
}

// Running maximum and sums of a part of a row: S and U relative to the maximum.
struct RowSum {
  float m, s, u;
};

// A thread's sums, of even and odd places apart.
struct LaneSum {
  float m;
  F2 s, u;
};
template <typename T, bool ENT, bool FUSED>
__device__ __forceinline__ RowLog<T, FUSED> raise(LaneSum &a, float m, float c) {
  if (m > a.m) {
    if (a.m != kNegInf) {
      const float d = RowLog<T, FUSED>(m, c).shift(RowLog<T, FUSED>(a.m, c)), f = ex2(d);
      if (ENT) a.u = f > 0.f ? F2(f) * fma2(F2(d), a.s, a.u) : F2(0.f);
      a.s = F2(f) * a.s;
    }
    a.m = m;
  }
  return RowLog<T, FUSED>(a.m, c);
}
// The sums of a vector's numbers relative to `log`.
template <typename T, bool ENT, bool FUSED>
__device__ __forceinline__ void add_vector(F2 &s, F2 &u, const uint4 &w,
                                           const RowLog<T, FUSED> &log) {
  const uint4 x = ENT ? finite_words<T, FUSED>(w) : w;
#pragma unroll
  for (int i = 0; i < Vec16<T>::kPairs; ++i) {
    const F2 y = log.of(Vec16<T>::pair(x, i)), e = ex2_both(y);
    s = s + e;
    if (ENT) u = fma2(e, finite_log<T, FUSED>(y), u);
  }
}
// K vectors of one thread.
template <typename T, bool ENT, bool FUSED, int K>
__device__ __forceinline__ void take_vectors(LaneSum &a, const uint4 (&w)[K], float c) {
  float m = Vec16<T>::max(w[0]);
#pragma unroll
  for (int k = 1; k < K; ++k) m = fmaxf(m, Vec16<T>::max(w[k]));
  const RowLog<T, FUSED> log = raise<T, ENT, FUSED>(a, m, c);
#pragma unroll
  for (int k = 0; k < K; ++k) add_vector<T, ENT, FUSED>(a.s, a.u, w[k], log);
}

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

template <typename T, bool ENT, bool FUSED, int NT = kRowThreads>
__device__ __forceinline__ RowSum part_sum(const T *p, uint32_t n, float c) {
  constexpr int N = Vec16<T>::kN;
  LaneSum a{kNegInf, F2(0.f), F2(0.f)};
  const Span<T> sp(p, n);
  if (threadIdx.x < sp.head + sp.tail) {
    const float v = to_f32(p[threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * N]);
    const float y = raise<T, ENT, FUSED>(a, v, c).of(v), e = ex2(y);
    a.s = a.s + F2(e, 0.f);
    if (ENT) a.u = fma2(F2(e, 0.f), F2(fmaxf(y, kNoLog), 0.f), a.u);
  }
  const uint4 *q = reinterpret_cast<const uint4 *>(p + sp.head);
  uint32_t i = threadIdx.x;
  for (; i + (kUnroll - 1) * NT < sp.vecs; i += kUnroll * NT) {
    uint4 w[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) w[k] = q[i + k * NT];
    take_vectors<T, ENT, FUSED>(a, w, c);
  }
  for (; i < sp.vecs; i += NT) {
    const uint4 w[1] = {q[i]};
    take_vectors<T, ENT, FUSED>(a, w, c);
  }
  return {a.m, a.s.x() + a.s.y(), a.u.x() + a.u.y()};
}

// The sum alone, relative to a number that is known.
template <typename T, bool FUSED, int NT>
__device__ __forceinline__ float part_sum_near(const T *p, uint32_t n,
                                               const RowLog<T, FUSED> &log) {
  const Span<T> sp(p, n);
  F2 s(0.f), u;
  if (threadIdx.x < sp.head + sp.tail) {
    const uint32_t i =
        threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * Vec16<T>::kN;
    s = F2(ex2(log.of(to_f32(p[i]))), 0.f);
  }
  const uint4 *q = reinterpret_cast<const uint4 *>(p + sp.head);
#pragma unroll 4
  for (uint32_t i = threadIdx.x; i < sp.vecs; i += NT)
    add_vector<T, false, FUSED>(s, u, q[i], log);
  return s.x() + s.y();
}

// The two halves of a barrier of the cluster (all of whose CTAs are resident, so
// that each arrives without waiting for another).
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
// The first, which only tells that the CTA has started.
__device__ __forceinline__ void cluster_started() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The sums of a warp's lanes, in all of them: first their maximum, to which each
// lane's sums go over, then plain sums in a fixed order (LANES: the lanes that hold
// any, the first of the warp; a power of two).
template <typename T, bool FUSED, int LANES = 32>
__device__ __forceinline__ RowSum warp_sum(RowSum a, float c) {
  static_assert((LANES & (LANES - 1)) == 0, "halved in each step");
  float m = a.m;
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAllLanes, m, o));
  if (a.m != kNegInf) {
    const float d = RowLog<T, FUSED>(m, c).shift(RowLog<T, FUSED>(a.m, c));
    const float f = a.m == m ? 1.f : ex2(d);
    // 2^(y + d) (y + d): a part whose factor underflowed has no product either
    a.u = a.m == m ? a.u : f > 0.f ? f * fmaf(d, a.s, a.u) : 0.f;
    a.s *= f;
  }  // else the sums are 0 (or NaN, which stays)
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    a.s += __shfl_xor_sync(kAllLanes, a.s, o);
    a.u += __shfl_xor_sync(kAllLanes, a.u, o);
  }
  return {m, a.s, a.u};
}

// The lanes that as many warps' sums take.
constexpr int lanes_for(int warps) { return warps <= 8 ? 8 : warps <= 16 ? 16 : 32; }

// The CTA's sums, in its first warp.
template <typename T, bool FUSED, int NT = kRowThreads>
__device__ __forceinline__ RowSum cta_join(RowSum a, float c, RowSum *red) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  a = warp_sum<T, FUSED>(a, c);
  if (lane == 0) red[wid] = a;
  __syncthreads();
  if (wid == 0)
    a = warp_sum<T, FUSED, lanes_for(NT / 32)>(
        lane < NT / 32 ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, c);
  return a;
}

// The sums of a row's parts, in every thread: each CTA's first warp gives its own to
// all of the cluster and adds up what it was given.  Every CTA has started.
template <typename T, bool FUSED>
__device__ __forceinline__ RowSum cluster_join(RowSum a, float c, uint32_t part, uint32_t np,
                                               RowSum *parts, RowSum *whole) {
  if (np > 1) {
    if (threadIdx.x < 32) {
      // lane 0's, by each of the lanes to one CTA
      const RowSum mine{__shfl_sync(kAllLanes, a.m, 0), __shfl_sync(kAllLanes, a.s, 0),
                        __shfl_sync(kAllLanes, a.u, 0)};
      if (threadIdx.x < np) cg::this_cluster().map_shared_rank(parts, threadIdx.x)[part] = mine;
    }
    cluster_arrive();
    cluster_wait();
    if (threadIdx.x < 32)
      a = warp_sum<T, FUSED, 8>(threadIdx.x < np ? parts[threadIdx.x] : RowSum{kNegInf, 0.f, 0.f},
                                c);
  }
  if (threadIdx.x == 0) *whole = a;
  __syncthreads();
  return *whole;
}

// The part of a row that CTA `part` of `parts` takes, as whole vectors' worth.
__device__ __forceinline__ uint32_t part_size(uint32_t vocab, uint32_t parts) {
  return (((vocab + parts - 1) / parts) + 7u) & ~7u;
}
__device__ __forceinline__ uint32_t owner_of(uint32_t vocab, uint32_t column, uint32_t parts) {
  return column / part_size(vocab, parts);
}
__device__ __forceinline__ void row_part(uint32_t vocab, uint32_t part, uint32_t parts,
                                         uint32_t *first, uint32_t *n) {
  const uint32_t each = part_size(vocab, parts);
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

// Whether the sums of a row with maximum m hold (see kFusedMost); without a maximum
// they are 0.
__device__ __forceinline__ bool sums_hold(float m, float c) {
  return m == kNegInf || fabsf(m * c) <= kFusedMost;
}
// 2^d - 1 to 2^-24 for |d| up to 2^-7: the first two terms of its series
__device__ __forceinline__ float exp2_less_1(float d) {
  const float x = d * kLn2;
  return fmaf(0.5f * x, x, x);
}
// The sums relative to m itself, not to the rounded m c.
template <typename T>
__device__ __forceinline__ RowSum exact_sums(RowSum a, float c) {
  if (!kFused<T> || a.m == kNegInf) return a;
  const float d = -fmaf(a.m, c, -(a.m * c));
  a.u = fmaf(d, a.s, a.u);
  const float f = exp2_less_1(d);
  return {a.m, fmaf(f, a.s, a.s), fmaf(f, a.u, a.u)};
}

struct RowOut {
  float logp, entropy, m, s;
};
// What the whole row's sums say (S = 0: no distribution).
__device__ __forceinline__ RowOut row_out(const RowSum &a, float zt, float inv_t) {
  if (a.m == kNegInf && !(a.s != a.s)) return {0.f, 0.f, 0.f, 0.f};
  const float ln = logf(a.s);
  return {(zt - a.m) * inv_t - ln, ln - kLn2 * (a.u / a.s), a.m, a.s};
}

struct RowArgs {
  const void *z;
  uint64_t stride;
  uint32_t vocab;
  const int32_t *target;
  const uint8_t *mask;
  float c, inv_t;  // log2(e) / T and 1 / T
};

// Gradient of a part of a row.  dz_j = (1/T) (g [j = t] - p_j (g + h (ln p_j + H)))
// = 2^y_j (A + B y_j) off the target, with p_j = 2^y_j / S, ln p_j = ln2 y_j - ln S.
struct RowGrad {
  float m, a, b;  // signed
  float at;       // added at the target
};
__device__ __forceinline__ RowGrad row_grad(float m, float s, float entropy, float g, float h,
                                            float inv_t) {
  RowGrad r;
  const float by = -inv_t / s;
  r.m = m;
  r.a = by * (g + h * (entropy - logf(s)));
  r.b = by * h * kLn2;
  r.at = inv_t * g;
  return r;
}
// y = RowLog's less d: what its rounding of m c left out, which 2^y / S and y take in.
template <typename T, bool FUSED>
__device__ __forceinline__ RowGrad exact_grad(RowGrad g, float c) {
  if (!FUSED) return g;
  const float d = -fmaf(g.m, c, -(g.m * c)), f = exp2_less_1(d);
  g.a = fmaf(d, g.b, g.a);
  g.a = fmaf(f, g.a, g.a);
  g.b = fmaf(f, g.b, g.b);
  return g;
}

template <typename T, bool ENT, bool FUSED>
struct GradOf {
  RowLog<T, FUSED> log;
  F2 a, b;
  __device__ __forceinline__ GradOf(const RowGrad &g, float c) : log(g.m, c) {
    const RowGrad x = exact_grad<T, FUSED>(g, c);
    a = F2(x.a);
    b = F2(x.b);
  }
  __device__ __forceinline__ F2 of(F2 z) const {
    const F2 y = log.of(z), e = ex2_both(y);
    return e * (ENT ? fma2(b, finite_log<T, FUSED>(y), a) : a);
  }
  __device__ __forceinline__ float of(float z) const {
    if constexpr (ENT && FUSED && std::is_same<T, __nv_bfloat16>::value)
      z = z < kLowLogit ? kLowLogit : z;
    return of(F2(z, 0.f)).x();
  }
  __device__ __forceinline__ uint4 of(const uint4 &w) const {
    const uint4 x = ENT ? finite_words<T, FUSED>(w) : w;
    uint4 o;
#pragma unroll
    for (int i = 0; i < Vec16<T>::kPairs; ++i) Vec16<T>::set(o, i, of(Vec16<T>::pair(x, i)));
    return o;
  }
};

template <typename T, bool ENT, bool FUSED, int NT>
__device__ __forceinline__ void part_grad(const T *p, T *d, uint32_t n, uint32_t at,
                                          const RowGrad &grad, float c) {
  constexpr int N = Vec16<T>::kN;
  const GradOf<T, ENT, FUSED> g(grad, c);
  // each thread reads what it writes (in place), the target among it
  auto one = [&](uint32_t i) {
    const float v = g.of(to_f32(p[i]));
    d[i] = from_f32<T>(i == at ? v + grad.at : v);
  };
  if ((((uintptr_t)p ^ (uintptr_t)d) & 15u) == 0) {
    const Span<T> sp(p, n);
    if (threadIdx.x < sp.head + sp.tail)
      one(threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * N);
    const uint4 *q = reinterpret_cast<const uint4 *>(p + sp.head);
    uint4 *o = reinterpret_cast<uint4 *>(d + sp.head);
    const uint32_t place = at - sp.head, hit = at >= sp.head ? place / N : 0xffffffffu;
    auto many = [&](const uint4 &w, uint32_t i) {
      uint4 x = g.of(w);
      if (i == hit) {
        const T *z = reinterpret_cast<const T *>(&w);
        T *y = reinterpret_cast<T *>(&x);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e == place % N) y[e] = from_f32<T>(g.of(to_f32(z[e])) + grad.at);
      }
      o[i] = x;
    };
    uint32_t i = threadIdx.x;
    for (; i + (kUnroll - 1) * NT < sp.vecs; i += kUnroll * NT) {
      uint4 w[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) w[k] = q[i + k * NT];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) many(w[k], i + k * NT);
    }
    for (; i < sp.vecs; i += NT) many(q[i], i);
  } else {
    for (uint32_t i = threadIdx.x; i < n; i += NT) one(i);
  }
}
// The way that the row's maximum asks for.  at: the target's place in the part, or
// beyond n.
template <typename T, bool ENT, int NT = kRowThreads>
__device__ __forceinline__ void part_grad_any(const T *p, T *d, uint32_t n, uint32_t at,
                                              const RowGrad &g, float c) {
  if (kFused<T> && sums_hold(g.m, c))
    part_grad<T, ENT, kFused<T>, NT>(p, d, n, at, g, c);
  else
    part_grad<T, ENT, false, NT>(p, d, n, at, g, c);
}

template <typename T, int NT = kRowThreads>
__device__ __forceinline__ void part_zero(T *d, uint32_t n) {
  constexpr int N = Vec16<T>::kN;
  const Span<T> sp(d, n);
  if (threadIdx.x < sp.head + sp.tail)
    d[threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * N] = from_f32<T>(0.f);
  uint4 *o = reinterpret_cast<uint4 *>(d + sp.head);
  for (uint32_t i = threadIdx.x; i < sp.vecs; i += NT) o[i] = make_uint4(0, 0, 0, 0);
}

// Parts of a row in shared memory (k_policy_resident has the measurements).
constexpr uint32_t kResidentPart = 80 * 1024;       // bytes of a part, where the row allows
constexpr uint32_t kResidentMost = 200 * 1024;
constexpr uint32_t kLeastPart = 32 * 1024;
constexpr uint64_t kRowWaitNs = 1000000000ull;      // bound of the wait for a part


// No preference for what leaves the second-level cache first: with the streaming
// policy 8,192 rows of 152,064 took 788 us, with this one 777.
__device__ __forceinline__ uint64_t policy_normal() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  return p;
}

// v to `to` in the shared memory of the cluster's CTA `rank`, counted on its `bar`.
__device__ __forceinline__ void send_float4(float4 *to, float4 v, unsigned long long *bar,
                                            uint32_t rank) {
  asm volatile(
      "{\n\t.reg .b32 d, b;\n\t"
      "mapa.shared::cluster.u32 d, %0, %2;\n\t"
      "mapa.shared::cluster.u32 b, %1, %2;\n\t"
      "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [d], {%3, %4, %5, %6}, "
      "[b];\n\t}"
      ::"r"(smem_addr(to)), "r"(smem_addr(bar)), "r"(rank), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
      : "memory");
}

inline RowArgs row_args(const Logits &z) {
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

// CTAs per row: up to 8 (a portable cluster), each with two vectors per thread, until
// there are per_sm for each SM.  Where they join their sums (per_sm 2) fewer and larger
// parts are faster (500 rows of 152,064: 25 us with 1 CTA each, 38 with 4); the
// gradient's need not wait for one another (16 per SM: 48 us, 53 with 2).
inline uint32_t row_parts(const edp_ctx *c, const Logits &z, uint64_t per_sm) {
  const uint64_t size = z.dtype == EDP_F32 ? 4 : 2;
  const uint64_t least = (uint64_t)kRowThreads * 32 / size;
  uint32_t p = 1;
  while (p < 8 && z.rows * p < per_sm * (uint64_t)c->coop_sms && z.vocab >= 2 * p * least) p *= 2;
  return p;
}

// Shared memory that a part of a row takes at any alignment.
inline size_t part_bytes(const Logits &z, uint32_t parts) {
  const uint64_t size = z.dtype == EDP_F32 ? 4 : 2;
  const uint64_t each = ((z.vocab + parts - 1) / parts + 7) & ~7ull;
  return (size_t)(((each * size + 15) & ~15ull) + 16);
}

template <typename... KArgs, typename... Args>
cudaError_t launch_rows(void (*kern)(KArgs...), uint64_t rows, uint32_t parts, bool cluster,
                        int threads, size_t smem, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)rows, parts);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
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

}  // namespace edp
