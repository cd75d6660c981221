// edp_stream.cuh -- rows of logits that are read once and not kept: the ring of asynchronous
// copies that a CTA's threads stream a part of a row through, sums relative to a number that
// is known before, and the shape of such launches.
#pragma once

#include "edp_rows.cuh"

namespace edp {

constexpr int kStreamLanes = 1024;  // threads per SM, which bounds the registers
constexpr uint32_t kMostParts = 8;
// Sums below lose bits of numbers whose power of 2 leaves fp32.  Of those above, eight parts'
// sums may add up to infinity, and what is divided by them leaves fp32 below.
constexpr float kLeastSum = 0x1p-64f;
constexpr float kMostSum = 0x1p64f;

// A vector of logits at -infinity.
template <typename T>
__device__ __forceinline__ uint4 no_logits() {
  const uint32_t x = std::is_same<T, float>::value           ? 0xff800000u
                     : std::is_same<T, __nv_bfloat16>::value ? 0xff80ff80u
                                                             : 0xfc00fc00u;
  return make_uint4(x, x, x, x);
}
__device__ __forceinline__ RowSum row_sum(const LaneSum &a) {
  return {a.m, a.s.x() + a.s.y(), a.u.x() + a.u.y()};
}

// 16 bytes to shared memory, beside the thread; groups of such copies, and waiting for all
// but the last N groups.
__device__ __forceinline__ void async_load(uint4 *to, const uint4 *from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(to)), "l"(from)
               : "memory");
}
__device__ __forceinline__ void async_mark() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A part of a row as its CTA's threads pass over it: the vectors in segments of a warp's 32,
// kUnroll segments per warp and round, and the numbers before and behind the vectors by the
// first threads.  Round g takes segments g, g + rounds, g + 2 rounds, ..., so that the
// first round's are spread evenly over the part.
// S: rounds in shared memory or on their way there.
template <typename T, int NT, int S>
struct Part {
  const T *p;
  uint32_t first;  // its first column
  Span<T> sp;
  uint32_t rounds;
  // this thread's first vector; from one of its segments of a round to the next; the rounds
  // that have all of them
  const uint4 *mine;
  uint32_t apart, whole;
  __device__ __forceinline__ Part(const T *p_, uint32_t first_, uint32_t n)
      : p(p_), first(first_), sp(p_, n) {
    rounds = max(1u, (sp.vecs + 32 * (NT / 32) * kUnroll - 1) / (32 * (NT / 32) * kUnroll));
    apart = 32 * (NT / 32) * rounds;
    const uint32_t at = vec_at(0, 0, threadIdx.x & 31), last = at + (kUnroll - 1) * apart;
    mine = reinterpret_cast<const uint4 *>(p + sp.head) + at;
    whole = last < sp.vecs ? min(rounds, (sp.vecs - last + 31) / 32) : 0;
  }
  __device__ __forceinline__ uint32_t vec_at(uint32_t g, uint32_t k, uint32_t lane) const {
    return ((k * (NT / 32) + (threadIdx.x >> 5)) * rounds + g) * 32 + lane;
  }
  __device__ __forceinline__ uint32_t column(uint32_t vec) const {
    return first + sp.head + vec * Vec16<T>::kN;
  }
  __device__ __forceinline__ uint4 vec(uint32_t i) const {
    return reinterpret_cast<const uint4 *>(p + sp.head)[i];
  }
  // Round g of this thread's vectors to its own places, -infinity where there are none.
  __device__ __forceinline__ void fetch(uint4 *ring, uint32_t g) const {
    uint4 *to = ring + g % S * (kUnroll * NT) + threadIdx.x;
    const uint4 *from = mine + 32 * g;
    if (g < whole) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) async_load(to + k * NT, from + k * apart);
    } else if (g < rounds) {
#pragma unroll 1
      for (int k = 0; k < kUnroll; ++k) {
        if (vec_at(g, k, threadIdx.x & 31) < sp.vecs) async_load(to + k * NT, from + k * apart);
        else to[k * NT] = no_logits<T>();
      }
    }
    async_mark();
  }
  __device__ __forceinline__ void start(uint4 *ring) const {
#pragma unroll
    for (int g = 0; g < S; ++g) fetch(ring, g);
  }
  __device__ __forceinline__ void load(uint4 (&w)[kUnroll], const uint4 *ring, uint32_t g) const {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
      w[k] = ring[(g % S * kUnroll + k) * NT + threadIdx.x];
  }
  // A lane's vector of round g, from the ring while it is there (after a __syncwarp).
  __device__ __forceinline__ uint4 vec_of(const uint4 *ring, uint32_t g, uint32_t k,
                                          uint32_t lane) const {
    if (g + S >= rounds)
      return ring[(g % S * kUnroll + k) * NT + (threadIdx.x & ~31u) + lane];
    return vec(vec_at(g, k, lane));
  }
  __device__ __forceinline__ bool single() const { return threadIdx.x < sp.head + sp.tail; }
  __device__ __forceinline__ uint32_t single_at() const {
    return threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * Vec16<T>::kN;
  }
  // f(vector, index) of this thread's vectors, streamed as the passes are (with -infinity
  // beyond them), for the rare passes: small code.
  template <typename F>
  __device__ __forceinline__ void each_vector(uint4 *ring, F f) const {
    start(ring);
#pragma unroll 1
    for (uint32_t g = 0; g < rounds; ++g) {
      async_wait<S - 1>();
#pragma unroll 1
      for (uint32_t k = 0; k < kUnroll; ++k) {
        const uint4 w = ring[(g % S * kUnroll + k) * NT + threadIdx.x];
        f(w, vec_at(g, k, threadIdx.x & 31));
      }
      fetch(ring, g + S);
    }
  }
  // f(number, column) of all of this thread's numbers.
  template <typename F>
  __device__ __forceinline__ void each(uint4 *ring, F f) const {
    if (single()) f(to_f32(p[single_at()]), first + single_at());
    each_vector(ring, [&](const uint4 &w, uint32_t i) {
#pragma unroll
      for (int e = 0; e < Vec16<T>::kN; ++e)
        f(to_f32(reinterpret_cast<const T *>(&w)[e]), column(i) + e);
    });
  }
};

__device__ __forceinline__ float warp_add(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kAllLanes, x, o);
  return x;
}

// Numbers that are alike round the same way: n of them, added one after another, lose up to
// n 2^-25 of their sum.  So a lane adds up 512 in each of its two sums (2^-16 at the worst) in the
// rounds between two carries, where its warp takes them over in pairs.  Parts with more rounds
// (LONG) have kernels of their own: with the carry in all of them 8,192 lists of 152,064
// columns took 406 us, without 384.  (8,388,001 fp16 numbers of one CTA: the logarithm of their
// sum was off by 6.6e-5 without the carry.)
template <typename T>
constexpr uint32_t kAloneRounds = 512 / (kUnroll * Vec16<T>::kPairs);
struct Carried {
  Pair s, u;
};
// take(g) of all rounds, which adds to s and u.  c: the warp's own.
template <typename T, bool LONG, bool ENT, typename F>
__device__ __forceinline__ void each_round(uint32_t rounds, Carried *c, F2 &s, F2 &u, F take) {
  if constexpr (!LONG) {
    for (uint32_t g = 0; g < rounds; ++g) take(g);
  } else {
    if ((threadIdx.x & 31) == 0) *c = Carried{};
    for (uint32_t g = 0; g < rounds;) {
      const uint32_t stop = min(rounds, g + kAloneRounds<T>);
      for (; g < stop; ++g) take(g);
      const float a = warp_add(s.x() + s.y()), b = ENT ? warp_add(u.x() + u.y()) : 0.f;
      if ((threadIdx.x & 31) == 0) {
        pair_add(c->s, a);
        if (ENT) pair_add(c->u, b);
      }
      s = u = F2(0.f);
    }
  }
}
// A thread's sums relative to ref; what its warp carried is its first lane's.
template <bool LONG>
__device__ __forceinline__ RowSum sums_of(const Carried *c, float ref, F2 s, F2 u) {
  if constexpr (!LONG) return {ref, s.x() + s.y(), u.x() + u.y()};
  if (threadIdx.x & 31) return {ref, 0.f, 0.f};
  return {ref, as_df(c->s).hi, as_df(c->u).hi};
}
// Two sums beside each other with their rounding errors, for the passes that are rare.
struct F2Pair {
  F2 hi = F2(0.f), lo = F2(0.f);
  __device__ __forceinline__ void add(F2 x) {
    const F2 less(-1.f), s = hi + x, b = fma2(hi, less, s);
    lo = lo + (fma2(fma2(b, less, s), less, hi) + fma2(b, less, x));
    hi = s;
  }
  // of both; the errors of infinities are NaN
  __device__ __forceinline__ float sum() const {
    const float s = hi.x() + hi.y();
    return isfinite(s) ? s + (lo.x() + lo.y()) : s;
  }
};
// A lane's sums relative to a number that it raises only where another is 32 powers of 2 above:
// a sum that is scaled then is 2^-32 of what comes, and its roundings are nothing.
struct FarSum {
  float m = kNegInf;
  F2Pair s, u;
  template <typename T, bool ENT>
  __device__ __forceinline__ RowLog<T, false> raise(float to, float c) {
    if (to > m + 32.f / c) {
      if (m != kNegInf) {
        const float d = (m - to) * c, f = ex2(d);
        if (ENT) {
          u.hi = f > 0.f ? F2(f) * fma2(F2(d), s.hi, u.hi) : F2(0.f);
          u.lo = f > 0.f ? F2(f) * fma2(F2(d), s.lo, u.lo) : F2(0.f);
        }
        s.hi = F2(f) * s.hi;
        s.lo = F2(f) * s.lo;
      }
      m = to;
    }
    return RowLog<T, false>(m, c);
  }
  __device__ __forceinline__ RowSum sum() const { return {m, s.sum(), u.sum()}; }
};

// A number's share of the sums relative to `log`.
template <typename T, bool ENT, bool FUSED>
__device__ __forceinline__ void add_one(F2 &s, F2 &u, const RowLog<T, FUSED> &log, float v) {
  const float y = log.of(v), e = ex2(y);
  s = s + F2(e, 0.f);
  if (ENT) u = fma2(F2(e, 0.f), F2(fmaxf(y, kNoLog), 0.f), u);
}

// The threads' sums and those that lanes 0 .. n - 1 of each warp have in `more`, in all.
template <typename T, int NT>
__device__ __forceinline__ RowSum joined(const RowSum &mine, const RowSum &more, uint32_t n,
                                         RowSum *left, float c) {
  static_assert(NT / 32 + kMostParts <= 32, "a lane each");
  const uint32_t lane = threadIdx.x & 31;
  const RowSum a = warp_sum<T, false>(mine, c);
  if (lane == 0) left[threadIdx.x >> 5] = a;
  const uint32_t from = lane - (NT / 32);
  RowSum b{__shfl_sync(kAllLanes, more.m, from), __shfl_sync(kAllLanes, more.s, from),
           __shfl_sync(kAllLanes, more.u, from)};
  __syncthreads();
  if (lane < (NT / 32)) b = left[lane];
  else if (from >= n) b = {kNegInf, 0.f, 0.f};
  b = warp_sum<T, false, 32>(b, c);
  return {__shfl_sync(kAllLanes, b.m, 0), __shfl_sync(kAllLanes, b.s, 0),
          __shfl_sync(kAllLanes, b.u, 0)};
}

// CTAs per row while there is one per SM at the most and their parts are not small, and
// threads by the size of a part.  Measured with the lists of likely tokens on bfloat16 rows
// (us, parts x threads): 1 row of 152,064: 13.8 as 1 x 256, 9.4 as 8 x 256, 9.9 as 8 x 512; of
// 32,003: 7.7 as 1 x 256, 8.1 as 8 x 256; 64 rows of 152,064: 19.5 as 1 x 256, 15.1 as 2 x
// 256, 13.1 as 2 x 512, 16.1 as 4 x 512; 128: 20.0 as 1 x 256, 15.6 as 1 x 512; 2,000 rows of
// 4,000: 28.3 as 1 x 256, 16.1 as 1 x 128; 5,400 of 16,000: 109 and 86; 4,000 of 32,003: 94 and
// 75; 2,000 of 100,000: 97 and 86, but of 152,064 116 and 126, and 700 of 61,882 30 and 41; 2,048
// of 152,064: 117 as 1 x 256, 147 as 1 x 512.  Of a part that is all sampled 128 threads give no
// bound for more entries than they are (2,000 rows of 4,000 with 128 entries: 92 us, 43 with 256).
// Four rounds in flight where CTAs are two per SM at the most: 256 rows of 32,003 fp16 logits
// 11.5 us in a stream however the calls come, with two 11.1 to 14.6.
struct StreamShape {
  uint32_t parts, threads, stages;
  uint64_t vecs;  // of a part
};
inline StreamShape stream_shape(const edp_ctx *ctx, const Logits &z, uint32_t entries) {
  const uint64_t sms = (uint64_t)ctx->coop_sms;
  const uint64_t vecs = (uint64_t)z.vocab * (z.dtype == EDP_F32 ? 4 : 2) / 16;
  uint32_t parts = 1;
  while (parts < kMostParts && 2 * parts * z.rows <= sms && vecs >= 2ull * parts * 2048) parts *= 2;
  const uint64_t each = vecs / parts;
  const bool small = each <= 1024 ? entries <= 96 : each <= 12800 && z.rows * parts >= 8 * sms;
  if (small) return {parts, 128, 2, each};
  if (each >= 8192 && z.rows * parts <= sms) return {parts, 512, 2, each};
  return {parts, 256, z.rows * parts <= 2 * sms ? 4u : 2u, each};
}
// f of constants: threads, stages, and whether lanes have so many numbers that warps carry
// their sums (no parts of 128 threads are so large).
template <typename T, typename F>
cudaError_t by_shape(const StreamShape &s, F f) {
  using Two = std::integral_constant<int, 2>;
  using Four = std::integral_constant<int, 4>;
  if (s.threads == 128) return f(std::integral_constant<int, 128>{}, Two{}, std::false_type{});
  auto by_threads = [&](auto is_long) {
    if (s.threads == 512) return f(std::integral_constant<int, 512>{}, Two{}, is_long);
    return s.stages == 4 ? f(std::integral_constant<int, 256>{}, Four{}, is_long)
                         : f(std::integral_constant<int, 256>{}, Two{}, is_long);
  };
  return s.vecs > (uint64_t)kAloneRounds<T> * kUnroll * s.threads ? by_threads(std::true_type{})
                                                                  : by_threads(std::false_type{});
}

}  // namespace edp
