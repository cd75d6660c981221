// k_top.cu -- the likeliest tokens of rows of logits with their log-probabilities, the
// log-probability of a given token, the entropy, and the logarithm of what is outside of
// the list.
//
// One pass over memory: a cluster of CTAs holds the row in shared memory and passes over
// it twice there.  First each thread's largest logit: a warp's r-th largest of those, and
// the least of the warps' ones, is a bound that at least the K largest logits of the part
// reach, and of tens of thousands hardly more than two or three times as many.  They are
// collected, ranked by counting (value, then index: all different, so that the order does
// not depend on the threads'), and the K first leave the row for the list.  Then the sums
// of exponentials of the others, from which `rest` comes without cancellation.  The row's
// first CTA merges the parts' lists.
#include <cmath>

#include "edp_rows.cuh"

namespace edp {
namespace {

constexpr int kThreads = 384;
constexpr int kWarps = kThreads / 32;
constexpr uint32_t kMostParts = 8;

using Key = unsigned long long;  // order of the logit, then 2^32 - 1 - column; 0: none

// fp32 numbers in the order of whole numbers (NaN apart; -0 comes as 0)
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
constexpr uint32_t kLeastOrder = 0x00800000u;  // the lowest finite number's
__device__ __forceinline__ Key key_of(float z, uint32_t column) {
  return (Key)order_of(z + 0.f) << 32 | (0xffffffffu - column);
}
__device__ __forceinline__ float value_of(Key k) { return of_order((uint32_t)(k >> 32)); }
__device__ __forceinline__ uint32_t column_of(Key k) { return 0xffffffffu - (uint32_t)k; }

__device__ __forceinline__ void send_key(Key *to, Key v, unsigned long long *bar, uint32_t rank) {
  asm volatile(
      "{\n\t.reg .b32 d, b;\n\t"
      "mapa.shared::cluster.u32 d, %0, %2;\n\t"
      "mapa.shared::cluster.u32 b, %1, %2;\n\t"
      "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b64 [d], %3, [b];\n\t}"
      ::"r"(smem_addr(to)), "r"(smem_addr(bar)), "r"(rank), "l"(v)
      : "memory");
}

// A part of a row in shared memory, by one CTA's threads: vectors i, i + threads, ... and
// the first of them one number each of those before and behind the vectors.
template <typename T>
struct Held {
  const T *at;
  Span<T> sp;
  __device__ __forceinline__ bool single() const { return threadIdx.x < sp.head + sp.tail; }
  __device__ __forceinline__ uint32_t single_at() const {
    return threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * Vec16<T>::kN;
  }
  __device__ __forceinline__ const uint4 *vecs() const {
    return reinterpret_cast<const uint4 *>(at + sp.head);
  }
  // f(number, place) of this thread's numbers that are `least` or more
  template <typename F>
  __device__ __forceinline__ void each(float least, F f) const {
    if (single()) {
      const float v = to_f32(at[single_at()]);
      if (v >= least) f(v, single_at());
    }
    for (uint32_t i = threadIdx.x; i < sp.vecs; i += kThreads) {
      const uint4 w = vecs()[i];
      if (!(Vec16<T>::max(w) >= least)) continue;
#pragma unroll
      for (int k = 0; k < Vec16<T>::kN; ++k) {
        const float v = to_f32(reinterpret_cast<const T *>(&w)[k]);
        if (v >= least) f(v, sp.head + i * Vec16<T>::kN + k);
      }
    }
  }
  __device__ __forceinline__ float largest() const {
    float m = single() ? to_f32(at[single_at()]) : kNegInf;
    uint32_t i = threadIdx.x;
    for (; i + 3 * kThreads < sp.vecs; i += 4 * kThreads) {
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = Vec16<T>::max(vecs()[i + k * kThreads]);
      m = fmaxf(m, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
    }
    for (; i < sp.vecs; i += kThreads) m = fmaxf(m, Vec16<T>::max(vecs()[i]));
    return m;
  }
};

// The count over the CTA's threads, in all of them.  red: kWarps numbers, free before.
__device__ __forceinline__ uint32_t cta_count(uint32_t n, uint32_t *red) {
  n = __reduce_add_sync(kAllLanes, n);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = n;
  __syncthreads();
  const uint32_t lane = threadIdx.x & 31;
  n = __reduce_add_sync(kAllLanes, lane < kWarps ? red[lane] : 0u);
  __syncthreads();
  return n;
}

// The candidates of a part more of whose numbers reach the bound `lo` than the list has
// room for: halving between lo and the largest until a bound leaves K to `cap` of them, or
// until the K-th largest number is known; of those equal to it the first in the row come
// in, up to a column found by halving again.  Rare (numbers that are equal by the
// hundred, as masked ones are), so it only has to end: 64 passes at the most.
template <typename T>
__device__ __forceinline__ void collect_slowly(const Held<T> &h, uint32_t n, uint32_t first,
                                               uint32_t lo, uint32_t K, uint32_t cap, Key *list,
                                               uint32_t *count, uint32_t *red) {
  auto reach = [&](uint32_t bound) {
    uint32_t c = 0;
    h.each(of_order(bound), [&](float, uint32_t) { ++c; });
    return cta_count(c, red);
  };
  uint32_t hi = 0xff800001u, some = cap + 1;  // nothing is above +infinity
  while (hi - lo > 1 && some > cap) {
    const uint32_t mid = lo + (hi - lo) / 2, c = reach(mid);
    if (c >= K) {
      lo = mid;
      some = c;
    } else {
      hi = mid;
    }
  }
  uint32_t end = n;  // numbers equal to lo count before this place
  if (some > cap) {
    const uint32_t above = reach(hi);
    uint32_t a = 0;  // fewer than K - above of them before a, as many before end
    while (end - a > 1) {
      const uint32_t mid = a + (end - a) / 2;
      uint32_t c = 0;
      h.each(of_order(lo), [&](float v, uint32_t i) { c += order_of(v + 0.f) == lo && i < mid; });
      if (cta_count(c, red) + above >= K) end = mid;
      else a = mid;
    }
  }
  if (threadIdx.x == 0) *count = 0;
  __syncthreads();
  h.each(of_order(lo), [&](float v, uint32_t i) {
    if (i < end || order_of(v + 0.f) > lo) {
      const uint32_t at = atomicAdd(count, 1u);
      if (at < cap) list[at] = key_of(v, first + i);
    }
  });
  __syncthreads();
}

struct TopOut {
  int32_t *ids;
  float *top_logp, *logp, *entropy, *rest, *stats;
  uint32_t top, cap;  // cap: room for candidates
};

__device__ __forceinline__ void write_none(const TopOut &o, uint64_t t) {
  for (uint32_t k = threadIdx.x; k < o.top; k += kThreads) {
    o.ids[t * o.top + k] = -1;
    o.top_logp[t * o.top + k] = kNegInf;
  }
  if (threadIdx.x) return;
  if (o.logp) o.logp[t] = 0.f;
  if (o.entropy) o.entropy[t] = 0.f;
  if (o.rest) o.rest[t] = 0.f;
  if (o.stats) o.stats[2 * t] = o.stats[2 * t + 1] = 0.f;
}

// A cluster of gridDim.y CTAs per row, each with its part in shared memory.
template <typename T, bool ENT>
__global__ void __launch_bounds__(kThreads)
k_token_top(RowArgs a, TopOut o, Ctrl *ctrl) {
  constexpr bool F = kFused<T>;
  extern __shared__ uint4 shared_words[];
  __shared__ RowSum red[kWarps];
  __shared__ uint32_t bound[kWarps];
  __shared__ float4 sums[kMostParts];  // what the cluster's CTAs send: m, S, U
  __shared__ uint32_t count;
  __shared__ bool careful;
  __shared__ unsigned long long bar, sent;
  const uint64_t t = blockIdx.x;
  const uint32_t part = blockIdx.y, np = gridDim.y, K = o.top;
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  Key *list = reinterpret_cast<Key *>(shared_words);  // [cap], of even length
  Key *inbox = list + o.cap;                          // [np][K]; the lists of the parts
  uint4 *room = shared_words + (o.cap + np * K + 1) / 2;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 1);
    mbar_init(&sent, 1);
    if (np > 1 && part == 0) mbar_arrive_tx(&sent, np * (K * sizeof(Key) + sizeof(float4)));
    mbar_init_fence();
    count = 0;
  }
  __syncthreads();
  pdl_wait();
  pdl_launch();
  const int32_t target = a.target ? a.target[t] : 0;
  const bool skip = (a.mask && !a.mask[t]) || target < 0;
  if (skip || (uint32_t)target >= a.vocab) {
    if (part == 0) {
      write_none(o, t);
      if (!skip && threadIdx.x == 0)
        flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)target);
    }
    return;  // the whole cluster
  }
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride, *p = row + first;
  // the part keeps its place within 16 bytes
  T *held = reinterpret_cast<T *>(room) + ((uintptr_t)p & 15u) / sizeof(T);
  const Held<T> h{held, Span<T>(p, n)};
  if (threadIdx.x == 0 && h.sp.vecs) {
    mbar_arrive_tx(&bar, h.sp.vecs * 16);
    bulk_load(held + h.sp.head, p + h.sp.head, h.sp.vecs * 16, &bar, policy_normal());
  }
  if (h.single()) held[h.single_at()] = p[h.single_at()];
  if (np > 1) cluster_started();
  const float zt = a.target && part == 0 ? to_f32(row[target]) : 0.f;
  if (h.sp.vecs && !mbar_wait(&bar, 0, kRowWaitNs)) {
    if (threadIdx.x == 0) flag(ctrl, DEVERR_TIMEOUT, t);
    mbar_wait(&bar, 0, kRowWaitNs);  // bounded: the copy lands before the CTA ends
  }
  // A bound that at least K numbers reach: from warps all of whose lanes have a vector.
  const uint32_t full = min((uint32_t)kWarps, h.sp.vecs / 32);
  const uint32_t need = full ? (K + full - 1) / full : 33;
  const float mine = h.largest();
  if (need <= 32) {
    uint32_t left = order_of(mine + 0.f), best = 0;
    for (uint32_t k = 0; k < need; ++k) {
      best = __reduce_max_sync(kAllLanes, left);
      if (lane == __ffs(__ballot_sync(kAllLanes, left == best)) - 1) left = 0;
    }
    if (lane == 0) bound[wid] = best;
  }
  if (np > 1) cluster_wait();  // every CTA has started, so that its shared memory is there
  __syncthreads();
  uint32_t lo = kLeastOrder;
  if (need <= 32)
    lo = max(lo, __reduce_min_sync(kAllLanes, lane < full ? bound[lane] : 0xffffffffu));
  const float least = of_order(lo);
  if (mine >= least)
    h.each(least, [&](float v, uint32_t i) {
      const uint32_t at = atomicAdd(&count, 1u);
      if (at < o.cap) list[at] = key_of(v, first + i);
    });
  __syncthreads();
  if (count > o.cap) collect_slowly<T>(h, n, first, lo, K, o.cap, list, &count, bound);
  const uint32_t found = count;
  // Ranked by counting; the first K leave the row.
  for (uint32_t i = threadIdx.x; i < max(found, K); i += kThreads) {
    if (i >= found) {
      if (i < K) {
        if (np > 1) send_key(inbox + part * K + i, 0, &sent, 0);
        else inbox[i] = 0;
      }
      continue;
    }
    const Key key = list[i];
    uint32_t r = 0;
    for (uint32_t j = 0; j + 2 <= found; j += 2) {
      const ulonglong2 two = *reinterpret_cast<const ulonglong2 *>(list + j);
      r += (two.x > key) + (two.y > key);
    }
    if (found & 1) r += list[found - 1] > key;
    if (r < K) {
      if (np > 1) send_key(inbox + part * K + r, key, &sent, 0);
      else inbox[r] = key;
      held[column_of(key) - first] = from_f32<T>(kNegInf);
    }
  }
  __syncthreads();
  RowSum sum = warp_sum<T, F>(part_sum<T, ENT, F, kThreads>(held, n, a.c), a.c);
  if (lane == 0) red[wid] = sum;
  __syncthreads();
  if (wid == 0) {
    sum = exact_sums<T>(warp_sum<T, F, lanes_for(kWarps)>(lane < kWarps ? red[lane] : RowSum{kNegInf, 0.f, 0.f},
                                           a.c), a.c);
    if (lane == 0) careful = F && !sums_hold(sum.m, a.c);
  }
  __syncthreads();
  if (careful) {  // rare: again, the careful way
    sum = warp_sum<T, false>(part_sum<T, ENT, false, kThreads>(held, n, a.c), a.c);
    if (lane == 0) red[wid] = sum;
    __syncthreads();
    if (wid == 0)
      sum = warp_sum<T, false, lanes_for(kWarps)>(lane < kWarps ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, a.c);
  }
  if (np > 1) {
    if (threadIdx.x == 0)
      send_float4(&sums[part], make_float4(sum.m, sum.s, sum.u, 0.f), &sent, 0);
    if (part) return;
    bool whole = mbar_wait(&sent, 0, kRowWaitNs);
    if (!whole) {
      if (lane == 0) flag(ctrl, DEVERR_TIMEOUT, t);
      whole = mbar_wait(&sent, 0, kRowWaitNs);  // none of them comes after the end
    }
    if (!__syncthreads_and(whole)) {
      write_none(o, t);
      return;
    }
    // What of the parts' lists is not of the row's joins the others.
    LaneSum drop{kNegInf, F2(0.f), F2(0.f)};
    for (uint32_t i = threadIdx.x; i < np * K; i += kThreads) {
      const Key key = inbox[i];
      const uint32_t own = i / K;
      uint32_t r = i - own * K;
      if (!key) {
        continue;
      }
      for (uint32_t q = 0; q < np; ++q) {
        if (q == own) continue;
        uint32_t b = 0, e = K;  // list q: keys before b are larger, those from e on are not
        while (b < e) {
          const uint32_t mid = (b + e) / 2;
          if (inbox[q * K + mid] > key) b = mid + 1;
          else e = mid;
        }
        r += b;
      }
      if (r < K) {
        list[r] = key;
      } else {
        const float z = value_of(key), y = raise<T, ENT, false>(drop, z, a.c).of(z), e = ex2(y);
        drop.s = drop.s + F2(e, 0.f);
        if (ENT) drop.u = fma2(F2(e, 0.f), F2(fmaxf(y, kNoLog), 0.f), drop.u);
      }
    }
    uint32_t have = 0;  // keys in all lists: the row's list may be shorter than K
    for (uint32_t i = threadIdx.x; i < np * K; i += kThreads) have += inbox[i] != 0;
    have = cta_count(have, bound);
    for (uint32_t i = have + threadIdx.x; i < K; i += kThreads) list[i] = 0;
    const RowSum dropped = cta_join<T, false, kThreads>(
        RowSum{drop.m, drop.s.x() + drop.s.y(), drop.u.x() + drop.u.y()}, a.c, red);
    if (wid) return;
    const float4 x = lane < np ? sums[lane] : make_float4(kNegInf, 0.f, 0.f, 0.f);
    const RowSum d0{__shfl_sync(kAllLanes, dropped.m, 0), __shfl_sync(kAllLanes, dropped.s, 0),
                    __shfl_sync(kAllLanes, dropped.u, 0)};
    sum = warp_sum<T, false, 16>(lane == kMostParts ? d0 : RowSum{x.x, x.y, x.z}, a.c);
  }
  if (wid) return;
  sum = {__shfl_sync(kAllLanes, sum.m, 0), __shfl_sync(kAllLanes, sum.s, 0),
         __shfl_sync(kAllLanes, sum.u, 0)};
  const Key *top = np > 1 ? list : inbox;
  const bool any = top[0] != 0;
  const float M = any ? value_of(top[0]) : kNegInf;
  float S = 0.f, U = 0.f;
  for (uint32_t k = lane; k < K; k += 32)
    if (top[k]) {
      const float y = (value_of(top[k]) - M) * a.c, e = ex2(y);
      S += e;
      U = fmaf(e, fmaxf(y, kNoLog), U);
    }
#pragma unroll
  for (int i = 16; i; i >>= 1) {
    S += __shfl_xor_sync(kAllLanes, S, i);
    U += __shfl_xor_sync(kAllLanes, U, i);
  }
  if (!any && !(sum.s != sum.s)) {  // no token has a probability
    if (lane == 0) flag(ctrl, DEVERR_ROW, t);
    for (uint32_t k = lane; k < K; k += 32) {
      o.ids[t * K + k] = -1;
      o.top_logp[t * K + k] = kNegInf;
    }
    if (lane) return;
    if (o.logp) o.logp[t] = 0.f;
    if (o.entropy) o.entropy[t] = 0.f;
    if (o.rest) o.rest[t] = 0.f;
    if (o.stats) o.stats[2 * t] = o.stats[2 * t + 1] = 0.f;
    return;
  }
  if (sum.m == kNegInf) {
    S += sum.s;  // 0 or NaN
  } else {
    const float d = (sum.m - M) * a.c, f = ex2(d);
    S = fmaf(f, sum.s, S);
    U += f > 0.f ? f * fmaf(d, sum.s, sum.u) : 0.f;
  }
  const float ln = logf(S);
  const bool nan = S != S;
  for (uint32_t k = lane; k < K; k += 32) {
    const Key key = top[k];
    o.ids[t * K + k] = key && !nan ? (int32_t)column_of(key) : -1;
    o.top_logp[t * K + k] = nan ? S : key ? (value_of(key) - M) * a.inv_t - ln : kNegInf;
  }
  if (lane) return;
  if (o.logp) o.logp[t] = (zt - M) * a.inv_t - ln;
  if (o.entropy) o.entropy[t] = ln - kLn2 * (U / S);
  if (o.rest)
    o.rest[t] = nan ? S : sum.s == 0.f ? kNegInf : (sum.m - M) * a.inv_t + logf(sum.s) - ln;
  if (o.stats) {
    o.stats[2 * t] = M;
    o.stats[2 * t + 1] = S;
  }
}

}  // namespace

cudaError_t launch_token_top(edp_ctx *ctx, const Logits &z, uint32_t top, int32_t *ids,
                             float *top_logp, float *logp, float *entropy, float *rest,
                             float *stats, cudaStream_t s) {
  const TopOut o{ids, top_logp, logp, entropy, rest, stats, top, top <= 64 ? 256u : 512u};
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    uint32_t parts = row_parts(ctx, z, 2);
    while (parts < kMostParts && part_bytes(z, parts) > kResidentPart) parts *= 2;
    auto kern = entropy ? k_token_top<T, true> : k_token_top<T, false>;
    const size_t lists = ((o.cap + parts * top + 1) / 2) * 16;
    const cudaError_t e = cudaFuncSetAttribute(
        kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kResidentMost + 16 * 1024));
    if (e != cudaSuccess) return e;
    return launch_rows(kern, z.rows, parts, true, kThreads, lists + part_bytes(z, parts), s,
                       row_args(z), o, ctx->ctrl);
  });
}

}  // namespace edp
