// k_top.cu -- the likeliest tokens of rows of logits with their log-probabilities, the
// log-probability of a given token, the entropy, and the logarithm of what is outside of
// the list.
//
// One pass over memory.  A CTA of each row (or of each part of a row, joined by a cluster)
// looks at its first rounds of vectors for a bound that a little more than the K largest
// logits reach, most likely (first_bound).  Then it passes over all: numbers that reach the
// bound are collected as candidates, the others go into the sums of exponentials, so that
// `rest` comes without cancellation.  Fewer than K candidates (a row in some hundred) ask for
// another pass with a lower bound of the sample, more than there is room for with a higher one;
// where that leads nowhere (logits that are equal by the hundred) the bound is searched by
// counts.  The candidates are ordered by value, then index (all different, so that nothing
// depends on the order in which they came), and those behind the list join the sums.  A row's
// first CTA merges its parts' lists.
//
// What bounds it, at 6.79 TB/s of measured copy:
//   8,192 x 152,064 bf16, 64 entries, entropy, a tenth masked   390 us   331 us to read them;
//                                      issue: 11 instructions an element at 2.9 of 4 a cycle
//   777 x 32,003 f32, 128 entries   31 us    14.8 us; 608 CTAs at a time, 169 in a second wave;
//                                      1,216 rows (two waves) 48 us, 23.1 to read them
//   256 x 32,003 f16, 8 entries     11.5 us  2.4 us; a chain of loads, sample, pass and order
//   one row of 152,064, 20 entries  9.4 us   the same, and the join of 8 lists
//   5,400 x 8,394 bf16, 128 entries 83 us    14 us; the order of the sample and of the candidates,
//                                      during which a CTA loads nothing (16,000 columns: 82 us)
//   8,000 x 2,000 bf16, 20 entries  27 us    4.9 us (k_top_small); issue, 39 instructions an element
// Four CTAs of 256 threads an SM leave 64 registers a thread: 27 of the 42 forms of k_token_top
// spill 4 or 8 bytes.
#include <algorithm>
#include <cmath>

#include "edp_stream.cuh"

namespace edp {
namespace {

constexpr uint32_t kNoted = 8;    // vectors of a thread that wait to be looked at
constexpr uint32_t kRoom = 1056;  // for candidates: all numbers of a part of 4 warps' vectors

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

// Which numbers are candidates: those above `least`, and of those equal to it the ones in
// columns before `end`.
struct Bound {
  float least;
  uint32_t end;
  __device__ __forceinline__ bool holds(float v, uint32_t column) const {
    return v > least || (v == least && column < end);
  }
};
struct Candidates {
  Key *list;
  uint32_t *count;
  uint32_t room;
  // too many already: the pass will be made again, whatever else it finds
  __device__ __forceinline__ bool full() const {
    return *const_cast<const volatile uint32_t *>(count) > room;
  }
  __device__ __forceinline__ void add(float v, uint32_t column) const {
    const uint32_t at = atomicAdd(count, 1u);
    if (at < room) list[at] = key_of(v, column);
  }
};

// The sums of a vector's numbers but its candidates, which go to the list.
template <typename T, bool ENT, bool FUSED>
__device__ __forceinline__ void add_but(F2 &s, F2 &u, const RowLog<T, FUSED> &log, const uint4 &w,
                                        uint32_t column, const Bound &b, const Candidates &to) {
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < Vec16<T>::kPairs; ++i) {
    const F2 z = Vec16<T>::pair(w, i);
    const bool x = b.holds(z.x(), column + 2 * i), y = b.holds(z.y(), column + 2 * i + 1);
    bits |= (x ? 1u : 0u) << 2 * i | (y ? 2u : 0u) << 2 * i;
    const F2 l = log.of(F2(x ? kNegInf : z.x(), y ? kNegInf : z.y())), e = ex2_both(l);
    s = s + e;
    if (ENT) u = fma2(e, F2(fmaxf(l.x(), kNoLog), fmaxf(l.y(), kNoLog)), u);
  }
#pragma unroll 1
  for (; bits; bits &= bits - 1) {
    const uint32_t e = __ffs(bits) - 1, word = e * sizeof(T) / 4;
    const uint32_t x = word < 2 ? word ? w.y : w.x : word == 2 ? w.z : w.w;
    const uint32_t half = sizeof(T) == 2 ? x >> (e & 1) * 16 : x;
    to.add(to_f32(*reinterpret_cast<const T *>(&half)), column + e);
  }
}

// Calls f(note, lane) for each of the notes of a warp's lanes, n of each, in a lane per
// note; they are in the lanes' columns of `notes`.
template <typename F>
__device__ __forceinline__ void each_note(const uint32_t *notes, uint32_t n, F f) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t upto = n;  // of this lane and those before
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const uint32_t x = __shfl_up_sync(kAllLanes, upto, o);
    if (lane >= o) upto += x;
  }
  const uint32_t all = __shfl_sync(kAllLanes, upto, 31);
  __syncwarp();
#pragma unroll 1
  for (uint32_t i = lane; i < ((all + 31) & ~31u); i += 32) {
    uint32_t owner = 0, before = 0;  // the lane of note i, and the notes before it
#pragma unroll
    for (int step = 16; step; step /= 2) {
      const uint32_t x = __shfl_sync(kAllLanes, upto, owner + step - 1);
      if (x <= i) {
        owner += step;
        before = x;
      }
    }
    if (i < all) f(notes[32 * (i - before) + owner], owner);
  }
  __syncwarp();
}

// One pass, which was started: candidates go to the list, the sums are of all others, all
// relative to `ref`, which none of them is above.  So no maximum is kept (with one, 8,192
// rows of 152,064 bfloat16 logits took 470 us, without 433).  A vector that has a candidate is
// taken out whole and noted; the warp looks at those at the end, or when a lane may have no
// room for another round's.
template <typename T, int NT, int ST, bool ENT, bool FUSED, bool LONG>
__device__ __forceinline__ RowSum take_part(const Part<T, NT, ST> &x, uint4 *ring, Bound b,
                                            float ref, const Candidates &to, uint32_t *noted,
                                            Carried *carried, float c) {
  const RowLog<T, FUSED> log(ref, c);
  F2 s(0.f), u(0.f);
  if (x.single()) {
    const uint32_t at = x.single_at();
    const float v = to_f32(x.p[at]);
    if (b.holds(v, x.first + at)) to.add(v, x.first + at);
    else add_one<T, ENT, FUSED>(s, u, log, v);
  }
  const uint32_t lane = threadIdx.x & 31;
  uint32_t n = 0;
  auto take = [&](uint32_t g) {
    async_wait<ST - 1>();
    uint4 w[kUnroll];
    x.load(w, ring, g);
    float m[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) m[k] = Vec16<T>::max(w[k]);
    if (fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) >= b.least) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (m[k] >= b.least) {
          noted[32 * n++ + lane] = kUnroll * g + k;
          w[k] = no_logits<T>();
        }
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) add_vector<T, ENT, FUSED>(s, u, w[k], log);
    x.fetch(ring, g + ST);
    if (__any_sync(kAllLanes, n > (g + 1 < x.rounds ? kNoted - kUnroll : 0))) {
      each_note(noted, n, [&](uint32_t note, uint32_t owner) {
        if (to.full()) return;
        const uint32_t round = note / kUnroll, k = note % kUnroll;
        add_but<T, ENT, FUSED>(s, u, log, x.vec_of(ring, round, k, owner),
                               x.column(x.vec_at(round, k, owner)), b, to);
      });
      n = 0;
    }
  };
  each_round<T, LONG, ENT>(x.rounds, carried, s, u, take);
  return sums_of<LONG>(carried, ref, s, u);
}
// The same relative to each thread's maximum, where the sums ask for that: rare.
template <typename T, int NT, int ST, bool ENT, bool LONG>
__device__ __forceinline__ RowSum take_carefully(const Part<T, NT, ST> &x, uint4 *ring, Bound b,
                                                 const Candidates &to, float c) {
  if constexpr (LONG) {
    FarSum a;
    x.each_vector(ring, [&](const uint4 &w, uint32_t i) {
      float m = kNegInf;
#pragma unroll
      for (int e = 0; e < Vec16<T>::kN; ++e) {
        const float v = to_f32(reinterpret_cast<const T *>(&w)[e]);
        m = b.holds(v, x.column(i) + e) ? m : fmaxf(m, v);
      }
      F2 s(0.f), u(0.f);
      add_but<T, ENT, false>(s, u, a.template raise<T, ENT>(m, c), w, x.column(i), b, to);
      a.s.add(s);
      if (ENT) a.u.add(u);
    });
    if (x.single()) {
      const uint32_t at = x.single_at();
      const float v = to_f32(x.p[at]);
      F2 s(0.f), u(0.f);
      if (b.holds(v, x.first + at)) to.add(v, x.first + at);
      else add_one<T, ENT, false>(s, u, a.template raise<T, ENT>(v, c), v);
      a.s.add(s);
      if (ENT) a.u.add(u);
    }
    return a.sum();
  }
  LaneSum a{kNegInf, F2(0.f), F2(0.f)};
  auto one = [&](float v, uint32_t column) {
    if (b.holds(v, column)) {
      to.add(v, column);
    } else {
      add_one<T, ENT, false>(a.s, a.u, raise<T, ENT, false>(a, v, c), v);
    }
  };
  x.each(ring, one);
  return row_sum(a);
}

// The count over the CTA's threads, in all of them.  red: a number per warp, free before.
template <int NT>
__device__ __forceinline__ uint32_t cta_count(uint32_t n, uint32_t *red) {
  n = __reduce_add_sync(kAllLanes, n);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = n;
  __syncthreads();
  const uint32_t lane = threadIdx.x & 31;
  n = __reduce_add_sync(kAllLanes, lane < (NT / 32) ? red[lane] : 0u);
  __syncthreads();
  return n;
}

// A bound that K to `room` numbers of n from column `first` on hold, searched from `lo` on
// (which more reach, unless it is the lowest) by counts: whether it is the K-th largest number
// itself (equal by the hundred, as masked ones are), else the number by halving; and of those
// equal to it an end, by steps that grow and by halving.  Rare, so that it only has to end: 80
// counts at the most.
template <typename Count>
__device__ __forceinline__ Bound search_bound(Count count, uint32_t first, uint32_t n, uint32_t lo,
                                              uint32_t K, uint32_t room) {
  constexpr uint32_t kAll = 0xffffffffu;
  enum { kLowest, kAbove, kValue, kColumn } look = lo == kLeastOrder ? kLowest : kAbove;
  uint32_t hi = 0xff800001u;              // nothing is above +infinity
  uint32_t a = first, b = first + n;  // too few with the end a, enough with b
  uint32_t step = 4 * K;
  for (;;) {
    if (look == kValue && hi - lo <= 1) look = kColumn;
    if (look == kColumn && b - a <= 1) return {of_order(lo), b};
    const uint32_t mid = look == kValue ? lo + (hi - lo) / 2 : lo;
    const uint32_t column = look == kAbove    ? 0
                            : look == kColumn ? a + min(step, (b - a) / 2)
                                              : kAll;
    const Bound probe{of_order(mid), column};
    const uint32_t c = count(probe);
    if (look != kAbove && c >= K && c <= room) return probe;
    if (look == kLowest) {
      if (c < K) return probe;
      look = kAbove;
    } else if (look == kAbove) {
      if (c < K) hi = lo + 1;
      look = kValue;
    } else if (look == kValue) {
      (c >= K ? lo : hi) = mid;
    } else {
      (c >= K ? b : a) = column;
      step = c >= K ? kAll : step > n / 8 ? n : 8 * step;  // (8 n may pass 32 bits)
    }
  }
}

// A warp's numbers, the largest first.
__device__ __forceinline__ uint32_t warp_ordered(uint32_t x) {
  const uint32_t lane = threadIdx.x & 31;
#pragma unroll
  for (uint32_t size = 2; size <= 32; size *= 2)
#pragma unroll
    for (uint32_t by = size / 2; by; by /= 2) {
      const uint32_t y = __shfl_xor_sync(kAllLanes, x, by);
      const bool large = ((lane & by) == 0) == ((lane & size) == 0 || size == 32);
      x = large ? max(x, y) : min(x, y);
    }
  return x;
}
// The place of x among the numbers of all threads, the largest first, equal ones in any order
// of their own.  runs: NT numbers, which then hold each warp's in order.
template <int NT>
__device__ __forceinline__ uint32_t place_of(uint32_t *x, uint32_t *runs) {
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  *x = warp_ordered(*x);
  runs[threadIdx.x] = *x;
  __syncthreads();
  constexpr uint32_t kSide = NT / 32 < 8 ? NT / 32 : 8;  // runs side by side
  uint32_t place = lane;
#pragma unroll 1
  for (uint32_t q = 0; q < NT / 32; q += kSide) {
    uint32_t at[kSide];
#pragma unroll
    for (uint32_t j = 0; j < kSide; ++j) at[j] = 0;
#pragma unroll
    for (uint32_t step = 32; step; step >>= 1) {
#pragma unroll
      for (uint32_t j = 0; j < kSide; ++j) {
        const uint32_t to = min(at[j] + step, 32u), y = runs[32 * (q + j) + to - 1];
        // larger, or as large in a run before
        at[j] = y + (q + j < wid) > *x ? to : at[j];
      }
    }
#pragma unroll
    for (uint32_t j = 0; j < kSide; ++j) place += q + j != wid ? at[j] : 0;
  }
  return place;
}

// A warp's keys, the largest first.
__device__ __forceinline__ Key warp_sorted(Key x) {
  const uint32_t lane = threadIdx.x & 31;
#pragma unroll
  for (uint32_t size = 2; size <= 32; size *= 2)
#pragma unroll
    for (uint32_t by = size / 2; by; by /= 2) {
      const Key y = __shfl_xor_sync(kAllLanes, x, by);
      const bool large = ((lane & by) == 0) == ((lane & size) == 0 || size == 32);
      x = large == (y > x) ? y : x;
    }
  return x;
}
// How many keys of `runs` descending runs of `each` (at most 2^k = most) are larger, four
// runs at a time side by side.
__device__ __forceinline__ uint32_t larger_in_runs(const Key *keys, uint32_t each, uint32_t runs,
                                                   uint32_t most, Key key) {
  uint32_t sum = 0;
#pragma unroll 1
  for (uint32_t q = 0; q < runs; q += 4) {
    uint32_t at[4] = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t step = most; step; step >>= 1) {
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t to = min(at[j] + step, each);
        const Key x = keys[min(q + j, runs - 1) * each + to - 1];
        at[j] = x > key ? to : at[j];
      }
    }
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) sum += q + j < runs ? at[j] : 0;
  }
  return sum;
}

struct TopOut {
  int32_t *ids;
  float *top_logp, *logp, *entropy, *rest, *stats;
  uint32_t top;
  uint32_t sampled;  // the place of the bound in a sample: see first_bound
};

// A row without a list, by threads i = 0 .. (128 at least, or as many as entries).
__device__ __forceinline__ void write_none(const TopOut &o, uint64_t t, uint32_t i) {
  if (i < o.top) {
    o.ids[t * o.top + i] = -1;
    o.top_logp[t * o.top + i] = kNegInf;
  }
  if (i) return;
  if (o.logp) o.logp[t] = 0.f;
  if (o.entropy) o.entropy[t] = 0.f;
  if (o.rest) o.rest[t] = 0.f;
  if (o.stats) o.stats[2 * t] = o.stats[2 * t + 1] = 0.f;
}

// Entry i of row t, and from entry 0 its other numbers.  M: the largest logit; S, U: the sums of
// the list relative to it; rest: those of all other tokens.
__device__ __forceinline__ void finish(const RowArgs &a, const TopOut &o, uint64_t t, uint32_t i,
                                       Key key, float M, float S, float U, const RowSum &rest,
                                       float zt) {
  if (rest.m == kNegInf) {
    S += rest.s;  // 0 or NaN
  } else {
    const float d = (rest.m - M) * a.c, f = ex2(d);
    S = fmaf(f, rest.s, S);
    U += f > 0.f ? f * fmaf(d, rest.s, rest.u) : 0.f;
  }
  const float ln = logf(S);
  const bool nan = S != S;
  if (i < o.top) {
    o.ids[t * o.top + i] = key && !nan ? (int32_t)column_of(key) : -1;
    o.top_logp[t * o.top + i] = nan ? S : key ? (value_of(key) - M) * a.inv_t - ln : kNegInf;
  }
  if (i) return;
  if (o.logp) o.logp[t] = (zt - M) * a.inv_t - ln;
  if (o.entropy) o.entropy[t] = ln - kLn2 * (U / S);
  if (o.rest)
    o.rest[t] = nan ? S : rest.s == 0.f ? kNegInf : (rest.m - M) * a.inv_t + logf(rest.s) - ln;
  if (o.stats) {
    o.stats[2 * t] = M;
    o.stats[2 * t + 1] = S;
  }
}

// A cluster of gridDim.y CTAs per row, each a part of it.
template <typename T, int NT, int ST, bool ENT, bool LONG>
__global__ void __launch_bounds__(NT, kStreamLanes / NT)
k_token_top(RowArgs a, TopOut o, Ctrl *ctrl) {
  constexpr bool F = kFused<T>;
  extern __shared__ uint4 shared_words[];
  __shared__ RowSum red[(NT / 32)], left[(NT / 32)];
  __shared__ uint32_t bound[NT], counts[(NT / 32)], noted[(NT / 32)][kNoted * 32];
  __shared__ float4 sums[kMostParts];  // what the cluster's CTAs send: m, S, U
  __shared__ Carried carried[LONG ? (NT / 32) : 1];
  __shared__ uint32_t count;
  __shared__ unsigned long long sent;
  const uint64_t t = blockIdx.x;
  const uint32_t part = blockIdx.y, np = gridDim.y, K = o.top;
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  Key *list = reinterpret_cast<Key *>(shared_words);  // [kRoom], as they come
  Key *inbox = list + kRoom;                          // [np][K], the lists of the parts
  uint4 *ring = shared_words + (kRoom + (np > 1 ? np * K : 0) + 1) / 2;
  Key *sorted = reinterpret_cast<Key *>(ring);        // [kRoom], in order, after the passes
  static_assert(kRoom * sizeof(Key) <= sizeof(uint4) * ST * kUnroll * NT, "in the ring");
  if (threadIdx.x == 0) {
    if (np > 1) {
      mbar_init(&sent, 1);
      if (part == 0) mbar_arrive_tx(&sent, np * (K * sizeof(Key) + sizeof(float4)));
      mbar_init_fence();
    }
    count = 0;
  }
  pdl_wait();
  pdl_launch();
  const int32_t target = a.target ? a.target[t] : 0;
  const bool skip = (a.mask && !a.mask[t]) || target < 0;
  if (skip || (uint32_t)target >= a.vocab) {
    if (part == 0) {
      write_none(o, t, threadIdx.x);
      if (!skip && threadIdx.x == 0)
        flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)target);
    }
    return;  // the whole cluster
  }
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
  const Part<T, NT, ST> x(row + first, first, n);
  x.start(ring);
  const float zt = a.target && part == 0 ? to_f32(row[target]) : 0.f;
  // The first rounds' numbers, each thread's largest, in order: the K-th is a bound that K of
  // the part reach, where these are all; else see first_bound.
  const uint32_t sample = min(x.rounds, (uint32_t)ST);
  const uint32_t full = min((uint32_t)NT, x.sp.vecs);  // threads that have any
  uint32_t nth = x.rounds > sample ? o.sampled : K;
  if (nth <= full) {
    float m = kNegInf;
    async_wait<0>();
#pragma unroll 1
    for (uint32_t g = 0; g < sample; ++g) {
      uint4 w[kUnroll];
      x.load(w, ring, g);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) m = fmaxf(m, Vec16<T>::max(w[k]));
    }
    uint32_t mine = order_of(m + 0.f);
    const uint32_t place = place_of<NT>(&mine, noted[0]);
    bound[place] = mine;
  }
  const bool sorted_sample = nth <= full;
  if (np > 1) cluster_started();
  __syncthreads();
  auto bound_at = [&](uint32_t i) {
    return sorted_sample && i - 1 < full ? max(kLeastOrder, bound[i - 1]) : kLeastOrder;
  };
  uint32_t lo = bound_at(nth);
  const Candidates to{list, &count, kRoom};
  Bound b{of_order(lo), 0xffffffffu};
  uint32_t found, reached = kLeastOrder;  // reached: by too many
  bool many = false, few = false;  // so far
  uint32_t tries = 0;
  RowSum sum;
#pragma unroll 1
  for (bool again = false, searched = false, careful = false;;) {
    // nothing but -infinity and NaN is left out by the lowest bound
    const bool all = lo == kLeastOrder && b.end == 0xffffffffu;
    const float ref = all ? 0.f : b.least;
    careful |= F && !sums_hold(ref, a.c);
    if (again) {
      if (threadIdx.x == 0) count = 0;
      if (!careful) x.start(ring);
      __syncthreads();
    }
    again = true;
    sum = careful ? take_carefully<T, NT, ST, ENT, LONG>(x, ring, b, to, a.c)
                  : take_part<T, NT, ST, ENT, F, LONG>(x, ring, b, ref, to, noted[wid],
                                                       &carried[LONG ? wid : 0], a.c);
    sum = warp_sum<T, false>(sum, a.c);
    if (lane == 0) red[wid] = sum;
    __syncthreads();
    found = count;
    const bool enough = searched || (found <= kRoom && (found >= K || all));
    if (enough) {
      sum = warp_sum<T, false, lanes_for(NT / 32)>(
          lane < (NT / 32) ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, a.c);
      if (!careful) sum = exact_sums<T>(sum, a.c);
      sum = {__shfl_sync(kAllLanes, sum.m, 0), __shfl_sync(kAllLanes, sum.s, 0),
             __shfl_sync(kAllLanes, sum.u, 0)};
      if (all) sum.m = kNegInf;  // (0 or NaN)
      // with sums as low as this the numbers lose bits or are lost: relative to their own
      // maximum they are not
      if (careful || all || !(sum.s < kLeastSum)) break;
      careful = true;
    }
    __syncthreads();
    if (enough) continue;
    // another of the sample's numbers, first a quarter of the way further (most lack little),
    // then more, unless there is none or that leads back
    const bool over = found > kRoom;
    if (over) reached = lo;
    (over ? many : few) = true;
    uint32_t next = lo;
    while (next == lo && nth - 1 < full) {
      const uint32_t by = max(1u, nth >> (tries < 2 ? 2 - tries : 0));
      nth = over ? (nth > by ? nth - by : nth / 2) : nth < full ? min(nth + by, full) : full + 1;
      next = bound_at(nth);
    }
    ++tries;
    if (nth - 1 < full && !(many && few)) {
      lo = next;
      b.least = of_order(lo);
    } else {
      auto count_all = [&](const Bound &probe) {
        uint32_t c = 0;
        x.each(ring, [&](float v, uint32_t at) { c += probe.holds(v, at); });
        return cta_count<NT>(c, counts);
      };
      b = search_bound(count_all, first, n, reached, K, kRoom);
      lo = order_of(b.least);
      searched = true;
    }
  }
  found = min(found, kRoom);  // (in bounds even if someone writes the row meanwhile)
  // In order: runs of 32 sorted by a warp each, then a key's place is its place in its own
  // run and the number of larger keys in each of the others.
  const uint32_t runs = (found + 31) / 32;
#pragma unroll 1
  for (uint32_t q = wid; q < runs; q += (NT / 32)) {
    const uint32_t i = 32 * q + lane;
    const Key key = warp_sorted(i < found ? list[i] : 0);
    list[i] = key;
  }
  __syncthreads();
#pragma unroll 1
  for (uint32_t i = threadIdx.x; i < found; i += NT) {
    const Key key = list[i];
    sorted[larger_in_runs(list, 32, runs, 32, key)] = key;
  }
  if (np > 1) cluster_wait();  // every CTA has started, so that its shared memory is there
  __syncthreads();
#pragma unroll 1
  for (uint32_t i = threadIdx.x; i < K; i += NT) {
    if (np > 1) send_key(inbox + part * K + i, i < found ? sorted[i] : 0, &sent, 0);
    else if (i >= found) sorted[i] = 0;
  }
  // Candidates behind the list join the others.
  LaneSum drop{kNegInf, F2(0.f), F2(0.f)};
  auto drop_key = [&](Key key) {
    const float z = value_of(key);
    add_one<T, ENT, false>(drop.s, drop.u, raise<T, ENT, false>(drop, z, a.c), z);
  };
#pragma unroll 1
  for (uint32_t i = K + threadIdx.x; i < found; i += NT) drop_key(sorted[i]);
  const Key *top = sorted;
  if (np > 1) {
    sum = joined<T, NT>(row_sum(drop), sum, 1, left, a.c);
    if (threadIdx.x == 0)
      send_float4(&sums[part], make_float4(sum.m, sum.s, sum.u, 0.f), &sent, 0);
    if (part) return;
    bool whole = mbar_wait(&sent, 0, kRowWaitNs);
    if (!whole) {
      if (lane == 0) flag(ctrl, DEVERR_TIMEOUT, t);
      whole = mbar_wait(&sent, 0, kRowWaitNs);  // none of them comes after the end
    }
    if (!__syncthreads_and(whole)) {
      write_none(o, t, threadIdx.x);
      return;
    }
    // A key's place in the row's list: how many are larger in each of the parts' lists.
    // Behind it, it joins the others, too.
    drop = {kNegInf, F2(0.f), F2(0.f)};
    uint32_t have = 0;  // keys in all lists: the row's list may be shorter than K
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < np * K; i += NT) {
      const Key key = inbox[i];
      if (!key) continue;
      ++have;
      const uint32_t rank = larger_in_runs(inbox, K, np, 128, key);
      if (rank < K) list[rank] = key;
      else drop_key(key);
    }
    have = cta_count<NT>(have, counts);
    if (threadIdx.x < K && threadIdx.x >= have) list[threadIdx.x] = 0;
    const float4 y = lane < np ? sums[lane] : make_float4(kNegInf, 0.f, 0.f, 0.f);
    sum = {y.x, y.y, y.z};
    top = list;
    __syncthreads();
  }
  // The list's own sums relative to the row's maximum, and the others'.
  const Key key = threadIdx.x < K ? top[threadIdx.x] : 0;
  const bool any = np > 1 ? top[0] != 0 : found != 0;
  const float M = any ? value_of(top[0]) : kNegInf;
  RowSum in{M, 0.f, 0.f};
  if (key) {
    const float y = (value_of(key) - M) * a.c;
    in.s = ex2(y);
    if (ENT) in.u = in.s * fmaxf(y, kNoLog);
  }
  if (wid * 32 < K) {
    in.s = warp_add(in.s);
    if (ENT) in.u = warp_add(in.u);
    if (lane == 0) red[wid] = in;
  }
  sum = joined<T, NT>(row_sum(drop), sum, np, left, a.c);
  if (wid * 32 >= K && wid) return;
  float S = 0.f, U = 0.f;
  for (uint32_t q = 0; 32 * q < K; ++q) {
    S += red[q].s;
    U += red[q].u;
  }
  if (!any && !(sum.s != sum.s)) {  // no token has a probability
    if (threadIdx.x == 0) flag(ctrl, DEVERR_ROW, t);
    write_none(o, t, threadIdx.x);
    return;
  }
  finish(a, o, t, threadIdx.x, key, M, S, U, sum, zt);
}

// A warp per row, held in shared memory (each lane its own vectors), for lists of up to 32:
// short rows cost a CTA more in its steps than in their numbers.  The bound is the K-th of the
// 64 largest numbers of the lanes' even and odd vectors, which K numbers reach.  8,000 rows of
// bfloat16 logits, lists of 20 (us; with a CTA of 128 threads): 500 columns 13 (64), 2,000 27
// (65), 4,000 49 (64), 6,000 73 (77); 600 rows: 5.1 (10), 8.3 (10), 11.6 (9.8); one row: 4.7
// (6.7), 7.4 (6.3), 9.4 (6.1).
constexpr uint32_t kSmallRoom = 256;
constexpr uint32_t kSmallTop = 32;
constexpr int kSmallRows = 4;  // per CTA

template <typename T, bool ENT>
__global__ void __launch_bounds__(32 * kSmallRows, 7)
k_top_small(RowArgs a, TopOut o, uint64_t rows, uint32_t vectors, Ctrl *ctrl) {
  constexpr int N = Vec16<T>::kN;
  extern __shared__ uint4 shared_words[];  // [kSmallRows][32 vectors]
  __shared__ Key lists[kSmallRows][2][kSmallRoom];
  __shared__ uint32_t counts[kSmallRows];
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, K = o.top;
  const uint64_t t = (uint64_t)blockIdx.x * kSmallRows + wid;
  Key *list = lists[wid][0], *sorted = lists[wid][1];
  pdl_wait();
  pdl_launch();
  if (t >= rows) return;
  const int32_t target = a.target ? a.target[t] : 0;
  const bool skip = (a.mask && !a.mask[t]) || target < 0;
  if (skip || (uint32_t)target >= a.vocab) {
    write_none(o, t, lane);
    if (!skip && lane == 0) flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)target);
    return;
  }
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
  const Span<T> sp(row, a.vocab);
  const uint4 *q = reinterpret_cast<const uint4 *>(row + sp.head);
  uint4 *w = shared_words + wid * vectors * 32 + lane;  // [32 k]
  const int all = (sp.vecs + 31) / 32;
#pragma unroll 4
  for (int k = 0; k < all; ++k) {
    if (32 * k + lane < sp.vecs) async_load(w + 32 * k, q + 32 * k + lane);
    else w[32 * k] = no_logits<T>();
  }
  async_mark();
  const bool one = lane < sp.head + sp.tail;  // a number before or behind the vectors
  const uint32_t at = lane < sp.head ? lane : lane + sp.vecs * N;
  const float v = one ? to_f32(row[at]) : kNegInf;
  const float zt = a.target ? to_f32(row[target]) : 0.f;
  auto column = [&](int k) { return sp.head + (32 * k + lane) * N; };
  // f(number, column) of the lane's numbers
  auto each = [&](auto f) {
    f(v, at);
#pragma unroll 1
    for (int k = 0; k < all; ++k) {
      const uint4 x = w[32 * k];
#pragma unroll
      for (int i = 0; i < N; ++i) f(to_f32(reinterpret_cast<const T *>(&x)[i]), column(k) + i);
    }
  };
  // a lane's largest of its even vectors and of its odd ones: the K-th of all
  float m = v, m1 = kNegInf;
  async_wait<0>();
  for (int k = 0; k < all; k += 2) {
    m = fmaxf(m, Vec16<T>::max(w[32 * k]));
    if (k + 1 < all) m1 = fmaxf(m1, Vec16<T>::max(w[32 * (k + 1)]));
  }
  uint32_t largest = warp_ordered(order_of(m + 0.f));
  {
    // two runs against each other: the larger of each pair are the 32 largest
    const uint32_t other = warp_ordered(order_of(m1 + 0.f));
    largest = max(largest, __shfl_sync(kAllLanes, other, 31 - lane));
#pragma unroll
    for (uint32_t by = 16; by; by /= 2) {
      const uint32_t y = __shfl_xor_sync(kAllLanes, largest, by);
      largest = lane & by ? min(largest, y) : max(largest, y);
    }
  }
  uint32_t lo = max(kLeastOrder, __shfl_sync(kAllLanes, largest, K - 1));
  const Candidates to{list, &counts[wid], kSmallRoom};
  Bound b{of_order(lo), 0xffffffffu};
  LaneSum sum;
  uint32_t found;
  for (bool own = false;;) {
    // nothing but -infinity and NaN is left out by the lowest bound
    const bool others = lo != kLeastOrder || b.end != 0xffffffffu;
    const float ref = own ? m : others ? b.least : 0.f;
    const RowLog<T, false> log(ref, a.c);
    F2 s(0.f), u(0.f);
    if (lane == 0) counts[wid] = 0;
    __syncwarp();
    if (b.holds(v, at)) to.add(v, at);
    else add_one<T, ENT, false>(s, u, log, v);
#pragma unroll 1
    for (int k = 0; k < all; ++k)
      if (const uint4 x = w[32 * k]; __any_sync(kAllLanes, Vec16<T>::max(x) >= b.least))
        add_but<T, ENT, false>(s, u, log, x, column(k), b, to);
      else
        add_vector<T, ENT, false>(s, u, x, log);
    __syncwarp();
    found = counts[wid];
    sum = {others ? ref : kNegInf, s, u};
    if (found > kSmallRoom) {  // equal ones, by the hundred
      auto count = [&](const Bound &probe) {
        uint32_t c = 0;
        each([&](float z, uint32_t i) { c += probe.holds(z, i); });
        return __reduce_add_sync(kAllLanes, c);
      };
      b = search_bound(count, 0, a.vocab, lo, K, kSmallRoom);
      lo = order_of(b.least);
      __syncwarp();
      continue;
    }
    if (own || !others || !(warp_add(s.x() + s.y()) < kLeastSum)) break;
    // so low that the numbers lose bits: relative to their own maximum
    m = kNegInf;
    each([&](float z, uint32_t i) { m = b.holds(z, i) ? m : fmaxf(m, z); });
#pragma unroll
    for (int i = 16; i; i >>= 1) m = fmaxf(m, __shfl_xor_sync(kAllLanes, m, i));
    own = true;
    __syncwarp();
  }
  const uint32_t runs = (found + 31) / 32;
#pragma unroll 1
  for (uint32_t r = 0; r < runs; ++r)
    list[32 * r + lane] = warp_sorted(32 * r + lane < found ? list[32 * r + lane] : 0);
  __syncwarp();
  if (runs > 1) {
#pragma unroll 1
    for (uint32_t i = lane; i < found; i += 32) {
      const Key key = list[i];
      sorted[larger_in_runs(list, 32, runs, 32, key)] = key;
    }
    __syncwarp();
  } else {
    sorted = list;
  }
  const Key key = lane < K && lane < found ? sorted[lane] : 0;
  // candidates behind the list join the others
#pragma unroll 1
  for (uint32_t i = K + lane; i < found; i += 32) {
    const float z = value_of(sorted[i]);
    add_one<T, ENT, false>(sum.s, sum.u, raise<T, ENT, false>(sum, z, a.c), z);
  }
  const RowSum rest = warp_sum<T, false>(row_sum(sum), a.c);
  if (!found && !(rest.s != rest.s)) {  // no token has a probability
    if (lane == 0) flag(ctrl, DEVERR_ROW, t);
    write_none(o, t, lane);
    return;
  }
  const float M = found ? value_of(__shfl_sync(kAllLanes, key, 0)) : kNegInf;
  float S = 0.f, U = 0.f;
  if (key) {
    const float y = (value_of(key) - M) * a.c;
    S = ex2(y);
    if (ENT) U = S * fmaxf(y, kNoLog);
  }
  S = warp_add(S);
  if (ENT) U = warp_add(U);
  finish(a, o, t, lane, key, M, S, U, rest, zt);
}

}  // namespace

// The bound for K numbers of a part from `sample` of its `rounds` of vectors: its place among
// the threads' largest.  The sample's share of the K is Poisson distributed (the vectors are
// spread evenly), so that three deviations more are hardly ever too few; so many numbers are
// the largest of fewer threads, some of which have several.
static uint32_t first_bound(double K, double sample, double rounds, double threads) {
  const double share = K * sample / std::max(rounds, sample);
  const double some = share + 3.0 * std::sqrt(share);
  return (uint32_t)std::max(std::ceil(threads * (1.0 - std::exp(-some / threads))), 1.0);
}

cudaError_t launch_token_top(edp_ctx *ctx, const Logits &z, uint32_t top, int32_t *ids,
                             float *top_logp, float *logp, float *entropy, float *rest,
                             float *stats, cudaStream_t s) {
  const uint64_t row_bytes = (uint64_t)z.vocab * (z.dtype == EDP_F32 ? 4 : 2);
  const uint64_t sms = (uint64_t)ctx->coop_sms;
  const uint64_t small = z.rows >= 8 * sms   ? top <= 8 ? 12288 : 8192
                         : z.rows >= 2 * sms ? 4096
                                             : 2048;
  if (top <= kSmallTop && row_bytes <= small) {
    return by_type(z.dtype, [&](auto x) {
      using T = decltype(x);
      const TopOut o{ids, top_logp, logp, entropy, rest, stats, top, 0};
      auto kern = entropy ? k_top_small<T, true> : k_top_small<T, false>;
      const uint32_t vectors = (uint32_t)(row_bytes / 16 + 31) / 32;  // per lane
      const cudaError_t e = cudaFuncSetAttribute(
          kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 48 * 1024);
      if (e != cudaSuccess) return e;
      return launch_rows(kern, (z.rows + kSmallRows - 1) / kSmallRows, 1, false, 32 * kSmallRows,
                         (size_t)kSmallRows * vectors * 512, s, row_args(z), o, z.rows, vectors,
                         ctx->ctrl);
    });
  }
  const StreamShape shape = stream_shape(ctx, z, top);
  const uint32_t parts = shape.parts;
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    return by_shape<T>(shape, [&](auto threads, auto stages, auto is_long) {
      constexpr int NT = decltype(threads)::value, ST = decltype(stages)::value;
      constexpr bool LONG = decltype(is_long)::value;
      const uint32_t sampled =
          first_bound(top, ST, std::ceil((double)shape.vecs / (NT * kUnroll)), NT);
      const TopOut o{ids, top_logp, logp, entropy, rest, stats, top, sampled};
      auto kern = entropy ? k_token_top<T, NT, ST, true, LONG>
                          : k_token_top<T, NT, ST, false, LONG>;
      const uint32_t keys = kRoom + (parts > 1 ? parts * top : 0);
      const size_t bytes = sizeof(uint4) * ((keys + 1) / 2 + ST * kUnroll * NT);
      const cudaError_t e = cudaFuncSetAttribute(
          kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 96 * 1024);
      if (e != cudaSuccess) return e;
      return launch_rows(kern, z.rows, parts, true, NT, bytes, s, row_args(z), o, ctx->ctrl);
    });
  });
}

}  // namespace edp
