// k_top.cu -- the likeliest tokens of rows of logits with their log-probabilities, the
// log-probability of a given token, the entropy, and the logarithm of what is outside of
// the list.
//
// One pass over memory.  A CTA of each row (or of each part of a row, joined by a cluster)
// looks at its first rounds of vectors for a bound that a little more than the K largest
// logits reach, most likely: each lane's largest, a warp's r-th largest of those, and of the
// warps' the one that lies right.  Then it passes over all: numbers that reach the bound are
// collected as candidates, the others go into the sums of exponentials, so that `rest` comes
// without cancellation.  Fewer than K candidates ask for another pass with a lower bound
// (the warps' least; one row in a hundred or less), too many (logits that are equal by the
// hundred) for a search of the bound by halving.  The candidates are ordered by value, then
// index (all different, so that nothing depends on the order in which they came), and those
// behind the list join the sums.  A row's first CTA merges its parts' lists.
#include <cmath>

#include "edp_rows.cuh"

namespace edp {
namespace {

constexpr int kThreads = 256;
constexpr int kCtas = 4;    // per SM, which bounds the registers
constexpr int kStages = 2;  // rounds in shared memory or on their way there
constexpr int kWarps = kThreads / 32;
constexpr uint32_t kMostParts = 8;
constexpr uint32_t kNoted = 8;    // vectors of a thread that wait to be looked at
constexpr float kLeastSum = 0x1p-64f;
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
__device__ __forceinline__ void async_mark() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A part of a row as its CTA's threads pass over it: the vectors in segments of a warp's 32,
// kUnroll segments per warp and round, and the numbers before and behind the vectors by the
// first threads.  Round g takes segments g, g + rounds, g + 2 rounds, ..., so that the
// first round's are spread evenly over the part.
template <typename T>
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
    rounds = max(1u, (sp.vecs + 32 * kWarps * kUnroll - 1) / (32 * kWarps * kUnroll));
    apart = 32 * kWarps * rounds;
    const uint32_t at = vec_at(0, 0, threadIdx.x & 31), last = at + (kUnroll - 1) * apart;
    mine = reinterpret_cast<const uint4 *>(p + sp.head) + at;
    whole = last < sp.vecs ? min(rounds, (sp.vecs - last + 31) / 32) : 0;
  }
  __device__ __forceinline__ uint32_t vec_at(uint32_t g, uint32_t k, uint32_t lane) const {
    return ((k * kWarps + (threadIdx.x >> 5)) * rounds + g) * 32 + lane;
  }
  __device__ __forceinline__ uint32_t column(uint32_t vec) const {
    return first + sp.head + vec * Vec16<T>::kN;
  }
  __device__ __forceinline__ uint4 vec(uint32_t i) const {
    return reinterpret_cast<const uint4 *>(p + sp.head)[i];
  }
  // Round g of this thread's vectors to its own places, -infinity where there are none.
  __device__ __forceinline__ void fetch(uint4 *ring, uint32_t g) const {
    uint4 *to = ring + g % kStages * (kUnroll * kThreads) + threadIdx.x;
    const uint4 *from = mine + 32 * g;
    if (g < whole) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) async_load(to + k * kThreads, from + k * apart);
    } else if (g < rounds) {
#pragma unroll 1
      for (int k = 0; k < kUnroll; ++k) {
        if (vec_at(g, k, threadIdx.x & 31) < sp.vecs) async_load(to + k * kThreads, from + k * apart);
        else to[k * kThreads] = no_logits<T>();
      }
    }
    async_mark();
  }
  __device__ __forceinline__ void start(uint4 *ring) const {
#pragma unroll
    for (int g = 0; g < kStages; ++g) fetch(ring, g);
  }
  __device__ __forceinline__ void load(uint4 (&w)[kUnroll], const uint4 *ring, uint32_t g) const {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
      w[k] = ring[(g % kStages * kUnroll + k) * kThreads + threadIdx.x];
  }
  __device__ __forceinline__ bool single() const { return threadIdx.x < sp.head + sp.tail; }
  __device__ __forceinline__ uint32_t single_at() const {
    return threadIdx.x < sp.head ? threadIdx.x : threadIdx.x + sp.vecs * Vec16<T>::kN;
  }
  // f(number, column) of this thread's numbers
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if (single()) f(to_f32(p[single_at()]), first + single_at());
    for (uint32_t i = threadIdx.x; i < sp.vecs; i += kThreads) {
      const uint4 w = vec(i);
#pragma unroll
      for (int k = 0; k < Vec16<T>::kN; ++k)
        f(to_f32(reinterpret_cast<const T *>(&w)[k]), column(i) + k);
    }
  }
};

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
  __device__ __forceinline__ void add(float v, uint32_t column) const {
    const uint32_t at = atomicAdd(count, 1u);
    if (at < kRoom) list[at] = key_of(v, column);
  }
};

// A number's share of the sums relative to `log`.
template <typename T, bool ENT, bool FUSED>
__device__ __forceinline__ void add_one(F2 &s, F2 &u, const RowLog<T, FUSED> &log, float v) {
  const float y = log.of(v), e = ex2(y);
  s = s + F2(e, 0.f);
  if (ENT) u = fma2(F2(e, 0.f), F2(fmaxf(y, kNoLog), 0.f), u);
}
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
// rows of 152,064 bfloat16 logits took 470 us, without XXX).  A vector that has a candidate is
// taken out whole and noted; the warp looks at those at the end, or when a lane may have no
// room for another round's.
template <typename T, bool ENT, bool FUSED>
__device__ __forceinline__ RowSum take_part(const Part<T> &x, uint4 *ring, Bound b, float ref,
                                            const Candidates &to, uint32_t *noted, float c) {
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
  for (uint32_t g = 0; g < x.rounds; ++g) {
    async_wait<kStages - 1>();
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
    x.fetch(ring, g + kStages);
    if (__any_sync(kAllLanes, n > (g + 1 < x.rounds ? kNoted - kUnroll : 0))) {
      each_note(noted, n, [&](uint32_t note, uint32_t owner) {
        const uint32_t at = x.vec_at(note / kUnroll, note % kUnroll, owner);
        add_but<T, ENT, FUSED>(s, u, log, x.vec(at), x.column(at), b, to);
      });
      n = 0;
    }
  }
  return {ref, s.x() + s.y(), u.x() + u.y()};
}
// The same relative to each thread's maximum, where the sums ask for that: rare.
template <typename T, bool ENT>
__device__ __forceinline__ RowSum take_carefully(const Part<T> &x, Bound b, const Candidates &to,
                                                 float c) {
  LaneSum a{kNegInf, F2(0.f), F2(0.f)};
  auto one = [&](float v, uint32_t column) {
    if (b.holds(v, column)) {
      to.add(v, column);
    } else {
      add_one<T, ENT, false>(a.s, a.u, raise<T, ENT, false>(a, v, c), v);
    }
  };
  x.each(one);
  return row_sum(a);
}

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

// A bound that K to kRoom numbers hold, by halving from `lo` on (which K or more reach,
// unless it is the lowest): or, where numbers are equal by the hundred, exactly K.  Rare, so
// that it only has to end: 64 counts at the most.
template <typename T>
__device__ __forceinline__ Bound search_bound(const T *p, uint32_t first, uint32_t n, uint32_t lo,
                                           uint32_t K, uint32_t *red) {
  const Part<T> x(p, first, n);
  auto reach = [&](uint32_t bound) {
    uint32_t c = 0;
    x.each([&](float v, uint32_t) { c += v >= of_order(bound); });
    return cta_count(c, red);
  };
  uint32_t hi = 0xff800001u, some = kRoom + 1;  // nothing is above +infinity
  if (lo == kLeastOrder) some = reach(lo);
  if (some < K) return {of_order(lo), 0xffffffffu};
  while (hi - lo > 1 && some > kRoom) {
    const uint32_t mid = lo + (hi - lo) / 2, c = reach(mid);
    if (c >= K) {
      lo = mid;
      some = c;
    } else {
      hi = mid;
    }
  }
  const float least = of_order(lo);
  if (some <= kRoom) return {least, 0xffffffffu};
  // of the numbers equal to it those before a column: fewer than needed before a, as many
  // before b
  const uint32_t above = reach(hi);
  uint32_t a = first, b = first + n;
  while (b - a > 1) {
    const uint32_t mid = a + (b - a) / 2;
    uint32_t c = 0;
    x.each([&](float v, uint32_t column) { c += v == least && column < mid; });
    if (cta_count(c, red) + above >= K) b = mid;
    else a = mid;
  }
  return {least, b};
}

// The r-th largest (MAX) or smallest of a warp's numbers, r <= 32; ties by lane.
template <bool MAX>
__device__ __forceinline__ uint32_t warp_nth(uint32_t x, uint32_t r) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t best = 0;
  for (uint32_t k = 0; k < r; ++k) {
    best = MAX ? __reduce_max_sync(kAllLanes, x) : __reduce_min_sync(kAllLanes, x);
    if (lane == __ffs(__ballot_sync(kAllLanes, x == best)) - 1) x = MAX ? 0u : 0xffffffffu;
  }
  return best;
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
  for (uint32_t q = 0; q < runs; q += 4) {
    uint32_t at[4] = {0, 0, 0, 0};
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

// A cluster of gridDim.y CTAs per row, each a part of it.
template <typename T, bool ENT>
__global__ void __launch_bounds__(kThreads, kCtas)
k_token_top(RowArgs a, TopOut o, Ctrl *ctrl) {
  constexpr bool F = kFused<T>;
  extern __shared__ uint4 shared_words[];
  __shared__ RowSum red[kWarps], left[kWarps];
  __shared__ uint32_t bound[kWarps], counts[kWarps], noted[kWarps][kNoted * 32];
  __shared__ float4 sums[kMostParts];  // what the cluster's CTAs send: m, S, U
  __shared__ uint32_t count;
  __shared__ unsigned long long sent;
  const uint64_t t = blockIdx.x;
  const uint32_t part = blockIdx.y, np = gridDim.y, K = o.top;
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  Key *list = reinterpret_cast<Key *>(shared_words);  // [kRoom], as they come
  Key *inbox = list + kRoom;                          // [np][K], the lists of the parts
  uint4 *ring = shared_words + (kRoom + (np > 1 ? np * K : 0) + 1) / 2;
  Key *sorted = reinterpret_cast<Key *>(ring);        // [kRoom], in order, after the passes
  static_assert(kRoom * sizeof(Key) <= sizeof(uint4) * kStages * kUnroll * kThreads, "in the ring");
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
      write_none(o, t);
      if (!skip && threadIdx.x == 0)
        flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)target);
    }
    return;  // the whole cluster
  }
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
  const Part<T> x(row + first, first, n);
  x.start(ring);
  const float zt = a.target && part == 0 ? to_f32(row[target]) : 0.f;
  // The first rounds' numbers, each lane's largest: a bound that K of the part reach (where
  // they are all, the least of the warps' r-th largest; else one that 2.5 K most likely do).
  const uint32_t sample = min(x.rounds, (uint32_t)kStages);
  const uint32_t full = x.rounds > 1 ? kWarps : min((uint32_t)kWarps, x.sp.vecs / 32);
  uint32_t r = 33, nth = 1;
  if (full) {
    if (x.rounds == sample) {
      r = (K + full - 1) / full;
    } else {
      const float per_warp = 2.5f * (float)(K * sample) / (float)(x.rounds * kWarps);
      r = max(1u, (uint32_t)(per_warp + 0.5f));
      nth = r > 1 ? kWarps * 2 / 5 : max(1u, (uint32_t)(kWarps * __expf(-per_warp)));
    }
  }
  uint32_t lo = kLeastOrder, lower = kLeastOrder;
  if (r <= 32) {
    float m = kNegInf;
    async_wait<0>();
    for (uint32_t g = 0; g < sample; ++g) {
      uint4 w[kUnroll];
      x.load(w, ring, g);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) m = fmaxf(m, Vec16<T>::max(w[k]));
    }
    const uint32_t best = warp_nth<true>(order_of(m + 0.f), r);
    if (lane == 0) bound[wid] = best;
  }
  if (np > 1) cluster_started();
  __syncthreads();
  if (r <= 32) {
    const uint32_t each = lane < full ? bound[lane] : 0xffffffffu;
    lower = max(lo, __reduce_min_sync(kAllLanes, each));
    lo = nth > 1 ? max(lo, warp_nth<false>(each, nth)) : lower;
  }
  const Candidates to{list, &count};
  Bound b{of_order(lo), 0xffffffffu};
  uint32_t found;
  RowSum sum;
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
    sum = careful ? take_carefully<T, ENT>(x, b, to, a.c)
                  : take_part<T, ENT, F>(x, ring, b, ref, to, noted[wid], a.c);
    sum = warp_sum<T, false>(sum, a.c);
    if (lane == 0) red[wid] = sum;
    __syncthreads();
    found = count;
    const bool enough = searched || (found <= kRoom && (found >= K || all));
    if (enough) {
      sum = warp_sum<T, false, lanes_for(kWarps)>(
          lane < kWarps ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, a.c);
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
    if (found <= kRoom && lo != lower) {
      lo = lower;
      b.least = of_order(lo);
    } else {
      b = search_bound<T>(row + first, first, n, found > kRoom ? lo : kLeastOrder, K, counts);
      lo = order_of(b.least);
      searched = true;
    }
  }
  found = min(found, kRoom);  // (in bounds even if someone writes the row meanwhile)
  // In order: runs of 32 sorted by a warp each, then a key's place is its place in its own
  // run and the number of larger keys in each of the others.
  const uint32_t runs = (found + 31) / 32;
  for (uint32_t q = wid; q < runs; q += kWarps) {
    const uint32_t i = 32 * q + lane;
    const Key key = warp_sorted(i < found ? list[i] : 0);
    list[i] = key;
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < found; i += kThreads) {
    const Key key = list[i];
    sorted[larger_in_runs(list, 32, runs, 32, key)] = key;
  }
  if (np > 1) cluster_wait();  // every CTA has started, so that its shared memory is there
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < K; i += kThreads) {
    if (np > 1) send_key(inbox + part * K + i, i < found ? sorted[i] : 0, &sent, 0);
    else if (i >= found) sorted[i] = 0;
  }
  // Candidates behind the list join the others.
  LaneSum drop{kNegInf, F2(0.f), F2(0.f)};
  auto drop_key = [&](Key key) {
    const float z = value_of(key), y = raise<T, ENT, false>(drop, z, a.c).of(z), e = ex2(y);
    drop.s = drop.s + F2(e, 0.f);
    if (ENT) drop.u = fma2(F2(e, 0.f), F2(fmaxf(y, kNoLog), 0.f), drop.u);
  };
  for (uint32_t i = K + threadIdx.x; i < found; i += kThreads) drop_key(sorted[i]);
  {
    const RowSum mine = warp_sum<T, false>(row_sum(drop), a.c);
    if (lane == 0) left[wid] = mine;
  }
  __syncthreads();
  if (wid == 0) {
    static_assert(kWarps <= 16, "and the sums of the others in lane 16");
    sum = {__shfl_sync(kAllLanes, sum.m, 0), __shfl_sync(kAllLanes, sum.s, 0),
           __shfl_sync(kAllLanes, sum.u, 0)};
    sum = warp_sum<T, false>(lane < kWarps ? left[lane]
                             : lane == 16  ? sum
                                           : RowSum{kNegInf, 0.f, 0.f}, a.c);
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
    // A key's place in the row's list: how many are larger in each of the parts' lists.
    drop = {kNegInf, F2(0.f), F2(0.f)};
    uint32_t have = 0;  // keys in all lists: the row's list may be shorter than K
    for (uint32_t i = threadIdx.x; i < np * K; i += kThreads) {
      const Key key = inbox[i];
      if (!key) continue;
      ++have;
      const uint32_t rank = larger_in_runs(inbox, K, np, 128, key);
      if (rank < K) list[rank] = key;
    }
    have = cta_count(have, counts);
    for (uint32_t i = have + threadIdx.x; i < K; i += kThreads) list[i] = 0;
    __syncthreads();
    // What of the parts' lists is not of the row's joins the others, too.
    const Key last = list[K - 1];
    for (uint32_t i = threadIdx.x; i < np * K; i += kThreads) {
      const Key key = inbox[i];
      if (key && key < last) drop_key(key);
    }
    const RowSum mine = warp_sum<T, false>(row_sum(drop), a.c);
    if (lane == 0) left[wid] = mine;
    __syncthreads();
    if (wid) return;
    const float4 y = lane - 16 < np ? sums[lane - 16] : make_float4(kNegInf, 0.f, 0.f, 0.f);
    sum = warp_sum<T, false>(lane < kWarps ? left[lane] : RowSum{y.x, y.y, y.z}, a.c);
  }
  if (wid) return;
  sum = {__shfl_sync(kAllLanes, sum.m, 0), __shfl_sync(kAllLanes, sum.s, 0),
         __shfl_sync(kAllLanes, sum.u, 0)};
  const Key *top = np > 1 ? list : sorted;
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
  const TopOut o{ids, top_logp, logp, entropy, rest, stats, top};
  return by_type(z.dtype, [&](auto x) {
    using T = decltype(x);
    const uint32_t parts = row_parts(ctx, z, 2);
    auto kern = entropy ? k_token_top<T, true> : k_token_top<T, false>;
    const uint32_t keys = kRoom + (parts > 1 ? parts * top : 0);
    const size_t bytes = sizeof(uint4) * ((keys + 1) / 2 + kStages * kUnroll * kThreads);
    const cudaError_t e = cudaFuncSetAttribute(
        kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024);
    if (e != cudaSuccess) return e;
    return launch_rows(kern, z.rows, parts, true, kThreads, bytes, s, row_args(z), o, ctx->ctrl);
  });
}

}  // namespace edp
