// k_pref.cu -- the preference loss over pairs of sequences of a packed batch, with
// the gradient of the tokens' log-probabilities.
//
// Three steps, since a token's gradient needs its pair's whole sequences: the
// sums of logp - ref by sequence (9 bytes a token), the pairs, and the gradient
// (1 byte read, 4 written).  For the sums each warp has a run of tokens: within
// a sequence its lanes add on their own; where sequences end in a tile, a
// segmented scan gives each one's part of the run.  Whoever wants a sequence's
// sum adds its parts in order.  A sequence's gradients from its pairs add up as
// whole numbers, in any order to the same bits.  A batch of up to 8,192 tokens
// takes all three steps in one CTA.
//
// 8,192 sequences of 128 to 4,096 tokens in 7,680 pairs, masked, with a reference (17.3 M
// tokens): 68 us, 3.3 TB/s; the floor is 34 us.  Sums 34 us, pairs 8, gradient 20.  What
// bounds it: the round trips at the ends of sequences (each warp meets two) and the three
// kernels' starts and ends.  With a search per token and fp64 pairs: 642 us.
#include "edp_loss.cuh"

namespace edp {
namespace {

constexpr int kThreads = 512;
constexpr int kPerSm = 2;            // CTAs of the sums, in one wave
constexpr int kGradPerSm = 4;        // and of the gradient
constexpr int kSmallThreads = 1024;  // a batch of up to 8,192 tokens, in one CTA
constexpr uint32_t kSmallRun = 2 * kTile;
constexpr uint32_t kSmallSeqs = 512;
constexpr int kPairThreads = 128;
constexpr uint32_t kSmallPairs = 4096;
constexpr uint32_t kAtOnce = 4;  // tiles in flight per warp

// A sequence's part of a run.
struct alignas(16) SeqPart {
  float hi, lo;
  uint32_t n, pad;
};
// Gradient by a sequence's u, before norm and grad_scale, in whole numbers of
// 2^-20 and of 2^-62.
struct SeqGrad {
  unsigned long long hi, lo;
};

struct PrefScratch {
  SeqPart *inner;  // [n_seq] the part in the run where the sequence starts
  SeqPart *head;   // [runs] the part of the sequence that comes in from the left
  SeqGrad *grad;   // [n_seq]
  uint32_t *bad;   // [n_seq] a gradient is not a finite number below 2^22
  Pair *part;
  uint32_t run;    // tokens per warp, a multiple of a tile's
};

struct PrefRule {
  df beta, margin, half;  // half: 1 / (2 beta)
  df per_norm, per_pair;  // 1 / norm and 1 / pairs
  float smooth;
  uint32_t kind, average;
};

struct PrefIn {
  TokenSet s;
  const float *logp, *ref;
  const int64_t *pair;
  uint32_t n_pair;
};
struct PrefOut {
  float *loss, *ratio, *pair_loss, *dlogp;
};

struct Run {
  Pair v;
  uint32_t n;
};
__device__ __forceinline__ Run run_join(Run a, Run b) { return {pair_join(a.v, b.v), a.n + b.n}; }
__device__ __forceinline__ Run run_up(Run a, int o) {
  return {{__shfl_up_sync(kAllLanes, a.v.hi, o), __shfl_up_sync(kAllLanes, a.v.lo, o)},
          __shfl_up_sync(kAllLanes, a.n, o)};
}
__device__ __forceinline__ void run_add(Run &r, float lp, float ref) {
  pair_add(r.v, lp);
  pair_add(r.v, -ref);
  ++r.n;
}

// Parts of the sequences in tokens [begin, stop) of a warp; [first, end) are those
// that the sequences hold.
template <bool VEC>
__device__ __forceinline__ void run_parts(const PrefIn &in, const PrefScratch &x, uint64_t begin,
                                          uint64_t stop, uint64_t first, uint64_t end) {
  const TokenSet &s = in.s;
  const int lane = threadIdx.x & 31;
  const uint32_t n_seq = (uint32_t)s.n_seq;
  stop = min(stop, end);
  if (begin >= stop) return;
  // the part of sequence q, which starts at `start`
  auto emit = [&](uint32_t q, uint64_t start, const Run &r) {
    const SeqPart p{r.v.hi, r.v.lo, r.n, 0};
    if (start >= begin) {
      x.inner[q] = p;
      x.grad[q] = SeqGrad{0, 0};
      x.bad[q] = 0;
    } else {
      x.head[begin / x.run] = p;
    }
  };
  const Run none{{0.f, 0.f}, 0};
  Run mine = none;  // a lane's share of the sequence that is open
  // the sequence of the tile's first token, and where the one after it ends
  SeqWalk walk;
  walk.start(s.off, n_seq, begin);
  uint64_t start = s.off[walk.q];
  auto end_after = [&](uint32_t q) { return q + 1 < n_seq ? s.off[q + 2] : ~0ull; };
  uint64_t after = end_after(walk.q);
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  for (uint64_t t0 = begin; t0 < stop; t0 += kTile) {
    // tiles that the sequence goes through, kAtOnce of them in flight
    if (VEC && t0 >= first) {
      const uint64_t top = min(walk.next, stop), room = top > t0 ? top - t0 : 0;
      for (uint32_t n = room > kTile ? (uint32_t)min((room - 1) / kTile, (uint64_t)x.run) : 0; n;) {
        const uint32_t m = min(n, kAtOnce);
        float4 lp[kAtOnce], rf[kAtOnce];
        uint32_t mk[kAtOnce];
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
          const uint64_t t = t0 + k * kTile + 4 * lane;
          lp[k] = rf[k] = zero;
          mk[k] = 0;
          if (k >= m) continue;
          lp[k] = *reinterpret_cast<const float4 *>(in.logp + t);
          if (in.ref) rf[k] = *reinterpret_cast<const float4 *>(in.ref + t);
          mk[k] = s.mask ? *reinterpret_cast<const uint32_t *>(s.mask + t) : 0xffffffffu;
        }
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
          const float l4[4] = {lp[k].x, lp[k].y, lp[k].z, lp[k].w};
          const float r4[4] = {rf[k].x, rf[k].y, rf[k].z, rf[k].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool b = mk[k] & (0xffu << (8 * i));
            pair_add(mine.v, b ? l4[i] : 0.f);
            if (in.ref) pair_add(mine.v, b ? -r4[i] : 0.f);
          }
          mine.n += some_bytes(mk[k]);
        }
        t0 += m * kTile;
        n -= m;
      }
    }
    const uint64_t t = t0 + 4 * lane;
    const float4 lp = load4<VEC>(in.logp, t, s.n);
    const float4 rf = in.ref ? load4<VEC>(in.ref, t, s.n) : zero;
    const uint32_t bits = token_bits<VEC>(s, t, first, stop);
    const float l4[4] = {lp.x, lp.y, lp.z, lp.w}, r4[4] = {rf.x, rf.y, rf.z, rf.w};
    // up to one end in this tile: the lanes go on adding, and give their shares at it
    if (t0 + kTile < walk.next || t0 + kTile < after) {
      const bool ends = walk.next <= t0 + kTile;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((bits >> i & 1u) && t + i < walk.next) run_add(mine, l4[i], r4[i]);
      if (!ends) continue;
      const Run all{warp_join(mine.v), __reduce_add_sync(kAllLanes, mine.n)};
      if (lane == 0 && walk.next > start && walk.next > begin) emit(walk.q, start, all);
      mine = none;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((bits >> i & 1u) && t + i >= walk.next) run_add(mine, l4[i], r4[i]);
      start = walk.next;
      walk.next = after;
      ++walk.q;
      after = end_after(walk.q);
      continue;
    }
    // several
    SeqWalk ahead = walk;
    ahead.to(s.off, n_seq, min(t0 + kTile, stop) - 1);
    Run carry{warp_join(mine.v), __reduce_add_sync(kAllLanes, mine.n)};
    mine = none;
    Run open = none, closed = none;
    uint32_t q = walk.q, closed_q = 0;
    uint64_t from = 0, next = 0, closed_from = 0;
    bool cut = false, pending = false;  // one ended here; its start is in another lane's tokens
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (t + i >= stop || t + i < first) continue;
      if (t + i >= next) {
        q = sequence_of(s.off, q, ahead.q + 1, t + i);
        from = s.off[q];
        next = s.off[q + 1];
      }
      if (bits >> i & 1u) run_add(open, l4[i], r4[i]);
      if (t + i + 1 == next) {
        if (!cut && from < t) {
          closed = open;
          closed_q = q;
          closed_from = from;
          pending = true;
        } else {
          emit(q, from, open);
        }
        cut = true;
        open = none;
      }
    }
    // what comes into each lane from those before it, since the last end
    Run incl = open;
    bool c = cut;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Run y = run_up(incl, o);
      const bool yc = __shfl_up_sync(kAllLanes, c, o);
      if (lane >= o && !c) {
        incl = run_join(y, incl);
        c = yc;
      }
    }
    Run into = run_up(incl, 1);
    bool into_cut = __shfl_up_sync(kAllLanes, c, 1);
    if (lane == 0) {
      into = none;
      into_cut = false;
    }
    if (pending) {
      if (!into_cut) into = run_join(carry, into);
      emit(closed_q, closed_from, run_join(into, closed));
    }
    if (lane == 31) mine = c ? incl : run_join(carry, incl);
    walk = ahead;
    // on to what the next tile starts in; past the last sequence there is none
    if (t0 + kTile < stop) walk.to(s.off, n_seq, t0 + kTile);
    start = s.off[walk.q];
    after = end_after(walk.q);
  }
  // the sequence that the run leaves open
  if (walk.q < n_seq && start < stop && walk.next > stop) {
    const Run all{warp_join(mine.v), __reduce_add_sync(kAllLanes, mine.n)};
    if (lane == 0) emit(walk.q, start, all);
  }
}

// What another thread of the call wrote: in shared memory (LOCAL: of one CTA), or read
// around the first-level cache.
template <bool LOCAL, typename V>
__device__ __forceinline__ V fresh(const V *p) {
  if constexpr (LOCAL) return *p;
  else return __ldcg(p);
}

// A sequence's sum and its number of tokens.
struct SeqSum {
  Pair v;
  uint64_t n;
};
template <bool LOCAL>
__device__ __forceinline__ SeqSum sequence_sum(const TokenSet &s, const PrefScratch &x, uint64_t seq) {
  const uint64_t a = s.off[seq], b = min(s.off[seq + 1], s.n);
  if (b <= a) return {{0.f, 0.f}, 0};
  const float4 p = fresh<LOCAL>(reinterpret_cast<const float4 *>(&x.inner[seq]));
  SeqSum r{{p.x, p.y}, __float_as_uint(p.z)};
  const uint64_t last = (b - 1) / x.run;
#pragma unroll 4
  for (uint64_t c = a / x.run + 1; c <= last; ++c) {
    const float4 h = fresh<LOCAL>(reinterpret_cast<const float4 *>(&x.head[c]));
    r = SeqSum{pair_join(r.v, Pair{h.x, h.y}), r.n + __float_as_uint(h.z)};
  }
  return r;
}

constexpr float kHiUnit = 1.f / 1048576.f;              // 2^-20
constexpr float kLoUnit = 1.f / 4611686018427387904.f;  // 2^-62
constexpr float kGradMost = 4194304.f;                  // 2^22

// x / n for a whole number n
__device__ __forceinline__ df df_over(df x, uint64_t n) {
  const float nh = (float)n, nl = (float)((long long)n - (long long)nh);
  const float q = x.hi / nh;
  const float rest = fmaf(-q, nl, fmaf(-q, nh, x.hi)) + x.lo;
  return isfinite(q) ? quick_two_sum(q, rest / nh) : df{q, 0.f};
}

__device__ __forceinline__ void grad_add(const PrefScratch &x, uint64_t seq, df v) {
  if (!(fabsf(v.hi) < kGradMost)) {
    x.bad[seq] = 1u;  // every writer writes the same
    return;
  }
  const float h = rintf(v.hi * (1.f / kHiUnit));  // all of this is exact but for
  const float rest = fmaf(-h, kHiUnit, v.hi);     // the roundings to whole units
  const long long lo = __float2ll_rn(rest * (1.f / kLoUnit)) + __float2ll_rn(v.lo * (1.f / kLoUnit));
  if (h != 0.f) atomicAdd(&x.grad[seq].hi, (unsigned long long)__float2ll_rn(h));
  if (lo) atomicAdd(&x.grad[seq].lo, (unsigned long long)lo);
}

// Pairs first, first + step, ...: their losses, gradients and sums.
template <bool LOCAL>
__device__ __forceinline__ void take_pairs(const PrefIn &in, const PrefRule &r,
                                           const PrefScratch &x, const PrefOut &out,
                                           uint32_t first, uint32_t step, Pair (&sum)[4],
                                           Ctrl *ctrl) {
  for (uint64_t i = first; i < in.n_pair; i += step) {
    const int64_t c = in.pair[2 * i], j = in.pair[2 * i + 1];
    float l = 0.f;
    if ((uint64_t)c >= in.s.n_seq || (uint64_t)j >= in.s.n_seq) {
      flag(ctrl, DEVERR_INDEX, (unsigned long long)((uint64_t)c >= in.s.n_seq ? c : j));
    } else {
      const SeqSum rc = sequence_sum<LOCAL>(in.s, x, c), rj = sequence_sum<LOCAL>(in.s, x, j);
      df uc = as_df(rc.v), uj = as_df(rj.v);
      if (r.average) {
        if (rc.n) uc = df_over(uc, rc.n);
        if (rj.n) uj = df_over(uj, rj.n);
      }
      const df h = as_df(pair_join(Pair{uc.hi, uc.lo}, Pair{-uj.hi, -uj.lo}));
      const df bh = df_mul(h, r.beta);
      const float d = isfinite(bh.hi) ? df_add(bh, df{-r.margin.hi, -r.margin.lo}).hi : h.hi;
      df g;  // by u of the chosen
      if (r.kind == EDP_PREF_LOGISTIC) {
        const float e = expf(-fabsf(d)), tail = log1pf(e);  // tail = -ln s(|d|)
        const float up = tail + fmaxf(-d, 0.f), down = tail + fmaxf(d, 0.f);
        l = r.smooth == 0.f ? up : fmaf(1.f - r.smooth, up, r.smooth * down);
        // s(-d) (1 - e) - s(d) e = s(-d) - e
        const float sd = d > 0.f ? e / (1.f + e) : 1.f / (1.f + e);
        g = df{-r.beta.hi * (sd - r.smooth), 0.f};
      } else if (r.kind == EDP_PREF_HINGE) {
        const df y = df_add(df_add(df{1.f, 0.f}, r.margin), df{-bh.hi, -bh.lo});
        l = y.hi > 0.f ? y.hi : isnan(d) ? d : d < 0.f ? -d : 0.f;
        g = y.hi > 0.f ? df{-r.beta.hi, -r.beta.lo} : df{0.f, 0.f};
      } else {
        const df y = df_add(h, df{-r.half.hi, -r.half.lo});
        l = isfinite(h.hi) ? y.hi * y.hi : h.hi * h.hi;
        g = df{2.f * y.hi, 2.f * y.lo};
      }
      if (!isfinite(h.hi)) g = r.kind == EDP_PREF_SQUARE || isnan(d) ? df{h.hi, 0.f} : g;
      grad_add(x, c, r.average && rc.n ? df_over(g, rc.n) : g);
      const df m{-g.hi, -g.lo};
      grad_add(x, j, r.average && rj.n ? df_over(m, rj.n) : m);
      pair_add(sum[0], l);
      if (h.hi > 0.f) pair_add(sum[1], 1.f);
      const df bc = df_mul(uc, r.beta), bj = df_mul(uj, r.beta);
      pair_add(sum[2], isfinite(bc.hi) ? bc.hi : uc.hi);
      if (isfinite(bc.hi)) pair_add(sum[2], bc.lo);
      pair_add(sum[3], isfinite(bj.hi) ? bj.hi : uj.hi);
      if (isfinite(bj.hi)) pair_add(sum[3], bj.lo);
    }
    if (out.pair_loss) out.pair_loss[i] = l;
  }
}

template <bool LOCAL>
__device__ __forceinline__ void take_ratios(const PrefIn &in, const PrefRule &r,
                                            const PrefScratch &x, const PrefOut &out,
                                            uint64_t first, uint64_t step) {
  if (!out.ratio) return;
  for (uint64_t q = first; q < in.s.n_seq; q += step) {
    const SeqSum v = sequence_sum<LOCAL>(in.s, x, q);
    const df u = as_df(v.v);
    out.ratio[q] = r.average && v.n ? df_over(u, v.n).hi : u.hi;
  }
}

// An output by each of four threads.
__device__ __forceinline__ void write_loss(const PrefRule &r, const Pair *total, float *loss) {
  if (threadIdx.x >= 4) return;
  const df v = as_df(total[threadIdx.x]), by = threadIdx.x ? r.per_pair : r.per_norm;
  loss[threadIdx.x] = isfinite(v.hi) ? df_mul(v, by).hi : v.hi;
}

// The gradient of each token of a sequence, rounded once.
template <bool LOCAL>
__device__ __forceinline__ float token_grad(const PrefScratch &x, uint32_t seq, df scale) {
  if (fresh<LOCAL>(&x.bad[seq])) return __int_as_float(0x7fc00000);
  const ulonglong2 g = fresh<LOCAL>(reinterpret_cast<const ulonglong2 *>(&x.grad[seq]));
  // what is whole units of 2^-20 in lo goes to hi, so that neither cancels much
  const long long up = ((long long)g.y + (1ll << 41)) >> 42;
  const long long whole = (long long)g.x + up;
  const float h = (float)whole, rest = (float)(whole - (long long)h);
  const float vh = h * kHiUnit;
  const float vl = fmaf(rest, kHiUnit, (float)((long long)g.y - (up << 42)) * kLoUnit);
  return fmaf(scale.hi, vh, fmaf(scale.hi, vl, scale.lo * vh));
}

// Gradients of tokens [begin, stop) of a warp.
template <bool VEC, bool LOCAL>
__device__ __forceinline__ void run_grad(const PrefIn &in, const PrefScratch &x, df scale,
                                         float *dlogp, uint64_t begin, uint64_t stop,
                                         uint64_t first, uint64_t end, bool wait) {
  const TokenSet &s = in.s;
  const uint32_t n_seq = (uint32_t)s.n_seq;
  const int lane = threadIdx.x & 31;
  stop = min(stop, s.n);
  SeqWalk walk;
  uint64_t after = 0;           // where the sequence after the walk's ends
  float here = 0.f, there = 0.f;  // gradients of both
  bool known = false;
  if (begin < min(stop, end)) walk.start(s.off, n_seq, begin);
  if (wait) pdl_wait();  // for the gradients: the offsets and the mask are inputs
  for (uint64_t t0 = begin; t0 < stop;) {
    const uint64_t t = t0 + 4 * lane;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (t0 < end) {
      if (!known || t0 >= walk.next) {
        if (known && after > t0) {
          ++walk.q;
          walk.next = after;
          here = there;
        } else {
          if (known) walk.to(s.off, n_seq, t0);
          here = token_grad<LOCAL>(x, walk.q, scale);
        }
        known = true;
        // and what will be wanted at its end
        const bool more = walk.q + 1 < n_seq;
        after = more ? s.off[walk.q + 2] : walk.next;
        there = more ? token_grad<LOCAL>(x, walk.q + 1, scale) : 0.f;
      }
      // tiles within the sequence, kAtOnce of them in flight
      const uint64_t top = min(walk.next, min(stop, end)), room = top > t0 ? top - t0 : 0;
      if (VEC && t0 >= first && room >= kTile) {
        const uint32_t m = (uint32_t)min(room / kTile, (uint64_t)kAtOnce);
        uint32_t mk[kAtOnce];
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k)
          mk[k] = s.mask && k < m ? *reinterpret_cast<const uint32_t *>(s.mask + t + k * kTile)
                                  : 0xffffffffu;
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k)
          if (k < m)
            *reinterpret_cast<float4 *>(dlogp + t + k * kTile) =
                make_float4(mk[k] & 0xffu ? here : 0.f, mk[k] & 0xff00u ? here : 0.f,
                            mk[k] & 0xff0000u ? here : 0.f, mk[k] & 0xff000000u ? here : 0.f);
        t0 += m * kTile;
        continue;
      }
      const uint32_t bits = token_bits<VEC>(s, t, first, end);
      if (t0 + kTile <= after || after >= end) {  // two sequences
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] = !(bits >> i & 1u) ? 0.f : t + i < walk.next ? here : there;
      } else {
        SeqWalk to = walk;
        to.to(s.off, n_seq, min(t0 + kTile, end) - 1);
        uint32_t q = walk.q;
        uint64_t next = 0;
        float each = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!(bits >> i & 1u)) continue;
          if (t + i >= next) {
            q = sequence_of(s.off, q, to.q + 1, t + i);
            next = s.off[q + 1];
            each = token_grad<LOCAL>(x, q, scale);
          }
          v[i] = each;
        }
      }
    }
    store4<VEC>(dlogp, t, s.n, make_float4(v[0], v[1], v[2], v[3]));
    t0 += kTile;
  }
}

template <bool VEC>
__global__ void __launch_bounds__(kThreads, kPerSm)
k_pref_parts(PrefIn in, PrefScratch x) {
  pdl_wait();
  pdl_launch();
  const uint64_t first = in.s.off[0], end = min(in.s.off[in.s.n_seq], in.s.n);
  const uint64_t begin = ((uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * x.run;
  run_parts<VEC>(in, x, begin, begin + x.run, first, end);
}

__global__ void __launch_bounds__(kPairThreads)
k_pref_pairs(PrefIn in, PrefRule r, PrefScratch x, PrefOut out, uint32_t pair_ctas, Ctrl *ctrl) {
  __shared__ Pair total[4];
  pdl_wait();
  pdl_launch();
  Pair sum[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = Pair{0.f, 0.f};
  if (blockIdx.x < pair_ctas)
    take_pairs<false>(in, r, x, out, blockIdx.x * kPairThreads + threadIdx.x, pair_ctas * kPairThreads,
               sum, ctrl);
  else
    take_ratios<false>(in, r, x, out, (blockIdx.x - pair_ctas) * kPairThreads + threadIdx.x,
                (uint64_t)(gridDim.x - pair_ctas) * kPairThreads);
  if (grid_join<kPairThreads, 4>(sum, total, x.part, &ctrl->loss_ticket))
    write_loss(r, total, out.loss);
}

template <bool VEC>
__global__ void __launch_bounds__(kThreads, kGradPerSm)
k_pref_grad(PrefIn in, PrefScratch x, df scale, uint32_t run, float *dlogp) {
  // behind k_pref_pairs, whose call waited for all that came before it
  pdl_launch();
  const uint64_t first = in.s.off[0], end = min(in.s.off[in.s.n_seq], in.s.n);
  const uint64_t begin = ((uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * run;
  run_grad<VEC, false>(in, x, scale, dlogp, begin, begin + run, first, end, true);
}

// All three steps of a batch of up to 8,192 tokens, one or two tiles per warp (run:
// tokens), and up to kSmallSeqs sequences, whose offsets, sums and gradients stay in
// shared memory.
template <bool VEC>
__global__ void __launch_bounds__(kSmallThreads)
k_pref_small(PrefIn in, PrefRule r, PrefOut out, df scale, uint32_t run, Ctrl *ctrl) {
  __shared__ uint64_t off[kSmallSeqs + 1];
  __shared__ SeqPart inner[kSmallSeqs], head[kSmallThreads / 32];
  __shared__ alignas(16) SeqGrad grad[kSmallSeqs];
  __shared__ uint32_t bad[kSmallSeqs];
  __shared__ Pair total[4];
  const PrefScratch x{inner, head, grad, bad, nullptr, run};
  pdl_wait();
  pdl_launch();
  // one round trip for the offsets, which every search goes to
  for (uint32_t q = threadIdx.x; q <= in.s.n_seq; q += kSmallThreads) off[q] = in.s.off[q];
  __syncthreads();
  in.s.off = off;
  const uint64_t first = in.s.off[0], end = min(in.s.off[in.s.n_seq], in.s.n);
  const uint64_t begin = (uint64_t)(threadIdx.x >> 5) * x.run;
  run_parts<VEC>(in, x, begin, begin + x.run, first, end);
  __syncthreads();
  Pair sum[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = Pair{0.f, 0.f};
  constexpr uint32_t kHalf = kSmallThreads / 2;  // the ratios by warps of their own
  if (threadIdx.x < kHalf) take_pairs<true>(in, r, x, out, threadIdx.x, kHalf, sum, ctrl);
  else take_ratios<true>(in, r, x, out, threadIdx.x - kHalf, kHalf);
  // the barriers of the join order the CTA's gradients before their use
  if (grid_join<kSmallThreads, 4>(sum, total, x.part, &ctrl->loss_ticket))
    write_loss(r, total, out.loss);
  if (out.dlogp)
    run_grad<VEC, true>(in, x, scale, out.dlogp, begin, begin + x.run, first, end, false);
}

}  // namespace

cudaError_t launch_preference_loss(edp_ctx *c, const edp_preference_config &cfg,
                                   const TokenSet &set, const float *logp, const float *ref,
                                   const int64_t *pair, uint32_t n_pair, float *loss,
                                   float *ratio, float *pair_loss, float *dlogp,
                                   cudaStream_t s) {
  const uint64_t sms = (uint64_t)c->coop_sms;
  const bool small = set.n <= kSmallRun * (kSmallThreads / 32) && n_pair <= kSmallPairs &&
                     set.n_seq <= kSmallSeqs;
  PrefRule r;
  auto both = [](double v) {
    const float hi = (float)v;
    return df{hi, (float)(v - (double)hi)};
  };
  r.beta = both(cfg.beta);
  r.smooth = (float)cfg.label_smoothing;
  r.margin = both(cfg.margin);
  r.half = both(0.5 / cfg.beta);
  const double norm = cfg.norm > 0.0 ? cfg.norm : (double)n_pair;
  r.per_norm = both(1.0 / norm);
  r.per_pair = both(1.0 / (double)n_pair);
  const df scale = both(cfg.grad_scale / norm);
  r.kind = cfg.kind;
  r.average = cfg.average;
  const PrefIn in{set, logp, ref, pair, n_pair};
  const PrefOut out{loss, ratio, pair_loss, dlogp};
  const bool vec = (((uintptr_t)logp | (uintptr_t)ref | (uintptr_t)dlogp) & 15) == 0 &&
                   ((uintptr_t)set.mask & 3) == 0;
  if (small)
    return launch_pdl(vec ? k_pref_small<true> : k_pref_small<false>, dim3(1),
                      dim3(kSmallThreads), s, in, r, out, scale,
                      set.n <= 4 * kSmallThreads ? kTile : kSmallRun, c->ctrl);
  // a run per warp of a full chip, so that all end together
  const uint64_t warps = kThreads / 32;
  auto run_of = [&](uint64_t per_sm) {
    const uint64_t chip = per_sm * warps * sms, each = (set.n + chip - 1) / chip;
    return (each + kTile - 1) / kTile * kTile;
  };
  const uint64_t run = run_of(kPerSm), grad_run = run_of(kGradPerSm);
  const uint64_t runs = (set.n + run - 1) / run;
  auto ctas = [&](uint64_t n) {
    const uint64_t want = (n + kPairThreads - 1) / kPairThreads;
    return (uint32_t)(want < 4 * sms ? want : 4 * sms);
  };
  const uint32_t pair_ctas = ctas(n_pair), pair_grid = pair_ctas + (ratio ? ctas(set.n_seq) : 0);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t a = at;
    at += (bytes + 15) & ~(size_t)15;
    return a;
  };
  const size_t inner = take(set.n_seq * sizeof(SeqPart)), grad = take(set.n_seq * sizeof(SeqGrad));
  const size_t head = take(runs * sizeof(SeqPart)), bad = take(set.n_seq * sizeof(uint32_t));
  const size_t part = take(4 * pair_grid * sizeof(Pair));
  void *blk = nullptr;
  cudaError_t e = ctx_scratch(c, at, s, &blk);
  if (e != cudaSuccess) return e;
  uint8_t *b = (uint8_t *)blk;
  const PrefScratch x{(SeqPart *)(b + inner), (SeqPart *)(b + head), (SeqGrad *)(b + grad),
                      (uint32_t *)(b + bad), (Pair *)(b + part), (uint32_t)run};
  const unsigned grid = (unsigned)((runs + warps - 1) / warps);
  e = launch_pdl(vec ? k_pref_parts<true> : k_pref_parts<false>, dim3(grid), dim3(kThreads), s, in,
                 x);
  if (e != cudaSuccess) return e;
  e = launch_pdl(k_pref_pairs, dim3(pair_grid), dim3(kPairThreads), s, in, r, x, out, pair_ctas,
                 c->ctrl);
  if (e != cudaSuccess || !dlogp) return e;
  const uint64_t grads = (set.n + grad_run - 1) / grad_run;
  return launch_pdl(vec ? k_pref_grad<true> : k_pref_grad<false>,
                    dim3((unsigned)((grads + warps - 1) / warps)), dim3(kThreads), s, in, x, scale,
                    (uint32_t)grad_run, dlogp);
}

}  // namespace edp
