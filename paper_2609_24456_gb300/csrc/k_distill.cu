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
// are taken out of the row before its sums, which then are those of the rest; the entries
// join them afterwards.
//
// With the gradient a row is read once, into the shared memory of a cluster, and its gradient
// written once (k_distill); without it the row is streamed (k_distill_stream).  What takes
// time besides the copies is made beside them, where it can be: a thread per entry reads the
// list and sums what does not need the row.  The sums are relative to the list's maximum,
// known by then (with a running maximum: 808 us where it now takes 761).
//
// What bounds it, at 6.79 TB/s of measured copy:
//   8,192 x 152,064 bf16, 64 entries, a tenth masked   761 us   697 us to read and write once
//   4,096 x 152,064 f16, 32 entries                    395 us   367 us
//   2,048 x 152,064 bf16, the loss alone               107 us   92 us to read once
//   515 x 32,003 f32, 100 entries, mixed              32.5 us   17.5 us: 2.3 waves of CTAs, whose
//                                                               copies and sums hardly overlap
//   16 x 32,003 bf16, 20 entries                       7.6 us   in a graph: a chain of loads (mask,
//                                                               entry, its logit), one copy, the
//                                                               cluster's join
#include <cmath>

#include "edp_stream.cuh"

namespace edp {
namespace {

// threads per SM, which bound the registers: three CTAs of 384, as parts of 76 KB allow
constexpr int kLanes = 1152;
constexpr uint32_t kTwoParts = 112 * 1024;  // bytes of a part, two of which fit an SM

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

constexpr float kNaN = __builtin_nanf("");

// NaN apart, which it is of NaN alone
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kAllLanes, x, o));
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

// Two numbers of each thread with an entry over all of them, in all threads.
__device__ __forceinline__ float2 list_sums(float x, float y, bool busy, uint32_t warps,
                                            float2 *room) {
  if (busy) {
    x = warp_add(x);
    y = warp_add(y);
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = make_float2(x, y);
  }
  __syncthreads();
  float2 a = room[0];
  for (uint32_t i = 1; i < warps; ++i) {
    a.x += room[i].x;
    a.y += room[i].y;
  }
  return a;
}

// A thread's entry of a row's list; id < 0: none.
struct Entry {
  int32_t id;
  float lp, p;  // the teacher's log-probability and probability
  float x, e;   // the student's logarithm relative to the list's maximum, and its power
};
// What does not need the row's sums, made while the row is on its way: the list's maximum,
// the sums of e, of p, and of p (lp - x) with FORWARD or of e (x - lp) with REVERSE.
// bad: NaN where the teacher has NaN or +infinity, which a student's q of 0 would hide, else 0.
struct ListSums {
  float m, s, p, cross, bad;
};
// NaN in the place of +infinity, which is no logarithm of a probability either.
__device__ __forceinline__ float teacher_log(float x) {
  return x < __builtin_huge_valf() ? x : kNaN;
}
// Of the whole row: its logarithms' normaliser relative to the list's maximum, what takes e
// to q; the others' q and its logarithm, their maximum and sum.
struct RowSums {
  float ln, by, qr, lqr, m, s;
  bool none;  // no token has a probability
};
__device__ __forceinline__ RowSums row_sums(const ListSums &l, const RowSum &o, float c,
                                            float inv_t) {
  const float M = fmaxf(l.m, o.m);
  const float to_row = l.m == kNegInf ? 1.f : ex2((l.m - M) * c);
  const float left = o.m == kNegInf ? o.s : o.s * ex2((o.m - M) * c);
  const float sum = fmaf(l.s, to_row, left), S = sum + l.bad, ln = logf(S), inv = 1.f / S;
  return {ln + (M - (l.m == kNegInf ? 0.f : l.m)) * inv_t,
          to_row * inv,
          left * inv,
          o.s == 0.f ? kNegInf : (o.m - M) * inv_t + logf(o.s) - ln,
          o.m,
          o.s,
          M == kNegInf && sum == sum};
}
// The row's loss, the others' gradient and `g`, by which an entry's goes, before the weight.
struct RowLoss {
  float loss, outside, g;
};
// FORWARD and REVERSE.
__device__ __forceinline__ RowLoss row_loss_of(uint32_t kind, const ListSums &l, const RowSums &r,
                                               float lpr, float pr) {
  if (kind == EDP_DISTILL_FORWARD) {
    const float P = l.p + pr;
    return {fmaf(l.p, r.ln, l.cross) + weigh(pr, lpr - r.lqr), fmaf(P, r.qr, -pr), P};
  }
  const float all = r.by * fmaf(-l.s, r.ln, l.cross) + weigh(r.qr, r.lqr - lpr);
  // where the teacher excludes what the student does not, an infinite loss has no gradient
  const float g = fmaf(0.f, all, all);
  return {all, weigh(r.qr, r.lqr - lpr - g), g};
}

// An entry as the list has it; asked for before anything else of the row is known.
__device__ __forceinline__ Entry load_entry(const TeacherLists &lists, uint64_t t) {
  Entry e{-1, kNaN, 0.f, kNegInf, 0.f};
  if (threadIdx.x < lists.top) {
    const uint64_t at = t * lists.top + threadIdx.x;
    e.id = lists.ids[at];
    e.lp = lists.value[at];
  }
  return e;
}

// Shared memory of the list's phase.
struct ListRoom {
  float2 sums[4][4];  // of list_sums, of each call its own
  float weight;
  int32_t strange;    // an id >= vocab, or -1 (set before)
};
// The row's weight by the last warp, the list by a thread per entry (the first 128).  Every
// logit of it is here when the function returns, and so is the weight.
template <typename T, int NT>
__device__ __forceinline__ ListSums read_list(const RowArgs &a, const RowWeights &weights,
                                              bool by_range, const TeacherLists &lists,
                                              const DistillRule &rule, const T *row, uint64_t t,
                                              float pr, Entry *entry, ListRoom *s) {
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const uint32_t warps = (lists.top + 31) / 32;
  const bool busy = wid < warps, has_rest = lists.rest != nullptr;
  Entry e = *entry;
  ListSums l{kNegInf, 0.f, 0.f, 0.f, 0.f};
  if (busy) {
    if (e.lp == kNegInf) e.id = -1;
    if (e.id >= 0) e.lp = teacher_log(e.lp);
    if (e.id >= 0 && (uint32_t)e.id >= a.vocab) {
      s->strange = e.id;
      e.id = -1;
    }
    const float z = e.id >= 0 ? to_f32(row[e.id]) : kNegInf;
    e.x = z;
    // v: NaN where there are no entries and NaN is all that the list has, which is how
    // edp_token_top marks the row of a teacher that went wrong
    const float m = warp_max(z), v = warp_max(e.id >= 0 || e.lp != e.lp ? e.lp : kNegInf);
    if (lane == 0) s->sums[0][wid] = make_float2(m, v);
  }
  if (wid == NT / 32 - 1) {
    float w;
    if (by_range) {
      const Range r = token_range(weights.set);
      w = 1.f / (float)(r.end - r.first);
    } else {
      w = row_weight(weights, t);
    }
    if (lane == 0) s->weight = w;
  }
  __syncthreads();
  float top_value = kNaN;
  for (uint32_t i = 0; i < warps; ++i) {
    l.m = fmaxf(l.m, s->sums[0][i].x);
    top_value = fmaxf(top_value, s->sums[0][i].y);
  }
  if (busy) {
    const float y = e.x - (l.m == kNegInf ? 0.f : l.m);
    e.e = e.id >= 0 ? ex2(y * a.c) : 0.f;
    e.x = y * a.inv_t;
    if (!has_rest) e.lp = (e.lp - top_value) * rule.inv_tt;  // the list's own softmax
    e.p = e.id >= 0 ? expf(e.lp) : 0.f;
  }
  float2 sums = list_sums(e.e, e.p, busy, warps, s->sums[1]);
  l.s = sums.x;
  l.p = sums.y;
  if (!has_rest && busy) {
    e.lp -= logf(l.p);
    e.p = e.id >= 0 ? expf(e.lp) : 0.f;
  }
  if (rule.kind != EDP_DISTILL_MIX) {
    const float cross = rule.kind == EDP_DISTILL_FORWARD ? weigh(e.p, e.lp - e.x)
                                                         : weigh(e.e, e.x - e.lp);
    sums = list_sums(e.id >= 0 ? cross : 0.f, e.p, busy, warps, s->sums[2]);
    l.cross = sums.x;
    l.p = sums.y;
  }
  const float all = l.p + pr;
  if (all != all || top_value != top_value) l.bad = kNaN;
  *entry = e;
  return l;
}
// MIX, by all threads; lm: the entry's ln m.
__device__ __forceinline__ RowLoss mix_loss(const DistillRule &rule, const TeacherLists &lists,
                                            const Entry &e, const RowSums &r, float lpr, float pr,
                                            ListRoom *s, float *lm) {
  const uint32_t warps = (lists.top + 31) / 32;
  const bool busy = threadIdx.x < 32 * warps;
  const float lq = e.x - r.ln, q = e.e * r.by;
  float x = 0.f, y = 0.f;
  if (busy) {
    *lm = log_add(e.lp + rule.ln_beta, lq + rule.ln_alpha);
    if (e.id >= 0) {
      x = weigh(rule.beta * e.p, e.lp - *lm);
      y = weigh(rule.alpha * q, lq - *lm);
    }
  }
  const float2 sums = list_sums(x, y, busy, warps, s->sums[3]);
  const float lmr = log_add(lpr + rule.ln_beta, r.lqr + rule.ln_alpha);
  const float g = sums.y + weigh(rule.alpha * r.qr, r.lqr - lmr);
  return {sums.x + weigh(rule.beta * pr, lpr - lmr) + g,
          weigh(r.qr, fmaf(rule.alpha, r.lqr - lmr, -g)), g};
}

// The gradient of the tokens outside of the list: a factor of their 2^y.  Without a finite
// logit among them there is no maximum to be relative to, and each 2^y is 0 (whose product
// with NaN is NaN).
__device__ __forceinline__ RowGrad others_grad(const RowSums &r, const RowLoss &f, float by) {
  return {r.m == kNegInf ? 0.f : r.m,
          r.s == 0.f && f.outside == f.outside ? 0.f : by * (f.outside / r.s), 0.f, 0.f};
}
// An entry's, before the weight.
__device__ __forceinline__ float entry_grad(const DistillRule &rule, const Entry &e,
                                            const RowSums &r, const RowLoss &f, float lm) {
  const float q = e.e * r.by;
  if (f.g != f.g) return f.g;  // (a weight of 0 would hide it)
  if (rule.kind == EDP_DISTILL_FORWARD) return fmaf(f.g, q, -e.p);
  if (rule.kind == EDP_DISTILL_REVERSE) return weigh(q, e.x - r.ln - e.lp - f.g);
  return weigh(q, fmaf(rule.alpha, e.x - r.ln - lm, -f.g));
}

// The weighted loss of a row, from one CTA of each row; the last of them adds up all
// rows in a fixed order and leaves the counters at 0.
template <int NT>
__device__ __forceinline__ void conclude(float weighted, float *per_row, float *loss,
                                         Ctrl *ctrl) {
  constexpr int NW = NT / 32;
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
  for (uint32_t i = threadIdx.x; i < gridDim.x; i += NT) pair_add(a, __ldcg(per_row + i));
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
template <typename T, int NT>
__global__ void __launch_bounds__(NT, kLanes / NT)
k_distill(RowArgs a, RowWeights weights, bool by_range, TeacherLists lists, DistillRule rule,
          float *loss, float *row_loss, float *per_row, void *dz, uint64_t dstride, bool early,
          Ctrl *ctrl) {
  constexpr bool F = kFused<T>;
  using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
  extern __shared__ uint4 resident[];
  __shared__ RowSum red[NT / 32];
  __shared__ float4 parts[2][8];  // what the cluster's CTAs send: m, S, -, a token twice
  __shared__ ListRoom list;
  __shared__ RowSums rows;        // what the first warp makes of them
  __shared__ RowLoss found;
  __shared__ bool twice, zero, careful;
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
    list.strange = -1;
    twice = false;
  }
  __syncthreads();
  // early: the kernel before is of this call, waited for all that came before it and
  // writes the weights alone
  if (!early) pdl_wait();
  pdl_launch();
  Entry e = load_entry(lists, t);
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  T *d = reinterpret_cast<T *>(dz) + t * dstride + first;
  if ((a.mask && !a.mask[t]) || !in_sequences(weights, t)) {
    part_zero<T, NT>(d, n);
    if (early) pdl_wait();  // so that what waits for this kernel finds the weights
    if (part) return;
    if (row_loss && threadIdx.x == 0) row_loss[t] = 0.f;
    conclude<NT>(0.f, per_row, loss, ctrl);
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
  // Beside the copy: the row's weight and its list (its logits in other parts, too: they are
  // here before this CTA's message leaves, and only then may another write its gradient in
  // their place, or set back the count behind the weight).
  if (early) pdl_wait();
  const float lpr = lists.rest ? teacher_log(lists.rest[t]) : kNegInf,
              pr = lists.rest ? expf(lpr) : 0.f;
  const ListSums l = read_list<T, NT>(a, weights, by_range, lists, rule, row, t, pr, &e, &list);
  if (sp.vecs && !mbar_wait(&bar, 0, kRowWaitNs)) {
    if (threadIdx.x == 0) flag(ctrl, DEVERR_TIMEOUT, t);
    mbar_wait(&bar, 0, kRowWaitNs);  // bounded: the copy lands before the CTA ends
  }
  // Each entry leaves its number in its place, looks whether it is still there (-infinity is
  // no entry's number), and takes itself out of the row.
  const bool here = e.id >= 0 && (uint32_t)e.id - first < n;
  Bits *place = reinterpret_cast<Bits *>(held) + (here ? (uint32_t)e.id - first : 0);
  if (here) *place = (Bits)threadIdx.x;
  __syncthreads();
  if (here) {
    if (*place != (Bits)threadIdx.x) twice = true;
    held[(uint32_t)e.id - first] = from_f32<T>(kNegInf);
  }
  __syncthreads();
  // The first warp joins the CTA's sums, gives them to the cluster's other CTAs and takes
  // theirs.
  auto join = [&](bool near, int round) {
    const bool has = lane < NT / 32;
    RowSum sum = warp_sum<T, false, lanes_for(NT / 32)>(
        has ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, a.c);
    bool all = true, again = twice;
    if (np > 1) {
      const float4 mine = make_float4(__shfl_sync(kAllLanes, sum.m, 0),
                                      __shfl_sync(kAllLanes, sum.s, 0), 0.f, again ? 1.f : 0.f);
      if (lane < np) send_float4(&parts[round][part], mine, &sent[round], lane);
      if (!mbar_wait(&sent[round], 0, kRowWaitNs)) {
        if (lane == 0) flag(ctrl, DEVERR_TIMEOUT, t);
        all = mbar_wait(&sent[round], 0, kRowWaitNs);  // none of them comes after the end
      }
      all = __all_sync(kAllLanes, all);
      const float4 x = lane < np ? parts[round][lane] : make_float4(kNegInf, 0.f, 0.f, 0.f);
      again = __any_sync(kAllLanes, x.w != 0.f);
      sum = warp_sum<T, false, 8>(RowSum{x.x, x.y, 0.f}, a.c);
    }
    if (near) sum = exact_sums<T>(sum, a.c);
    const RowSums r = row_sums(l, sum, a.c, a.inv_t);
    const RowLoss f = rule.kind == EDP_DISTILL_MIX ? RowLoss{}
                                                   : row_loss_of(rule.kind, l, r, lpr, pr);
    if (lane) return;
    careful = near && !(sum.s >= kLeastSum && sum.s <= kMostSum);
    rows = r;
    found = f;
    twice = again;
    zero = r.none || list.strange >= 0 || again || !all;
  };
  auto whole_row = [&](const RowSum &sum, bool near, int round) {
    if (lane == 0) red[wid] = sum;
    if (np > 1 && round == 0) cluster_wait();  // every CTA has started: its shared memory is there
    __syncthreads();
    if (wid == 0) join(near, round);
    __syncthreads();
  };
  // Relative to the list's maximum, which is near the row's, most likely; a sum that is far
  // from 1 that way is made again relative to each thread's own.  (The gradient's factor of
  // 2^y is divided by it: in a mean over 8,192 rows it would be below fp32's least normal
  // number from 2^113 on.)
  const bool near = fabsf(l.m) < __builtin_huge_valf() && (!F || sums_hold(l.m, a.c));
  whole_row(near ? warp_sum<T, false>(
                       RowSum{l.m, part_sum_near<T, F, NT>(held, n, RowLog<T, F>(l.m, a.c)), 0.f},
                       a.c)
                 : RowSum{kNegInf, 0.f, 0.f}, near, 0);
  if (!near || careful)
    whole_row(warp_sum<T, false>(part_sum<T, false, false, NT>(held, n, a.c), a.c), false, 1);
  const RowSums r = rows;
  RowLoss f = found;
  float lm = 0.f;
  if (rule.kind == EDP_DISTILL_MIX) f = mix_loss(rule, lists, e, r, lpr, pr, &list, &lm);
  if (part == 0 && threadIdx.x == 0) {
    if (list.strange >= 0)
      flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)list.strange);
    if (twice) flag(ctrl, DEVERR_TWICE, t);
    if (r.none) flag(ctrl, DEVERR_ROW, t);
    if (row_loss) row_loss[t] = zero ? 0.f : f.loss;
  }
  if (zero) {
    part_zero<T, NT>(d, n);
  } else {
    const float by = rule.grad_scale * list.weight * a.inv_t;
    part_grad_any<T, false, NT>(held, d, n, n, others_grad(r, f, by), a.c);
    __syncthreads();  // before the entries take their places
    if (here) d[(uint32_t)e.id - first] = from_f32<T>(by * entry_grad(rule, e, r, f, lm));
  }
  if (part == 0) conclude<NT>(zero ? 0.f : list.weight * f.loss, per_row, loss, ctrl);
}

// The loss alone: the row is streamed, and read once too.  BACK: its gradient, with the
// logits read a second time, for rows of which too little fits shared memory.  A vector with
// an entry in it is left out of the sums; the first of its entries adds what else there is in
// it.  All is relative to the list's maximum (no maximum is kept), which is near the row's,
// most likely: a part whose sum is far from 1 is summed again relative to its own.
template <typename T, int NT, int ST, bool BACK, bool LONG>
__global__ void __launch_bounds__(NT, kStreamLanes / NT)
k_distill_stream(RowArgs a, RowWeights weights, bool by_range, TeacherLists lists,
                 DistillRule rule, float *loss, float *row_loss, float *per_row, void *dz,
                 uint64_t dstride,
                 uint32_t words, bool early, Ctrl *ctrl) {
  constexpr bool F = kFused<T>;
  constexpr int N = Vec16<T>::kN;
  extern __shared__ uint4 shared_words[];
  __shared__ __align__(16) int32_t ids[128];
  __shared__ RowSum red[NT / 32];
  __shared__ float4 sums[kMostParts];  // what the cluster's CTAs send: m, S
  __shared__ Carried carried[LONG ? NT / 32 : 1];
  __shared__ ListRoom list;
  __shared__ uint32_t singles;         // entries before and behind the vectors
  __shared__ bool twice;
  __shared__ unsigned long long sent;
  const uint64_t t = blockIdx.x;
  const uint32_t part = blockIdx.y, np = gridDim.y;
  const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  uint4 *ring = shared_words;
  uint32_t *marks = reinterpret_cast<uint32_t *>(ring + ST * kUnroll * NT);  // [words]
  if (threadIdx.x == 0) {
    if (np > 1) {
      mbar_init(&sent, 1);
      if (BACK || part == 0) mbar_arrive_tx(&sent, np * sizeof(float4));
      mbar_init_fence();
    }
    list.strange = -1;
    singles = 0;
    twice = false;
  }
  for (uint32_t i = threadIdx.x; i < words; i += NT) marks[i] = 0;
  __syncthreads();
  if (!early) pdl_wait();  // as in k_distill
  pdl_launch();
  Entry e = load_entry(lists, t);
  uint32_t first, n;
  row_part(a.vocab, part, np, &first, &n);
  T *d = reinterpret_cast<T *>(dz) + t * dstride + first;
  if ((a.mask && !a.mask[t]) || !in_sequences(weights, t)) {
    if (BACK) part_zero<T, NT>(d, n);
    if (early) pdl_wait();
    if (part) return;
    if (row_loss && threadIdx.x == 0) row_loss[t] = 0.f;
    conclude<NT>(0.f, per_row, loss, ctrl);
    return;  // the whole cluster
  }
  const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
  const Part<T, NT, ST> x(row + first, first, n);
  x.start(ring);
  if (np > 1) cluster_started();
  if (early) pdl_wait();
  const float lpr = lists.rest ? teacher_log(lists.rest[t]) : kNegInf,
              pr = lists.rest ? expf(lpr) : 0.f;
  const ListSums l = read_list<T, NT>(a, weights, by_range, lists, rule, row, t, pr, &e, &list);
  // Marks: a bit for each vector with an entry, and for each other number that is one.
  const uint32_t place = (uint32_t)e.id - first - x.sp.head;  // among the vectors' numbers
  const bool here = e.id >= 0 && (uint32_t)e.id - first < n, inside = here && place < x.sp.vecs * N;
  if (threadIdx.x < 128) ids[threadIdx.x] = e.id;
  if (inside) atomicOr(&marks[place / N / 32], 1u << (place / N & 31));
  else if (here)
    atomicOr(&singles, 1u << ((uint32_t)e.id - first < x.sp.head ? (uint32_t)e.id - first
                                                                  : (uint32_t)e.id - first -
                                                                        x.sp.vecs * N));
  __syncthreads();
  // The vector of an entry without its entries, by the first of them; others have none.
  bool mine = inside;
  uint4 rest_of = no_logits<T>();
  if (e.id >= 0) {
    const uint32_t begin = (uint32_t)e.id - place % N;
    uint32_t bits = 0;
    bool again = false;
#pragma unroll 2
    for (uint32_t j = 0; j < lists.top; j += 4) {
      const int4 four = *reinterpret_cast<const int4 *>(ids + j);
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) {
        const int32_t id = k == 0 ? four.x : k == 1 ? four.y : k == 2 ? four.z : four.w;
        const uint32_t d = (uint32_t)id - begin;
        if (d < N) {
          bits |= 1u << d;
          mine &= j + k >= threadIdx.x;
        }
        again |= id == e.id && j + k != threadIdx.x;
      }
    }
    if (again) twice = true;
    if (mine) {
      rest_of = x.vec(place / N);
      T *z = reinterpret_cast<T *>(&rest_of);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (bits >> i & 1) z[i] = from_f32<T>(kNegInf);
    }
  }
  const bool alone = x.single() && !(singles >> threadIdx.x & 1);
  const float single = alone ? to_f32(x.p[x.single_at()]) : kNegInf;
  RowSum sum;
  bool careful = !(fabsf(l.m) < __builtin_huge_valf()) || (F && !sums_hold(l.m, a.c));
  if (!careful) {
    const RowLog<T, F> log(l.m, a.c);
    F2 s(0.f), u(0.f);
    if (alone) add_one<T, false, F>(s, u, log, single);
    add_vector<T, false, F>(s, u, rest_of, log);
    Carried *own = &carried[LONG ? wid : 0];
    each_round<T, LONG, false>(x.rounds, own, s, u, [&](uint32_t g) {
      async_wait<ST - 1>();
      uint4 w[kUnroll];
      x.load(w, ring, g);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const uint32_t mark = marks[(k * (NT / 32) + wid) * x.rounds + g];
        if (mark && mark >> lane & 1) w[k] = no_logits<T>();
        add_vector<T, false, F>(s, u, w[k], log);
      }
      x.fetch(ring, g + ST);
    });
    sum = warp_sum<T, false>(sums_of<LONG>(own, l.m, s, F2(0.f)), a.c);
    if (lane == 0) red[wid] = sum;
    __syncthreads();
    sum = exact_sums<T>(
        warp_sum<T, false, lanes_for(NT / 32)>(
            lane < (NT / 32) ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, a.c), a.c);
    const float S = __shfl_sync(kAllLanes, sum.s, 0);
    careful = !(S >= kLeastSum && S <= kMostSum);
    if (careful) __syncthreads();
  }
  if (careful) {
    std::conditional_t<LONG, FarSum, LaneSum> b;
    if constexpr (!LONG) b = {kNegInf, F2(0.f), F2(0.f)};
    auto take = [&](const uint4 &w) {
      if constexpr (LONG) {
        F2 s(0.f), u;
        add_vector<T, false, false>(s, u, w, b.template raise<T, false>(Vec16<T>::max(w), a.c));
        b.s.add(s);
      } else {
        const uint4 v[1] = {w};
        take_vectors<T, false, false>(b, v, a.c);
      }
    };
    if (alone) {
      if constexpr (LONG) {
        F2 s(0.f), u;
        add_one<T, false, false>(s, u, b.template raise<T, false>(single, a.c), single);
        b.s.add(s);
      } else {
        add_one<T, false, false>(b.s, b.u, raise<T, false, false>(b, single, a.c), single);
      }
    }
    take(rest_of);
    x.each_vector(ring, [&](const uint4 &w, uint32_t i) {
      if (!(marks[i / 32] >> (i & 31) & 1)) take(w);
    });
    if constexpr (LONG) sum = warp_sum<T, false>(b.sum(), a.c);
    else sum = warp_sum<T, false>(row_sum(b), a.c);
    if (lane == 0) red[wid] = sum;
    __syncthreads();
    sum = warp_sum<T, false, lanes_for(NT / 32)>(
        lane < (NT / 32) ? red[lane] : RowSum{kNegInf, 0.f, 0.f}, a.c);
  }
  bool whole = true;
  if (np > 1) {
    cluster_wait();  // every CTA has started, so that its shared memory is there
    if (wid == 0) {
      const float4 own = make_float4(__shfl_sync(kAllLanes, sum.m, 0),
                                     __shfl_sync(kAllLanes, sum.s, 0), 0.f, 0.f);
      if (lane < (BACK ? np : 1)) send_float4(&sums[part], own, &sent, lane);
    }
    if (!BACK && part) return;
    whole = mbar_wait(&sent, 0, kRowWaitNs);
    if (!whole) {
      if (lane == 0) flag(ctrl, DEVERR_TIMEOUT, t);
      whole = mbar_wait(&sent, 0, kRowWaitNs);  // none of them comes after the end
    }
    whole = __syncthreads_and(whole);
    const float4 y = lane < np ? sums[lane] : make_float4(kNegInf, 0.f, 0.f, 0.f);
    sum = warp_sum<T, false, 8>(RowSum{y.x, y.y, 0.f}, a.c);
  }
  sum = {__shfl_sync(kAllLanes, sum.m, 0), __shfl_sync(kAllLanes, sum.s, 0), 0.f};
  const RowSums r = row_sums(l, sum, a.c, a.inv_t);
  RowLoss f;
  float lm = 0.f;
  if (rule.kind == EDP_DISTILL_MIX) {
    f = mix_loss(rule, lists, e, r, lpr, pr, &list, &lm);
  } else {
    f = row_loss_of(rule.kind, l, r, lpr, pr);
  }
  const bool zero = r.none || list.strange >= 0 || twice || !whole;
  if (part == 0 && threadIdx.x == 0) {
    if (list.strange >= 0)
      flag(ctrl, DEVERR_INDEX, (unsigned long long)(uint32_t)list.strange);
    if (twice) flag(ctrl, DEVERR_TWICE, t);
    if (r.none) flag(ctrl, DEVERR_ROW, t);
    if (row_loss) row_loss[t] = zero ? 0.f : f.loss;
  }
  if (BACK) {
    if (zero) {
      part_zero<T, NT>(d, n);
    } else {
      const float by = rule.grad_scale * list.weight * a.inv_t;
      part_grad_any<T, false, NT>(row + first, d, n, n, others_grad(r, f, by), a.c);
      __syncthreads();  // before the entries take their places
      if (here) d[(uint32_t)e.id - first] = from_f32<T>(by * entry_grad(rule, e, r, f, lm));
    }
  }
  if (part == 0)
    conclude<NT>(zero ? 0.f : list.weight * f.loss, per_row, loss, ctrl);
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
    auto stream = [&](auto back) {
      constexpr bool BACK = decltype(back)::value;
      StreamShape shape = stream_shape(ctx, z, 1);
      if (shape.vecs > 8 * 64 * 1024) shape.threads = 256, shape.stages = 2;  // room for the marks
      return by_shape<T>(shape, [&](auto threads, auto stages, auto is_long) {
        constexpr int NT = decltype(threads)::value, ST = decltype(stages)::value;
        constexpr bool LONG = decltype(is_long)::value;
        constexpr uint64_t round = kUnroll * (NT / 32);  // segments
        const uint32_t words = (uint32_t)(((shape.vecs + 8) / 32 / round + 1) * round);
        const size_t bytes = sizeof(uint4) * ST * kUnroll * NT + 4 * words;
        auto kern = k_distill_stream<T, NT, ST, BACK, LONG>;
        const cudaError_t err = cudaFuncSetAttribute(
            kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kResidentMost);
        if (err != cudaSuccess) return err;
        return launch_rows(kern, z.rows, shape.parts, true, NT, bytes, s, row_args(z), w,
                           p.w.by_range, lists, rule, loss, row_loss, p.per_token, dz, dstride,
                           words, p.early, ctx->ctrl);
      });
    };
    if (!dz) return stream(std::false_type{});
    // Parts of which not two fit an SM are read twice.  1,000 rows of 262,144 fp32 logits
    // (128 KB): 498 us so, 544 resident; 500 of 400,000 bfloat16 ones (98 KB): 215 and 156.
    if (part_bytes(z, 8) > kTwoParts) return stream(std::true_type{});
    uint32_t parts = row_parts(ctx, z, 2);
    while (parts < 8 && part_bytes(z, parts) > kResidentPart) parts *= 2;
    // few rows: smaller parts, so that the last of them are a small share
    while (parts < 8 && z.rows * parts < 8ull * ctx->coop_sms && part_bytes(z, parts) > kLeastPart)
      parts *= 2;
    const size_t bytes = part_bytes(z, parts);
    auto go = [&](auto threads) {
      constexpr int NT = decltype(threads)::value;
      auto kern = k_distill<T, NT>;
      const cudaError_t err = cudaFuncSetAttribute(
          kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kResidentMost);
      if (err != cudaSuccess) return err;
      return launch_rows(kern, z.rows, parts, true, NT, bytes, s, row_args(z), w, p.w.by_range,
                         lists, rule, loss, row_loss, p.per_token, dz, dstride, p.early,
                         ctx->ctrl);
    };
    // As many CTAs per SM as its shared memory and kLanes allow alike; few CTAs: more threads.
    // Measured (us, parts x threads): 515 rows of 32,003 fp32: 37.4 as 4 x 192, 46.7 as 4 x 384,
    // 42.6 as 4 x 256; of bfloat16 20.8 as 2 x 192, 26.6 as 2 x 384; 2,000 of 4,000: 17.6 as
    // 1 x 128, 31.0 as 1 x 384; 64 of 152,064: 12.6 as 8 x 256, 17.5 as 8 x 384.
    if (z.rows * parts <= (uint64_t)ctx->coop_sms) return go(std::integral_constant<int, 256>{});
    if (bytes > 55 * 1024) return go(std::integral_constant<int, 384>{});
    if (bytes > 36 * 1024) return go(std::integral_constant<int, 256>{});
    if (bytes > 24 * 1024) return go(std::integral_constant<int, 192>{});
    return go(std::integral_constant<int, 128>{});
  });
  if (e != cudaSuccess) forget_count(ctx, p, s);
  return e;
}

}  // namespace edp
