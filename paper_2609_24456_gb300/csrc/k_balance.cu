// k_balance.cu -- the balance loss of a router over a batch's tokens: how often
// each expert was chosen, the mean probability of each, their product's sum and
// its gradient by the router's logits.
//
// The counts need the choices alone (4 bytes each), so they come first; the
// gradient then takes one pass over the logits, read once and written once.  A
// row is a group of lanes with a few 16-byte vectors each (or a warp, element by
// element, where rows do not lie on 16-byte boundaries); the softmax stays in
// registers.  Counts and probabilities add up over CTAs as whole numbers, in
// any order to the same bits.  Up to kOneCta elements one CTA does both steps
// (256 rows of 64 experts 6.2 us, 6.4 in two kernels; 511 rows 8.2 and 6.4).
//
// 131,072 rows of 128 experts in bfloat16, 8 chosen: 22.8 us, 3.1 TB/s of the bytes
// that the call cannot do without.  What bounds it: 19 instructions an element, at 2.4
// of 4 a cycle from the 16 warps per SM that 128 registers leave (18 us); the counts'
// kernel and the starts and ends take the rest.  Forms off the vector path spill beyond
// 256 experts (96 bytes, 264 beyond 512), as do fp32's of more than 512 (260).
#include <type_traits>

#include "edp_loss.cuh"

namespace edp {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kMaxExperts = 1024;
constexpr uint64_t kOneCta = 16384;
// Rows of a lane: its fp32 sums of so many probabilities are good to 2^-16 at the worst
// before they go over to whole numbers.  More rows take more CTAs than one wave.
constexpr uint64_t kLaneRows = 256;
// An expert's probabilities add up in units of 2^-40 or, from so many rows on that all of
// them on one expert would pass 64 bits, of 2^-32.
constexpr float kProbUnits = 1099511627776.f;    // 2^40
constexpr float kProbUnitsMany = 4294967296.f;   // 2^32
constexpr uint64_t kManyRows = 1ull << 23;

}  // namespace

// Sums over CTAs, all 0 between calls.
struct BalanceSums {
  unsigned long long tokens;
  uint32_t nan, pad;
  unsigned long long prob[kMaxExperts];  // in units of 2^-40 or 2^-32
  uint32_t count[kMaxExperts];
};

namespace {

struct BalanceArgs {
  const void *z;
  uint64_t rows, stride;
  uint32_t E, top;
  const int32_t *sel;
  const uint8_t *mask;
  float coef, scale;  // coef, grad_scale coef
  float *loss, *prob;
  int64_t *counts;
  void *dz;
  uint64_t dstride;
  uint32_t *carry;  // beyond 32 bits of the counts, where a batch may come to them
};

// An expert's choices, over all CTAs.
__device__ __forceinline__ uint64_t count_of(const BalanceArgs &a, const BalanceSums *sums,
                                             uint32_t e) {
  return (a.carry ? (uint64_t)__ldcg(&a.carry[e]) << 32 : 0) | __ldcg(&sums->count[e]);
}

// Rows first, first + step, ... (a thread each) into hist; how many of them count.
__device__ __forceinline__ uint32_t count_choices(const BalanceArgs &a, uint64_t first,
                                                  uint64_t step, uint32_t *hist, Ctrl *ctrl) {
  uint32_t tokens = 0;
  auto take = [&](int32_t e) {
    if (e < 0) return;
    if ((uint32_t)e < a.E) atomicAdd(&hist[e], 1u);
    else flag(ctrl, DEVERR_INDEX, (unsigned long long)e);
  };
  const bool quads = a.top % 4 == 0 && ((uintptr_t)a.sel & 15u) == 0;
  for (uint64_t t = first; t < a.rows; t += step) {
    if (a.mask && !a.mask[t]) continue;
    ++tokens;
    const int32_t *sel = a.sel + t * a.top;
    if (quads) {
#pragma unroll 2
      for (uint32_t k = 0; k < a.top; k += 4) {
        const int4 e = *reinterpret_cast<const int4 *>(sel + k);
        take(e.x), take(e.y), take(e.z), take(e.w);
      }
    } else {
#pragma unroll 4
      for (uint32_t k = 0; k < a.top; ++k) take(sel[k]);
    }
  }
  return tokens;
}

__global__ void __launch_bounds__(kThreads)
k_expert_counts(BalanceArgs a, BalanceSums *sums, Ctrl *ctrl) {
  __shared__ uint32_t hist[kMaxExperts];
  pdl_wait();
  pdl_launch();
  for (uint32_t e = threadIdx.x; e < a.E; e += kThreads) hist[e] = 0;
  __syncthreads();
  uint32_t n = count_choices(a, (uint64_t)blockIdx.x * kThreads + threadIdx.x,
                             (uint64_t)gridDim.x * kThreads, hist, ctrl);
  n = __reduce_add_sync(kAllLanes, n);
  if ((threadIdx.x & 31) == 0 && n) atomicAdd(&sums->tokens, (unsigned long long)n);
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < a.E; e += kThreads)
    if (hist[e]) {
      const uint32_t before = atomicAdd(&sums->count[e], hist[e]);
      if (a.carry && before + hist[e] < before) atomicAdd(&a.carry[e], 1u);
    }
}

// CTAs per SM, by the elements of a lane.
template <int N>
constexpr int kBalancePerSm = N <= 4 ? 6 : N <= 8 ? 4 : N <= 16 ? 3 : N <= 32 ? 2 : 1;

// L lanes per row, V loads of VN elements per lane: element i of lane l is in
// column ((i / VN) L + l) VN + i % VN.
template <typename T, int VN>
struct Raw {
  using type = uint4;
};
template <typename T>
struct Raw<T, 1> {
  using type = T;
};
template <typename T, int VN>
__device__ __forceinline__ void unpack_row(const typename Raw<T, VN>::type &w, float (&v)[VN]) {
  const T *x = reinterpret_cast<const T *>(&w);
#pragma unroll
  for (int i = 0; i < VN; ++i) v[i] = to_f32(x[i]);
}
// A vector of -infinity.
template <typename T, int VN>
__device__ __forceinline__ typename Raw<T, VN>::type lowest_row() {
  if constexpr (VN == 1) {
    return from_f32<T>(kNegInf);
  } else {
    const uint32_t x = sizeof(T) == 4 ? 0xff800000u
                       : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;
    return make_uint4(x, x, x, x);
  }
}
// The largest element (NaN apart), of 16-bit types two at a time.
template <typename T, int V, int VN>
__device__ __forceinline__ float row_max(const typename Raw<T, VN>::type (&w)[V]) {
  if constexpr (VN == 8) {
    using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2,
                                         __nv_bfloat162>::type;
    const T2 *x = reinterpret_cast<const T2 *>(w);
    T2 m = x[0];
#pragma unroll
    for (int i = 1; i < 4 * V; ++i) m = __hmax2(m, x[i]);
    return fmaxf(to_f32(m.x), to_f32(m.y));
  } else {
    const T *x = reinterpret_cast<const T *>(w);
    float m = to_f32(x[0]);
#pragma unroll
    for (int i = 1; i < V * VN; ++i) m = fmaxf(m, to_f32(x[i]));
    return m;
  }
}
template <typename T, int VN>
__device__ __forceinline__ void store_row(T *p, const float (&v)[VN]) {
  if constexpr (VN == 1) {
    *p = from_f32<T>(v[0]);
  } else {
    uint4 w;
    T *x = reinterpret_cast<T *>(&w);
#pragma unroll
    for (int i = 0; i < VN; ++i) x[i] = from_f32<T>(v[i]);
    *reinterpret_cast<uint4 *>(p) = w;
  }
}

__device__ __forceinline__ void copy16(void *shared, const void *global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(shared)), "l"(global)
               : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// ONE: a single CTA, which counts the choices itself.  Otherwise a lane's vectors
// of its next rows are on their way to shared memory, in slots of its own: rows in
// flight then cost no registers (71 MB of logits and gradients of 128 experts:
// 44 us with one row ahead in registers).
template <typename T, int L, int V, int VN, int NT, bool ONE>
__global__ void __launch_bounds__(NT, ONE ? 1 : kBalancePerSm<V * VN>)
k_balance(BalanceArgs a, BalanceSums *sums, Ctrl *ctrl) {
  constexpr int N = V * VN, kGroups = NT / L, kWarps = NT / 32;
  constexpr uint32_t kCols = (uint32_t)N * L;  // columns with room for all experts
  constexpr int kDepth = ONE || VN == 1 ? 1 : V >= 8 ? 1 : V == 4 ? 2 : 4;
  constexpr bool kRing = kDepth > 1;
  constexpr size_t kRingBytes = kRing ? (size_t)kDepth * V * NT * 16 : 16;
  constexpr size_t kColBytes = (size_t)kWarps * kCols * sizeof(float);
  __shared__ alignas(16) uint8_t room[kRingBytes > kColBytes ? kRingBytes : kColBytes];
  __shared__ alignas(16) float fs[kCols];
  __shared__ uint32_t hist[ONE ? kMaxExperts : 1];
  __shared__ uint32_t one_tokens;
  __shared__ bool last;
  float(*col)[kCols] = reinterpret_cast<float(*)[kCols]>(room);  // once the ring is empty
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int l = threadIdx.x % L;
  const uint64_t step = (uint64_t)gridDim.x * kGroups;
  // the warp's groups take neighbouring rows and leave together
  uint64_t t0 = (uint64_t)blockIdx.x * kGroups + (threadIdx.x / 32) * (32 / L);
  using W = typename Raw<T, VN>::type;
  W *ring = reinterpret_cast<W *>(room);
  auto slot = [&](uint32_t d, int k) { return ((d % kDepth) * V + k) * NT + threadIdx.x; };
  auto fetch = [&](uint64_t t, uint32_t d) {
    if constexpr (kRing) {
      const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const uint32_t e = ((uint32_t)k * L + l) * VN;
        if (t < a.rows && e < a.E) copy16(&ring[slot(d, k)], row + e);
      }
      copies_end();
    }
  };
  // Only the counts come from the kernel before, which waited for all that came
  // before it: the first rows may be on their way while it runs.
  if (ONE) pdl_wait();
  uint32_t ahead = 0;
  if constexpr (kRing)
    for (; ahead < kDepth - 1; ++ahead) fetch(t0 + lane / L + ahead * step, ahead);
  if (!ONE) pdl_wait();
  if (ONE) pdl_launch();
  unsigned long long tokens;
  if (ONE) {
    for (uint32_t e = threadIdx.x; e < a.E; e += NT) hist[e] = 0;
    if (threadIdx.x == 0) one_tokens = 0;
    __syncthreads();
    uint32_t n = count_choices(a, threadIdx.x, NT, hist, ctrl);
    n = __reduce_add_sync(kAllLanes, n);
    if (lane == 0 && n) atomicAdd(&one_tokens, n);
    __syncthreads();
    tokens = one_tokens;
  } else {
    tokens = __ldcg(&sums->tokens);
  }
  const float inv_n = 1.f / (float)(tokens ? tokens : 1);
  const float per = (float)a.E / (float)a.top * inv_n;  // f_e = counts[e] * per
  const float scale = a.scale * inv_n;
  for (uint32_t e = threadIdx.x; e < kCols; e += NT)
    fs[e] = e < a.E ? ONE ? (float)hist[e] * per
                     : (a.carry ? (float)count_of(a, sums, e) : (float)__ldcg(&sums->count[e])) *
                           per : 0.f;
  __syncthreads();
  float ps[N];
#pragma unroll
  for (int i = 0; i < N; ++i) ps[i] = 0.f;
  bool nan = false;
  bool next = t0 + lane / L < a.rows && (!a.mask || a.mask[t0 + lane / L]);
  for (uint32_t d = 0; t0 < a.rows; t0 += step, ++d) {
    const uint64_t t = t0 + lane / L;
    const bool in = t < a.rows, use = next;
    next = t + step < a.rows && (!a.mask || a.mask[t + step]);
    // a masked row is loaded too: whatever it holds goes no further
    W w[V];
    if constexpr (kRing) {
      fetch(t + (kDepth - 1) * step, d + kDepth - 1);
      copies_wait<kDepth - 1>();
#pragma unroll
      for (int k = 0; k < V; ++k) w[k] = ring[slot(d, k)];
    } else {
      const T *row = reinterpret_cast<const T *>(a.z) + t * a.stride;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const uint32_t e = ((uint32_t)k * L + l) * VN;
        if (in && e < a.E) w[k] = *reinterpret_cast<const W *>(row + e);
      }
    }
    // what is not used is -infinity
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (!use || ((uint32_t)k * L + l) * VN >= a.E) w[k] = lowest_row<T, VN>();
    float y[N], m = row_max<T, V, VN>(w);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float v[VN];
      unpack_row<T, VN>(w[k], v);
#pragma unroll
      for (int i = 0; i < VN; ++i) y[k * VN + i] = v[i];
    }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAllLanes, m, o));
    if (m == kNegInf) m = 0.f;
    float s = 0.f, fp = 0.f;
    auto f = [&](int i) { return fs[((uint32_t)(i / VN) * L + l) * VN + i % VN]; };
#pragma unroll
    for (int i = 0; i < N; ++i) {
      y[i] = ex2((y[i] - m) * (float)kLog2e);
      s += y[i];
      fp = fmaf(y[i], f(i), fp);
    }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) {
      s += __shfl_xor_sync(kAllLanes, s, o);
      fp += __shfl_xor_sync(kAllLanes, fp, o);
    }
    if (use && s == 0.f && l == 0) flag(ctrl, DEVERR_ROW, t);  // no distribution: p = 0
    const float inv = s == 0.f ? 0.f : 1.f / s;
    nan |= isnan(inv);
#pragma unroll
    for (int i = 0; i < N; ++i) ps[i] = fmaf(y[i], inv, ps[i]);
    if (a.dz && in) {
      // p (f - sum f p) = (y / s) (f - fp / s)
      const float by = scale * inv, less = -by * (fp * inv);
      T *d = reinterpret_cast<T *>(a.dz) + t * a.dstride;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const uint32_t e = ((uint32_t)k * L + l) * VN;
        float v[VN];
#pragma unroll
        for (int i = 0; i < VN; ++i) v[i] = y[k * VN + i] * fmaf(f(k * VN + i), by, less);
        if (e < a.E) store_row<T, VN>(d + e, v);
      }
    }
  }
  if (!ONE) pdl_launch();
  if (nan) atomicExch(&sums->nan, 1u);
  if constexpr (kRing) copies_wait<0>();
  __syncthreads();  // the ring's room is free
  const float units = a.rows > kManyRows ? kProbUnitsMany : kProbUnits;
  // over the warp's groups, then its CTA's warps, in order
#pragma unroll
  for (int i = 0; i < N; ++i) {
#pragma unroll
    for (int o = L; o < 32; o <<= 1) ps[i] += __shfl_xor_sync(kAllLanes, ps[i], o);
    const uint32_t e = ((uint32_t)(i / VN) * L + l) * VN + i % VN;
    if (lane < L && e < a.E) col[wid][e] = ps[i];
  }
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < a.E; e += NT) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += col[w][e];
    if (ONE) col[0][e] = v;
    else if (v > 0.f) atomicAdd(&sums->prob[e], (unsigned long long)__float2ull_rn(v * units));
  }
  __threadfence();
  __syncthreads();
  if (!ONE) {
    if (threadIdx.x == 0) last = atomicAdd(&ctrl->loss_ticket, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
  }
  const bool bad = __ldcg(&sums->nan) != 0;
  Pair v{0.f, 0.f};
  for (uint32_t e = threadIdx.x; e < a.E; e += NT) {
    const uint64_t n = ONE ? hist[e] : count_of(a, sums, e);
    float p = ONE ? col[0][e]
                  : (float)__ldcg(&sums->prob[e]) *
                        (a.rows > kManyRows ? 1.f / kProbUnitsMany : 1.f / kProbUnits);
    p = bad ? __int_as_float(0x7fc00000) : p * inv_n;
    if (a.prob) a.prob[e] = p;
    a.counts[e] = (int64_t)n;
    pair_add(v, (float)n * per * p);
    if (!ONE) {
      sums->prob[e] = 0;
      sums->count[e] = 0;
      if (a.carry) a.carry[e] = 0;
    }
  }
  v = warp_join(v);
  __shared__ Pair red[kWarps];
  if (lane == 0) red[wid] = v;
  __syncthreads();  // every thread has seen sums->nan
  if (threadIdx.x) return;
  for (int w = 1; w < kWarps; ++w) v = pair_join(v, red[w]);
  a.loss[0] = a.coef * as_df(v).hi;
  sums->tokens = 0;
  sums->nan = 0;
  ctrl->loss_ticket = 0;
}

template <typename T, int L, int V, int VN>
cudaError_t launch_shape(edp_ctx *c, const BalanceArgs &a, BalanceSums *sums, cudaStream_t s) {
  if (a.rows * a.E <= kOneCta) {
    // the warps' columns fit shared memory, their elements the registers
    constexpr int N = V * VN, kCols = N * L;
    constexpr int NT = N <= 8 && kCols <= 256 ? 1024 : kCols <= 512 ? 512 : 256;
    return launch_pdl(k_balance<T, L, V, VN, NT, true>, dim3(1), dim3(NT), s, a, sums, c->ctrl);
  }
  const uint64_t sms = (uint64_t)c->coop_sms;
  const uint64_t cb = (a.rows + kThreads - 1) / kThreads;
  cudaError_t e = launch_pdl(k_expert_counts, dim3((unsigned)(cb < 4 * sms ? cb : 4 * sms)),
                             dim3(kThreads), s, a, sums, c->ctrl);
  if (e != cudaSuccess) return e;
  const uint64_t b = (a.rows * L + kThreads - 1) / kThreads;
  const uint64_t wave = kBalancePerSm<V * VN> * sms, least = (b + kLaneRows - 1) / kLaneRows;
  const uint64_t most = wave > least ? wave : least;
  e = launch_pdl(k_balance<T, L, V, VN, kThreads, false>,
                 dim3((unsigned)(b < most ? b : most)), dim3(kThreads), s, a, sums, c->ctrl);
  if (e != cudaSuccess) {  // the counts go no further
    cudaMemsetAsync(sums, 0, sizeof *sums, s);
    if (a.carry) cudaMemsetAsync(a.carry, 0, kMaxExperts * sizeof *a.carry, s);
  }
  return e;
}

template <typename T>
cudaError_t launch_type(edp_ctx *c, const BalanceArgs &a, BalanceSums *sums, cudaStream_t s) {
  constexpr int VN = 16 / sizeof(T);
  const uint64_t bytes = sizeof(T);
  const bool vec = ((uintptr_t)a.z | (uintptr_t)a.dz | a.E * bytes | a.stride * bytes |
                    (a.dz ? a.dstride * bytes : 0)) % 16 == 0;
  if (vec) {
    // vectors of a row: two per lane, and four from 16 on, where fewer lanes join their
    // sums (bfloat16, 33.5 M logits of 128, 256, 512 experts: 24.9, 25.0, 25.5 us with
    // two, 23.4, 22.4, 22.8 with four; fp32, 32 experts: 16.2 with two, 18.0 with four)
    const uint32_t n = a.E / VN;
    if (n <= 1) return launch_shape<T, 1, 1, VN>(c, a, sums, s);
    if (n <= 2) return launch_shape<T, 1, 2, VN>(c, a, sums, s);
    if (n <= 4) return launch_shape<T, 2, 2, VN>(c, a, sums, s);
    if (n <= 8) return launch_shape<T, 4, 2, VN>(c, a, sums, s);
    if (n <= 16) return launch_shape<T, 4, 4, VN>(c, a, sums, s);
    if (n <= 32) return launch_shape<T, 8, 4, VN>(c, a, sums, s);
    if (n <= 64) return launch_shape<T, 16, 4, VN>(c, a, sums, s);
    if (n <= 128) return launch_shape<T, 32, 4, VN>(c, a, sums, s);
    if constexpr (VN == 4) return launch_shape<T, 32, 8, VN>(c, a, sums, s);
  }
  if (a.E <= 32) return launch_shape<T, 32, 1, 1>(c, a, sums, s);
  if (a.E <= 64) return launch_shape<T, 32, 2, 1>(c, a, sums, s);
  if (a.E <= 128) return launch_shape<T, 32, 4, 1>(c, a, sums, s);
  if (a.E <= 256) return launch_shape<T, 32, 8, 1>(c, a, sums, s);
  if (a.E <= 512) return launch_shape<T, 32, 16, 1>(c, a, sums, s);
  return launch_shape<T, 32, 32, 1>(c, a, sums, s);
}

}  // namespace

cudaError_t launch_balance_loss(edp_ctx *c, const Logits &z, const int32_t *sel, uint32_t top,
                                double coef, double grad_scale, float *loss, int64_t *counts,
                                float *prob, void *dz, uint64_t dstride, cudaStream_t s) {
  void *blk = nullptr;
  // the carries only where they may be wanted: with the sums in a larger block 131,072 rows
  // of 128 experts took 25.0 us, 22.7 with this one
  const bool wide = z.rows * top >> 32 != 0;
  cudaError_t e = ctx_zeroed_scratch(
      c, sizeof(BalanceSums) + (wide ? kMaxExperts * sizeof(uint32_t) : 0), s, &blk);
  if (e != cudaSuccess) return e;
  BalanceSums *sums = (BalanceSums *)blk;
  uint32_t *carry = wide ? (uint32_t *)(sums + 1) : nullptr;
  const BalanceArgs a{z.z, z.rows, z.stride, z.vocab, top, sel, z.mask, (float)coef,
                      (float)(grad_scale * coef), loss, prob, counts, dz, dstride, carry};
  switch (z.dtype) {
    case EDP_BF16: return launch_type<__nv_bfloat16>(c, a, sums, s);
    case EDP_F16: return launch_type<__half>(c, a, sums, s);
    default: return launch_type<float>(c, a, sums, s);
  }
}

}  // namespace edp
