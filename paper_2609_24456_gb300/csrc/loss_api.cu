// loss_api.cu -- the C ABI of the losses over a packed batch: argument checks
// and dispatch to k_logits.cu, k_top.cu, k_policy.cu, k_pref.cu, k_balance.cu and
// k_distill.cu.
#include <cmath>
#include <initializer_list>

#include "edp_internal.cuh"

using namespace edp;

namespace {

bool device_arrays(const edp_ctx *ctx, std::initializer_list<const void *> ps) {
  const void *v;
  for (const void *p : ps)
    if (p && !device_view(ctx, p, &v, false)) return false;
  return true;
}

// Addresses at multiples of their elements' size: of 4 bytes and of 8.
bool aligned_arrays(std::initializer_list<const void *> fours,
                    std::initializer_list<const void *> eights) {
  uintptr_t a = 0, b = 0;
  for (const void *p : fours) a |= (uintptr_t)p;
  for (const void *p : eights) b |= (uintptr_t)p;
  return !(a & 3u) && !(b & 7u);
}
edp_status not_aligned(edp_ctx *ctx, const char *who) {
  return fail(ctx, EDP_ERR_INVALID, "%s: arrays are not aligned to their type", who);
}

size_t size_of(uint32_t dtype) { return dtype == EDP_F32 ? 4 : 2; }

bool in_order(double lo, double x) { return std::isfinite(x) && x >= lo; }

// Shape and type of logits, and of their gradient where it is given.
edp_status check_logits(edp_ctx *c, const char *who, const Logits &z, const void *dz,
                        uint64_t dstride, bool targets = true) {
  if (!z.z || (targets && !z.target))
    return fail(c, EDP_ERR_INVALID, "%s: NULL logits or target", who);
  if (z.dtype > EDP_F16) return fail(c, EDP_ERR_INVALID, "%s: unknown dtype", who);
  if (z.vocab == 0 || z.vocab > 0x7FFFFFFFu || z.rows > 0x7FFFFFFFull || z.stride < z.vocab ||
      z.stride > (1ull << 40))
    return fail(c, EDP_ERR_INVALID, "%s: need 0 < vocab <= stride, rows and vocab below 2^31", who);
  if (!(z.temperature >= 1e-6 && z.temperature <= 1e6))
    return fail(c, EDP_ERR_INVALID, "%s: temperature must be in [1e-6, 1e6]", who);
  if (((uintptr_t)z.z | (uintptr_t)dz) % size_of(z.dtype))
    return fail(c, EDP_ERR_INVALID, "%s: logits are not aligned to their type", who);
  if (dz && (dstride < z.vocab || dstride > (1ull << 40) || (dz == z.z && dstride != z.stride)))
    return fail(c, EDP_ERR_INVALID,
                "%s: dstride must be >= vocab, and the logits' own in their array", who);
  return EDP_OK;
}

// The distillation loss holds a bit for each 16 bytes of a row in a CTA's shared memory.
constexpr uint64_t kMostRowBytes = 16ull << 20;

edp_status check_top(edp_ctx *c, const char *who, uint32_t top) {
  if (top == 0 || top > 128) return fail(c, EDP_ERR_INVALID, "%s: need 0 < top <= 128", who);
  return EDP_OK;
}

edp_status check_tokens(edp_ctx *c, const char *who, const TokenSet &s) {
  if (s.n == 0 || s.n >= (1ull << 40))
    return fail(c, EDP_ERR_INVALID, "%s: need 0 < tokens < 2^40", who);
  if ((s.off != nullptr) != (s.n_seq != 0) || s.n_seq > 0x7FFFFFFFull ||
      (!s.off && s.reduce != EDP_REDUCE_TOKEN_MEAN))
    return fail(c, EDP_ERR_INVALID, "%s: off and n_seq go together, and by sequences both", who);
  return EDP_OK;
}

edp_status check_policy(edp_ctx *c, const char *who, const edp_policy_config *g,
                        const TokenSet &s, const PolicyTokens &p, bool has_entropy,
                        const float *loss) {
  if (!g || !p.old_logp || !p.adv || !loss)
    return fail(c, EDP_ERR_INVALID, "%s: NULL argument", who);
  if (!in_order(0.0, g->clip_low) || g->clip_low >= 1.0 || !in_order(0.0, g->clip_high) ||
      !in_order(0.0, g->dual_clip) || (g->dual_clip > 0.0 && g->dual_clip <= 1.0))
    return fail(c, EDP_ERR_INVALID,
                "%s: need 0 <= clip_low < 1, clip_high >= 0, dual_clip 0 or > 1", who);
  if (!in_order(0.0, g->kl_coef) || !in_order(0.0, g->entropy_coef) || !in_order(0.0, g->norm) ||
      !std::isfinite(g->grad_scale))
    return fail(c, EDP_ERR_INVALID, "%s: coefficients and norm must be finite and >= 0", who);
  if (g->kl > EDP_KL_K3 || g->reduce > EDP_REDUCE_SEQ_SUM || g->reserved[0] || g->reserved[1])
    return fail(c, EDP_ERR_INVALID, "%s: unknown kl or reduce, or reserved fields set", who);
  if (g->kl_coef > 0.0 && !p.ref_logp)
    return fail(c, EDP_ERR_INVALID, "%s: kl_coef needs ref_logp", who);
  if (g->entropy_coef > 0.0 && !has_entropy)
    return fail(c, EDP_ERR_INVALID, "%s: entropy_coef needs entropy", who);
  return check_tokens(c, who, s);
}

edp_status check_distill(edp_ctx *c, const char *who, const edp_distill_config *g,
                         const TokenSet &s, bool has_rest) {
  if (!g) return fail(c, EDP_ERR_INVALID, "%s: NULL argument", who);
  if (g->kind > EDP_DISTILL_MIX || g->reduce > EDP_REDUCE_SEQ_SUM || g->reserved[0] ||
      g->reserved[1])
    return fail(c, EDP_ERR_INVALID, "%s: unknown kind or reduce, or reserved fields set", who);
  if (g->kind == EDP_DISTILL_MIX ? !(g->beta > 0.0 && g->beta < 1.0) : g->beta != 0.0)
    return fail(c, EDP_ERR_INVALID, "%s: need 0 < beta < 1 with MIX, 0 else", who);
  if (has_rest ? g->teacher_temperature != 1.0
               : !(g->teacher_temperature >= 1e-6 && g->teacher_temperature <= 1e6))
    return fail(c, EDP_ERR_INVALID,
                "%s: teacher_temperature must be in [1e-6, 1e6], and 1 with rest", who);
  if (!has_rest && g->kind != EDP_DISTILL_FORWARD)
    return fail(c, EDP_ERR_INVALID, "%s: REVERSE and MIX need rest", who);
  if (!in_order(0.0, g->norm) || !std::isfinite(g->grad_scale))
    return fail(c, EDP_ERR_INVALID, "%s: norm and grad_scale must be finite, norm >= 0", who);
  return check_tokens(c, who, s);
}

void count_traffic(edp_ctx *c, uint64_t read, uint64_t write) {
  c->cnt.hbm_read += read;
  c->cnt.hbm_write += write;
  ++c->cnt.calls;
}

}  // namespace

extern "C" {

edp_status edp_token_logprob(edp_ctx *ctx, const void *logits, uint32_t dtype, uint64_t rows,
                             uint32_t vocab, uint64_t stride, const int32_t *target,
                             const uint8_t *mask, double temperature, float *logp,
                             float *entropy, float *stats, edp_stream stream) {
  if (!ctx) return EDP_ERR_INVALID;
  if (rows == 0) return EDP_OK;
  const Logits z{logits, dtype, vocab, rows, stride, target, mask, temperature};
  const edp_status st = check_logits(ctx, "edp_token_logprob", z, nullptr, 0);
  if (st != EDP_OK) return st;
  if (!logp || !device_arrays(ctx, {logits, target, mask, logp, entropy, stats}))
    return fail(ctx, EDP_ERR_INVALID, "edp_token_logprob: arrays must be device memory");
  if (!aligned_arrays({target, logp, entropy, stats}, {}))
    return not_aligned(ctx, "edp_token_logprob");
  DeviceGuard dg(ctx->cfg.device);
  EDP_TRACE(__func__);
  const cudaError_t e =
      launch_token_logprob(ctx, z, logp, entropy, stats, (cudaStream_t)stream);
  if (e != cudaSuccess) return launch_fail(ctx, e, "edp_token_logprob");
  count_traffic(ctx, rows * (vocab * size_of(dtype) + 4 + (mask != nullptr)),
                rows * (4 + 4 * (entropy != nullptr) + 8 * (stats != nullptr)));
  return EDP_OK;
}

edp_status edp_token_logprob_grad(edp_ctx *ctx, const void *logits, uint32_t dtype,
                                  uint64_t rows, uint32_t vocab, uint64_t stride,
                                  const int32_t *target, const uint8_t *mask,
                                  double temperature, const float *stats, const float *entropy,
                                  const float *dlogp, const float *dentropy, void *dlogits,
                                  uint64_t dstride, edp_stream stream) {
  if (!ctx) return EDP_ERR_INVALID;
  if (rows == 0) return EDP_OK;
  const Logits z{logits, dtype, vocab, rows, stride, target, mask, temperature};
  const edp_status st = check_logits(ctx, "edp_token_logprob_grad", z, dlogits, dstride);
  if (st != EDP_OK) return st;
  if (!stats || !dlogp || !dlogits)
    return fail(ctx, EDP_ERR_INVALID, "edp_token_logprob_grad: NULL stats, dlogp or dlogits");
  if ((entropy != nullptr) != (dentropy != nullptr))
    return fail(ctx, EDP_ERR_INVALID,
                "edp_token_logprob_grad: entropy and dentropy go together");
  if (!device_arrays(ctx, {logits, target, mask, stats, entropy, dlogp, dentropy, dlogits}))
    return fail(ctx, EDP_ERR_INVALID, "edp_token_logprob_grad: arrays must be device memory");
  if (!aligned_arrays({target, stats, entropy, dlogp, dentropy}, {}))
    return not_aligned(ctx, "edp_token_logprob_grad");
  DeviceGuard dg(ctx->cfg.device);
  EDP_TRACE(__func__);
  const cudaError_t e = launch_token_logprob_grad(ctx, z, stats, entropy, dlogp, dentropy,
                                                  dlogits, dstride, (cudaStream_t)stream);
  if (e != cudaSuccess) return launch_fail(ctx, e, "edp_token_logprob_grad");
  count_traffic(ctx,
                rows * (vocab * size_of(dtype) + 16 + (mask != nullptr) +
                        8 * (entropy != nullptr)),
                rows * vocab * size_of(dtype));
  return EDP_OK;
}

edp_status edp_token_top(edp_ctx *ctx, const void *logits, uint32_t dtype, uint64_t rows,
                         uint32_t vocab, uint64_t stride, const int32_t *target,
                         const uint8_t *mask, double temperature, uint32_t top, int32_t *ids,
                         float *top_logp, float *logp, float *entropy, float *rest,
                         float *stats, edp_stream stream) {
  if (!ctx) return EDP_ERR_INVALID;
  if (rows == 0) return EDP_OK;
  const Logits z{logits, dtype, vocab, rows, stride, target, mask, temperature};
  edp_status st = check_logits(ctx, "edp_token_top", z, nullptr, 0, false);
  if (st == EDP_OK) st = check_top(ctx, "edp_token_top", top);
  if (st != EDP_OK) return st;
  if (!ids || !top_logp || (logp && !target))
    return fail(ctx, EDP_ERR_INVALID, "edp_token_top: NULL ids or top_logp, or logp without target");
  if (!device_arrays(ctx, {logits, target, mask, ids, top_logp, logp, entropy, rest, stats}))
    return fail(ctx, EDP_ERR_INVALID, "edp_token_top: arrays must be device memory");
  if (!aligned_arrays({target, ids, top_logp, logp, entropy, rest, stats}, {}))
    return not_aligned(ctx, "edp_token_top");
  DeviceGuard dg(ctx->cfg.device);
  EDP_TRACE(__func__);
  const cudaError_t e = launch_token_top(ctx, z, top, ids, top_logp, logp, entropy, rest, stats,
                                         (cudaStream_t)stream);
  if (e != cudaSuccess) return launch_fail(ctx, e, "edp_token_top");
  count_traffic(ctx,
                rows * (vocab * size_of(dtype) + 4 * (target != nullptr) + (mask != nullptr)),
                rows * (8ull * top + 4 * (logp != nullptr) + 4 * (entropy != nullptr) +
                        4 * (rest != nullptr) + 8 * (stats != nullptr)));
  return EDP_OK;
}

edp_status edp_distill_loss(edp_ctx *ctx, const edp_distill_config *cfg, const void *logits,
                            uint32_t dtype, uint64_t rows, uint32_t vocab, uint64_t stride,
                            double temperature, const int32_t *ids, const float *value,
                            uint32_t top, const float *rest, const uint8_t *mask,
                            const uint64_t *off, uint64_t n_seq, float *loss, float *row_loss,
                            void *dlogits, uint64_t dstride, edp_stream stream) {
  if (!ctx) return EDP_ERR_INVALID;
  const Logits z{logits, dtype, vocab, rows, stride, nullptr, mask, temperature};
  const TokenSet set{mask, off, nullptr, vocab, cfg ? cfg->reduce : 0, n_seq, rows,
                     cfg ? cfg->norm : 0.0};
  edp_status st = check_distill(ctx, "edp_distill_loss", cfg, set, rest != nullptr);
  if (st == EDP_OK) st = check_logits(ctx, "edp_distill_loss", z, dlogits, dstride, false);
  if (st == EDP_OK) st = check_top(ctx, "edp_distill_loss", top);
  if (st != EDP_OK) return st;
  if (vocab * size_of(dtype) > kMostRowBytes)
    return fail(ctx, EDP_ERR_INVALID, "edp_distill_loss: a row of logits takes more than 16 MiB");
  if (!ids || !value || !loss)
    return fail(ctx, EDP_ERR_INVALID, "edp_distill_loss: NULL ids, value or loss");
  if (!device_arrays(ctx, {logits, ids, value, rest, mask, off, loss, row_loss, dlogits}))
    return fail(ctx, EDP_ERR_INVALID, "edp_distill_loss: arrays must be device memory");
  if (!aligned_arrays({ids, value, rest, loss, row_loss}, {off}))
    return not_aligned(ctx, "edp_distill_loss");
  DeviceGuard dg(ctx->cfg.device);
  EDP_TRACE(__func__);
  const cudaError_t e = launch_distill_loss(ctx, *cfg, set, z, ids, value, top, rest, loss,
                                            row_loss, dlogits, dstride, (cudaStream_t)stream);
  if (e != cudaSuccess) return launch_fail(ctx, e, "edp_distill_loss");
  count_traffic(ctx,
                rows * (vocab * size_of(dtype) + 8ull * top + 4 * (rest != nullptr) +
                        (mask != nullptr)) +
                    (off ? 8 * (n_seq + 1) : 0),
                rows * (vocab * size_of(dtype) * (dlogits != nullptr) +
                        4 * (row_loss != nullptr)) + 4);
  return EDP_OK;
}

edp_status edp_policy_loss(edp_ctx *ctx, const edp_policy_config *cfg, const float *logp,
                           const float *old_logp, const float *ref_logp, const float *adv,
                           const float *entropy, const uint8_t *mask, const uint64_t *off,
                           uint64_t n_seq, uint64_t n_tokens, float *loss, float *dlogp,
                           float *dentropy, edp_stream stream) {
  if (!ctx) return EDP_ERR_INVALID;
  const TokenSet set{mask, off, nullptr, 0, cfg ? cfg->reduce : 0, n_seq, n_tokens,
                     cfg ? cfg->norm : 0.0};
  const PolicyTokens p{logp, old_logp, ref_logp, adv, entropy};
  const edp_status st =
      check_policy(ctx, "edp_policy_loss", cfg, set, p, entropy != nullptr, loss);
  if (st != EDP_OK) return st;
  if (!logp || !device_arrays(ctx, {logp, old_logp, ref_logp, adv, entropy, mask, off, loss,
                                    dlogp, dentropy}))
    return fail(ctx, EDP_ERR_INVALID, "edp_policy_loss: arrays must be device memory");
  if (!aligned_arrays({logp, old_logp, ref_logp, adv, entropy, loss, dlogp, dentropy}, {off}))
    return not_aligned(ctx, "edp_policy_loss");
  DeviceGuard dg(ctx->cfg.device);
  EDP_TRACE(__func__);
  const cudaError_t e =
      launch_policy_loss(ctx, *cfg, set, p, loss, dlogp, dentropy, (cudaStream_t)stream);
  if (e != cudaSuccess) return launch_fail(ctx, e, "edp_policy_loss");
  count_traffic(ctx,
                n_tokens * (12 + 4 * (ref_logp != nullptr) + 4 * (entropy != nullptr) +
                            (mask != nullptr)) +
                    (off ? 8 * (n_seq + 1) : 0),
                n_tokens * 4 * ((dlogp != nullptr) + (dentropy != nullptr)) + 32);
  return EDP_OK;
}

edp_status edp_policy_loss_logits(edp_ctx *ctx, const edp_policy_config *cfg,
                                  const void *logits, uint32_t dtype, uint64_t rows,
                                  uint32_t vocab, uint64_t stride, const int32_t *target,
                                  double temperature, const float *old_logp,
                                  const float *ref_logp, const float *adv, const uint8_t *mask,
                                  const uint64_t *off, uint64_t n_seq, float *loss, float *logp,
                                  float *entropy, void *dlogits, uint64_t dstride,
                                  edp_stream stream) {
  if (!ctx) return EDP_ERR_INVALID;
  const Logits z{logits, dtype, vocab, rows, stride, target, mask, temperature};
  const TokenSet set{mask, off, target, vocab, cfg ? cfg->reduce : 0, n_seq, rows,
                     cfg ? cfg->norm : 0.0};
  const PolicyTokens p{nullptr, old_logp, ref_logp, adv, nullptr};
  edp_status st = check_policy(ctx, "edp_policy_loss_logits", cfg, set, p, true, loss);
  if (st == EDP_OK) st = check_logits(ctx, "edp_policy_loss_logits", z, dlogits, dstride);
  if (st != EDP_OK) return st;
  if (!logp || !dlogits)
    return fail(ctx, EDP_ERR_INVALID, "edp_policy_loss_logits: NULL logp or dlogits");
  if (!device_arrays(ctx, {logits, target, old_logp, ref_logp, adv, mask, off, loss, logp,
                           entropy, dlogits}))
    return fail(ctx, EDP_ERR_INVALID, "edp_policy_loss_logits: arrays must be device memory");
  if (!aligned_arrays({target, old_logp, ref_logp, adv, loss, logp, entropy}, {off}))
    return not_aligned(ctx, "edp_policy_loss_logits");
  DeviceGuard dg(ctx->cfg.device);
  EDP_TRACE(__func__);
  const cudaError_t e = launch_policy_loss_logits(ctx, *cfg, set, p, z, loss, logp, entropy,
                                                  dlogits, dstride, (cudaStream_t)stream);
  if (e != cudaSuccess) return launch_fail(ctx, e, "edp_policy_loss_logits");
  count_traffic(ctx,
                rows * (vocab * size_of(dtype) + 12 + 4 * (ref_logp != nullptr) +
                        (mask != nullptr)) +
                    (off ? 8 * (n_seq + 1) : 0),
                rows * (vocab * size_of(dtype) + 4 + 4 * (entropy != nullptr)) + 32);
  return EDP_OK;
}

edp_status edp_preference_loss(edp_ctx *ctx, const edp_preference_config *cfg,
                               const float *logp, const float *ref_logp, const uint8_t *mask,
                               const uint64_t *off, uint64_t n_seq, uint64_t n_tokens,
                               const int64_t *pair, uint32_t n_pair, float *loss,
                               float *seq_ratio, float *pair_loss, float *dlogp,
                               edp_stream stream) {
  if (!ctx) return EDP_ERR_INVALID;
  if (!cfg || !logp || !off || !pair || !loss)
    return fail(ctx, EDP_ERR_INVALID, "edp_preference_loss: NULL argument");
  if (!std::isfinite(cfg->beta) || !(cfg->beta > 0.0) || cfg->kind > EDP_PREF_HINGE ||
      cfg->average > 1 || !in_order(0.0, cfg->norm) || !std::isfinite(cfg->grad_scale) ||
      !std::isfinite(cfg->margin) || cfg->reserved[0] || cfg->reserved[1])
    return fail(ctx, EDP_ERR_INVALID, "edp_preference_loss: configuration out of range");
  if (!in_order(0.0, cfg->label_smoothing) || cfg->label_smoothing >= 0.5 ||
      (cfg->kind != EDP_PREF_LOGISTIC && cfg->label_smoothing != 0.0) ||
      (cfg->kind == EDP_PREF_SQUARE && cfg->margin != 0.0))
    return fail(ctx, EDP_ERR_INVALID,
                "edp_preference_loss: label_smoothing in [0, 1/2) and with LOGISTIC alone, no "
                "margin with SQUARE");
  if (n_seq == 0 || n_seq > 0x7FFFFFFFull || n_tokens == 0 || n_tokens >= (1ull << 40) ||
      n_pair == 0 || n_pair > (1u << 20))
    return fail(ctx, EDP_ERR_INVALID,
                "edp_preference_loss: need 0 < n_seq < 2^31, 0 < n_tokens < 2^40, 0 < n_pair <= "
                "2^20");
  if (!device_arrays(ctx, {logp, ref_logp, mask, off, pair, loss, seq_ratio, pair_loss, dlogp}))
    return fail(ctx, EDP_ERR_INVALID, "edp_preference_loss: arrays must be device memory");
  if (!aligned_arrays({logp, ref_logp, loss, seq_ratio, pair_loss, dlogp}, {off, pair}))
    return not_aligned(ctx, "edp_preference_loss");
  DeviceGuard dg(ctx->cfg.device);
  EDP_TRACE(__func__);
  const TokenSet set{mask, off, nullptr, 0, EDP_REDUCE_SEQ_SUM, n_seq, n_tokens, 0.0};
  const cudaError_t e =
      launch_preference_loss(ctx, *cfg, set, logp, ref_logp, pair, n_pair, loss, seq_ratio,
                             pair_loss, dlogp, (cudaStream_t)stream);
  if (e != cudaSuccess) return launch_fail(ctx, e, "edp_preference_loss");
  count_traffic(ctx,
                n_tokens * (4 + 4 * (ref_logp != nullptr) + (mask != nullptr)) +
                    8 * (n_seq + 1) + 16ull * n_pair,
                n_tokens * 4 * (dlogp != nullptr) + 4 * n_seq * (seq_ratio != nullptr) +
                    4ull * n_pair * (pair_loss != nullptr) + 16);
  return EDP_OK;
}

edp_status edp_balance_loss(edp_ctx *ctx, const void *logits, uint32_t dtype, uint64_t rows,
                            uint32_t experts, uint64_t stride, const int32_t *sel, uint32_t top,
                            const uint8_t *mask, double coef, double grad_scale, float *loss,
                            int64_t *counts, float *prob, void *dlogits, uint64_t dstride,
                            edp_stream stream) {
  if (!ctx) return EDP_ERR_INVALID;
  const Logits z{logits, dtype, experts, rows, stride, sel, mask, 1.0};
  const edp_status st = check_logits(ctx, "edp_balance_loss", z, dlogits, dstride);
  if (st != EDP_OK) return st;
  if (!loss || !counts) return fail(ctx, EDP_ERR_INVALID, "edp_balance_loss: NULL output");
  if (rows == 0 || experts > 1024 || top == 0 || top > 64)
    return fail(ctx, EDP_ERR_INVALID,
                "edp_balance_loss: need rows > 0, experts <= 1024, 0 < top <= 64");
  if (!std::isfinite(coef) || !std::isfinite(grad_scale))
    return fail(ctx, EDP_ERR_INVALID, "edp_balance_loss: coef and grad_scale must be finite");
  if (!device_arrays(ctx, {logits, sel, mask, loss, counts, prob, dlogits}))
    return fail(ctx, EDP_ERR_INVALID, "edp_balance_loss: arrays must be device memory");
  if (!aligned_arrays({sel, loss, prob}, {counts})) return not_aligned(ctx, "edp_balance_loss");
  DeviceGuard dg(ctx->cfg.device);
  EDP_TRACE(__func__);
  const cudaError_t e = launch_balance_loss(ctx, z, sel, top, coef, grad_scale, loss, counts,
                                            prob, dlogits, dstride, (cudaStream_t)stream);
  if (e != cudaSuccess) return launch_fail(ctx, e, "edp_balance_loss");
  count_traffic(ctx, rows * (experts * size_of(dtype) + 4 * top + (mask != nullptr)),
                rows * experts * size_of(dtype) * (dlogits != nullptr) + 4 +
                    experts * (8 + 4 * (prob != nullptr)));
  return EDP_OK;
}

}  // extern "C"
