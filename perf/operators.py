"""The learner's losses over a packed batch of token sequences, as cases that
can be timed.

A post-training program that has its batch from the packed delivery (tokens,
offsets, an advantage on every token) goes on with these operators:

* logprob        -- log-probabilities (and entropies) of the batch's tokens from
                    the logits, and the gradient of the logits;
* policy         -- the clipped policy loss with its KL and entropy terms, with
                    the gradients of the log-probabilities and entropies;
* policy_logits  -- both at once, from the logits to the gradient of the logits;
* preference     -- the loss of pairs of sequences (log ratios to a reference),
                    with the gradient of the log-probabilities;
* balance        -- counts of tokens per expert and the balance loss of a
                    router, with the gradient of its logits.

With `own` false the same is computed from elementary torch operations in 32
bits.  Inputs come from the seed alone.
"""
import math

import torch

own = False

DTYPES = dict(bf16=torch.bfloat16, f16=torch.float16, f32=torch.float32)
CLIP_LOW, CLIP_HIGH, DUAL_CLIP, KL_COEF, ENTROPY_COEF = 0.2, 0.28, 3.0, 0.02, 0.003
PREF_BETA, BALANCE_COEF = 0.1, 0.01
# gradients that are kept in 16 bits with 5 bits of exponent need a scale
SCALE, ROUTER_SCALE = 1024.0, 32_768.0


def listed():
    return [
        # serving: the log-probability of one sampled token, while an actor
        # generates; latency alone
        dict(name="logprob_one_token", kind="logprob", rows=1, vocab=152_064, pad=0, dtype="bf16",
             keep=1.0, entropy=True, back=False, temperature=0.7, banned=0),
        # scoring a micro-batch of responses under the old or the reference
        # policy; a tenth of the rows are prompt tokens
        dict(name="logprob_8192", kind="logprob", rows=8_192, vocab=152_064, pad=0, dtype="bf16",
             keep=0.9, entropy=True, back=False, temperature=1.0, banned=64),
        # the backward pass of a micro-batch with an entropy bonus
        dict(name="logprob_grad_4096", kind="logprob", rows=4_096, vocab=152_064, pad=0,
             dtype="bf16", keep=0.9, entropy=True, back=True, temperature=1.0, banned=0),
        # a small vocabulary of an odd size: rows at every alignment
        dict(name="logprob_grad_odd", kind="logprob", rows=777, vocab=32_003, pad=0, dtype="f16",
             keep=1.0, entropy=False, back=True, temperature=0.9, banned=5),
        # one micro-batch of short responses: launches and latency
        dict(name="policy_small", kind="policy", seqs=32, lmin=8, lmax=128, reduce="token_mean",
             ref=True, entropy=True, masked=True),
        # a whole post-training batch, 512 prompts of 16 responses
        dict(name="policy_8192", kind="policy", seqs=8_192, lmin=128, lmax=4_096,
             reduce="seq_mean", ref=True, entropy=False, masked=True),
        # loss and gradient from a micro-batch's logits in one call
        dict(name="policy_logits_8192", kind="policy_logits", rows=8_192, seqs=12, vocab=152_064,
             pad=0, dtype="bf16", keep=0.9, reduce="token_mean", ref=True, entropy=True,
             temperature=1.0),
        # the same in 32 bits over a small vocabulary of an odd size
        dict(name="policy_logits_odd", kind="policy_logits", rows=515, seqs=9, vocab=32_003,
             pad=0, dtype="f32", keep=0.8, reduce="seq_mean", ref=False, entropy=False,
             temperature=1.0),
        # a micro-batch of pairs
        dict(name="preference_8", kind="preference", groups=8, size=2, lmin=16, lmax=512,
             loss="logistic", average=False, ref=True, masked=True),
        # the best of 16 responses against each of the others, for 512 prompts
        dict(name="preference_7680", kind="preference", groups=512, size=16, lmin=128,
             lmax=4_096, loss="logistic", average=False, ref=True, masked=True),
        # a router at a decoding step's batch
        dict(name="balance_256", kind="balance", rows=256, experts=64, top=6, dtype="f32",
             masked=False),
        # one layer's router over a training batch
        dict(name="balance_131072", kind="balance", rows=131_072, experts=128, top=8,
             dtype="bf16", masked=True),
    ]


# --- draws ---------------------------------------------------------------------
_LOGITS = 1_245_708_288  # elements of the largest listed logits


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_shape(rng, least):
    vocab = rng.choice([152_064, 32_000, _log(rng, 500, 262_144), _log(rng, 500, 262_144)])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    most = _LOGITS // vocab // (2 if dtype == "f32" else 1)
    return dict(rows=_log(rng, least, min(8_192, most)), vocab=vocab, dtype=dtype,
                pad=rng.choice([0, 0, -vocab % 64]), keep=rng.choice([1.0, 0.9, 0.5]),
                temperature=rng.choice([1.0, 1.0, 0.7]))


def _draw_logprob(rng):
    c = dict(kind="logprob", **_draw_shape(rng, 1))
    c.update(entropy=rng.random() < 0.5, back=rng.random() < 0.5,
             banned=rng.choice([0, 0, 1, 64]))
    return c


def _draw_policy(rng):
    lmax = _log(rng, 4, 32_768)
    return dict(kind="policy", seqs=max(1, min(_log(rng, 1, 65_536), 17_000_000 // lmax)),
                lmin=rng.choice([0, 1, lmax // 8]), lmax=lmax,
                reduce=rng.choice(["token_mean", "seq_mean", "seq_sum"]), ref=rng.random() < 0.6,
                entropy=rng.random() < 0.4, masked=rng.random() < 0.7)


def _draw_policy_logits(rng):
    c = dict(kind="policy_logits", **_draw_shape(rng, 8))
    c.update(seqs=_log(rng, 1, max(1, c["rows"] // 4)),
             reduce=rng.choice(["token_mean", "seq_mean", "seq_sum"]), ref=rng.random() < 0.6,
             entropy=rng.random() < 0.5)
    return c


def _draw_preference(rng):
    lmax = _log(rng, 4, 32_768)
    size = rng.choice([2, 2, 2, 4, 16])
    return dict(kind="preference",
                groups=max(1, min(_log(rng, 1, 16_384), 17_000_000 // lmax // size)), size=size,
                lmin=rng.choice([1, max(1, lmax // 8)]), lmax=lmax,
                loss=rng.choice(["logistic", "logistic", "square", "hinge"]),
                average=rng.random() < 0.3, ref=rng.random() < 0.8, masked=rng.random() < 0.7)


def _draw_balance(rng):
    experts = rng.choice([8, 16, 60, 64, 128, 256, 384, _log(rng, 2, 512)])
    return dict(kind="balance", rows=_log(rng, 1, min(131_072, 16_777_216 // experts)),
                experts=experts, top=rng.randint(1, min(8, experts)),
                dtype=rng.choice(["bf16", "f32", "f16"]), masked=rng.random() < 0.5)


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        c = rng.choice([_draw_logprob, _draw_logprob, _draw_policy, _draw_policy_logits,
                        _draw_preference, _draw_balance])(rng)
        if work(c)["bytes"] <= most:
            return c


# --- inputs ----------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _uniform(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _logits_inputs(c, seed):
    """Logits as a language model gives them (a wide bulk and a few likely
    tokens, the target most often among them), targets, and the mask."""
    g = _gen(seed)
    R, V = c["rows"], c["vocab"]
    z = torch.empty(R, V + c["pad"], dtype=DTYPES[c["dtype"]], device="cuda")
    T = c["temperature"]
    z.normal_(0.0, 2.5 * T, generator=g)
    z = z[:, :V]
    target = torch.randint(0, V, (R,), generator=g, device="cuda")
    # about as likely as all of the bulk, whose log-sum is ln V + 3
    z.scatter_(1, target[:, None], (T * (math.log(V) + 3 + _normal(g, R, 1))).to(z.dtype))
    other = torch.randint(0, V, (R, 4), generator=g, device="cuda")
    z.scatter_(1, torch.where(other == target[:, None], (other + 1) % V, other),
               (T * (math.log(V) + 1 + 2 * _normal(g, R, 4))).to(z.dtype))
    if c.get("banned"):  # tokens that the sampler excludes
        ban = torch.randint(0, V, (R, c["banned"]), generator=g, device="cuda")
        ban = torch.where(ban == target[:, None], (ban + 1) % V, ban)
        ban = torch.where(ban == target[:, None], (ban + 1) % V, ban)
        z.scatter_(1, ban, -math.inf)
    mask = (_uniform(g, R) < c["keep"]).to(torch.uint8) if c["keep"] < 1 else None
    return g, z, target.to(torch.int32), mask


def _plain_stats(z, target, T):
    """log p(target), entropy, p and ln p in the type of z."""
    x = z / T
    y = x - x.amax(1, keepdim=True)
    e = torch.exp(y)
    s = e.sum(1, keepdim=True)
    logq = y - torch.log(s)
    p = e / s
    plogq = torch.where(p > 0, p * logq, torch.zeros_like(p))
    logp = logq.gather(1, target.long()[:, None])[:, 0]
    return logp, -plogq.sum(1), p, plogq


def _tokens(c, n):
    return max(1, n * (c["lmin"] + c["lmax"]) // 2)


def _ragged(g, c, n):
    """Offsets of n sequences of lmin to lmax tokens, about, and one total."""
    lens = torch.randint(c["lmin"], c["lmax"] + 1, (n,), generator=g, device="cuda")
    ends = torch.cumsum(lens + (lens.sum() == 0), 0)
    return torch.cat([ends.new_zeros(1), ends * _tokens(c, n) // ends[-1]])


def _sequences_of(off, n):
    """The sequence of each of the n tokens."""
    return torch.searchsorted(off[1:], torch.arange(n, device=off.device), right=True)


def _response_mask(g, off, n, masked):
    """1 on the tokens of the responses: not on a prompt's (an eighth of the
    sequence at most), and not on one in fifty that a tool wrote."""
    if not masked:
        return None
    seg = _sequences_of(off, n)
    lens = off[1:] - off[:-1]
    prompt = off[:-1] + (lens * _uniform(g, lens.numel()) / 8).long()
    keep = (torch.arange(n, device="cuda") >= prompt[seg]) & (_uniform(g, n) >= 0.02)
    return keep.to(torch.uint8)


def _policy_inputs(g, logp, off, n, ref):
    """Old and reference log-probabilities around the present ones, and an
    advantage per sequence on its tokens."""
    old = (logp + 0.15 * _normal(g, n)).clamp(max=0.0)
    refp = (logp + 0.25 * _normal(g, n)).clamp(max=0.0) if ref else None
    adv = _normal(g, off.numel() - 1)[_sequences_of(off, n)].contiguous()
    return old, refp, adv


def _logp_values(g, n):
    return -torch.empty(n, device="cuda").exponential_(1.4, generator=g)


def _token_inputs(c, seed):
    g = _gen(seed)
    off, n = _ragged(g, c, c["seqs"]), _tokens(c, c["seqs"])
    logp = _logp_values(g, n)
    old, ref, adv = _policy_inputs(g, logp, off, n, c["ref"])
    entropy = 2 * _uniform(g, n) if c["entropy"] else None
    return off, n, logp, old, ref, adv, _response_mask(g, off, n, c["masked"]), entropy


def _row_inputs(c, seed):
    g, z, target, mask = _logits_inputs(c, seed)
    R = c["rows"]
    cuts = torch.sort(torch.randint(0, R + 1, (c["seqs"] - 1,), generator=g, device="cuda"))[0]
    off = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), R)])
    lse = torch.logsumexp(z, 1) if c["dtype"] == "f32" else torch.cat(
        [torch.logsumexp(part.float(), 1) for part in z.split(1024)])
    # an approximation serves: the old policy's values are noisy all the same
    logp = (z.gather(1, target.long()[:, None])[:, 0].float() - lse) / c["temperature"]
    old, ref, adv = _policy_inputs(g, logp, off, R, c["ref"])
    return z, target, mask, off, old, ref, adv


def _pair_inputs(c, seed):
    """Pairs (the first of a group, each of its others), in groups' order."""
    g = _gen(seed)
    G, size = c["groups"], c["size"]
    off, n = _ragged(g, c, G * size), _tokens(c, G * size)
    logp = _logp_values(g, n)
    ref = logp + 0.03 * _normal(g, n) if c["ref"] else None
    first = torch.arange(G, device="cuda")[:, None] * size
    others = first + torch.arange(1, size, device="cuda")
    pair = torch.stack([first.expand_as(others), others], 2).reshape(-1, 2).contiguous()
    return off, n, logp, ref, _response_mask(g, off, n, c["masked"]), pair


def _router_inputs(c, seed):
    g = _gen(seed)
    N, E = c["rows"], c["experts"]
    z = (_normal(g, N, E) + 0.5 * _normal(g, E)).to(DTYPES[c["dtype"]])
    # the router explores: noise in its choice, which also leaves no ties
    sel = torch.topk(z.float() + 0.1 * _normal(g, N, E), c["top"], 1)[1].to(torch.int32)
    mask = (_uniform(g, N) < 0.9).to(torch.uint8) if c["masked"] else None
    return z, sel, mask


# --- prepare ---------------------------------------------------------------------
def _like(z):
    return torch.zeros(z.shape[0], z.stride(0), dtype=z.dtype, device="cuda")[:, :z.shape[1]]


def _prepare_logprob(c, seed):
    g, z, target, mask = _logits_inputs(c, seed)
    R = c["rows"]
    s = dict(z=z, target=target, mask=mask)
    if not c["back"]:
        s["out"] = dict(logp=torch.zeros(R, device="cuda"))
        if c["entropy"]:
            s["out"]["entropy"] = torch.zeros(R, device="cuda")
        return s
    # what the forward pass left: the rows' largest logits, their sums of
    # exponentials relative to it, and entropies
    T = c["temperature"]
    parts = [_forward_of(part, t, T) for part, t in zip(z.split(512), target.split(512))]
    m, sums, entropy = (torch.cat(v) for v in zip(*parts))
    s.update(stats=torch.stack([m, sums], 1).contiguous(),
             entropy=entropy if c["entropy"] else None, out=dict(dlogits=_like(z)))
    s["dlogp"], s["dentropy"] = _upstream(c, g)
    return s


def _upstream(c, g):
    """Gradients by the log-probabilities and the entropies."""
    R, by = c["rows"], _scale(c) / c["rows"]
    dh = torch.full((R,), -ENTROPY_COEF * by, device="cuda") if c["entropy"] else None
    return _normal(g, R) * by, dh


def _scale(c):
    if c.get("dtype") != "f16":
        return 1.0
    return ROUTER_SCALE if c["kind"] == "balance" else SCALE


def _forward_of(z, target, T):
    m = z.amax(1, keepdim=True).float()
    y = (z.float() - m) / T
    e = torch.exp(y)
    s = e.sum(1)
    h = torch.where(e > 0, e * y, torch.zeros_like(e)).sum(1)
    return m[:, 0], s, torch.log(s) - h / s


def _prepare_policy(c, seed):
    off, n, logp, old, ref, adv, mask, entropy = _token_inputs(c, seed)
    o = dict(loss=torch.zeros(8, device="cuda"), dlogp=torch.zeros(n, device="cuda"))
    if c["entropy"]:
        o["dentropy"] = torch.zeros(n, device="cuda")
    return dict(off=off, n=n, logp=logp, old=old, ref=ref, adv=adv, mask=mask, entropy=entropy,
                cfg=_policy_config(c), out=o)


def _prepare_policy_logits(c, seed):
    z, target, mask, off, old, ref, adv = _row_inputs(c, seed)
    o = dict(loss=torch.zeros(8, device="cuda"), logp=torch.zeros(c["rows"], device="cuda"),
             dlogits=_like(z))
    return dict(z=z, target=target, mask=mask, off=off, old=old, ref=ref, adv=adv,
                cfg=_policy_config(c), out=o)


def _prepare_preference(c, seed):
    off, n, logp, ref, mask, pair = _pair_inputs(c, seed)
    o = dict(loss=torch.zeros(4, device="cuda"),
             ratio=torch.zeros(off.numel() - 1, device="cuda"),
             pair_loss=torch.zeros(pair.shape[0], device="cuda"),
             dlogp=torch.zeros(n, device="cuda"))
    return dict(off=off, n=n, logp=logp, ref=ref, mask=mask, pair=pair, out=o)


def _prepare_balance(c, seed):
    z, sel, mask = _router_inputs(c, seed)
    o = dict(loss=torch.zeros(1, device="cuda"), dlogits=torch.zeros_like(z),
             counts=torch.zeros(c["experts"], dtype=torch.int64, device="cuda"),
             prob=torch.zeros(c["experts"], device="cuda"))
    return dict(z=z, sel=sel, mask=mask, out=o)


def _policy_config(c):
    return dict(clip_low=CLIP_LOW, clip_high=CLIP_HIGH, dual_clip=DUAL_CLIP,
                kl_coef=KL_COEF if c["ref"] else 0.0, kl="k3", reduce=c["reduce"],
                entropy_coef=ENTROPY_COEF if c["entropy"] else 0.0, grad_scale=_scale(c))


def prepare(case, seed):
    s = globals()["_prepare_" + case["kind"]](case, seed)
    s["case"] = case
    return s


# --- run: the framework's operators ------------------------------------------------
_program = {}


def _ctx():
    """The program's context (these operators use its GPU, not its ring)."""
    from paper_2609_24456_gb300 import edp
    if not _program:
        _program["ring"] = edp.Ring(
            edp.make_config(16, (1, 4, 4), edp.EDP_XFORM_CHW_NORM_BF16), action=False,
            reward=False, done=False)
    return _program["ring"].ctx


def _own_config(edp, cfg):
    return edp.make_policy_config(**dict(
        cfg, kl=getattr(edp, "EDP_KL_" + cfg["kl"].upper()),
        reduce=getattr(edp, "EDP_REDUCE_" + cfg["reduce"].upper())))


def _own_logprob(s):
    from paper_2609_24456_gb300 import edp
    c, o = s["case"], s["out"]
    if c["back"]:
        edp.edp_token_logprob_grad(_ctx(), s["z"], s["target"], s["stats"], s["dlogp"],
                                   o["dlogits"], mask=s["mask"], temperature=c["temperature"],
                                   entropy=s["entropy"], dentropy=s["dentropy"])
    else:
        edp.edp_token_logprob(_ctx(), s["z"], s["target"], o["logp"], mask=s["mask"],
                              temperature=c["temperature"], entropy=o.get("entropy"))
    return o


def _own_policy(s):
    from paper_2609_24456_gb300 import edp
    o = s["out"]
    edp.edp_policy_loss(_ctx(), _own_config(edp, s["cfg"]), s["logp"], s["old"],
                        s["adv"], s["n"], o["loss"], ref_logp=s["ref"], mask=s["mask"],
                        off=s["off"], n_seq=s["case"]["seqs"], entropy=s["entropy"],
                        dlogp=o["dlogp"], dentropy=o.get("dentropy"))
    return o


def _own_policy_logits(s):
    from paper_2609_24456_gb300 import edp
    c, o = s["case"], s["out"]
    edp.edp_policy_loss_logits(_ctx(), _own_config(edp, s["cfg"]), s["z"],
                               s["target"], s["old"], s["adv"], o["loss"], o["logp"],
                               o["dlogits"], ref_logp=s["ref"], mask=s["mask"], off=s["off"],
                               n_seq=c["seqs"], temperature=c["temperature"])
    return o


def _own_preference(s):
    from paper_2609_24456_gb300 import edp
    o = s["out"]
    c = s["case"]
    cfg = edp.make_preference_config(PREF_BETA, average=c["average"],
                                     kind=getattr(edp, "EDP_PREF_" + c["loss"].upper()))
    edp.edp_preference_loss(_ctx(), cfg, s["logp"], s["off"], s["off"].numel() - 1, s["n"], s["pair"],
                            s["pair"].shape[0], o["loss"], ref_logp=s["ref"], mask=s["mask"],
                            seq_ratio=o["ratio"], pair_loss=o["pair_loss"], dlogp=o["dlogp"])
    return o


def _own_balance(s):
    from paper_2609_24456_gb300 import edp
    o = s["out"]
    edp.edp_balance_loss(_ctx(), s["z"], s["sel"], BALANCE_COEF, o["loss"], o["counts"],
                         mask=s["mask"], prob=o["prob"], dlogits=o["dlogits"],
                         grad_scale=_scale(s["case"]))
    return o


# --- run: the plain form -------------------------------------------------------------
def _plain_logprob(s):
    c, o = s["case"], s["out"]
    z, T = s["z"].float(), c["temperature"]
    live = s["mask"].bool() if s["mask"] is not None else torch.ones_like(s["target"]).bool()
    if not c["back"]:
        logp, h, _, _ = _plain_stats(z, s["target"], T)
        out = dict(logp=torch.where(live, logp, torch.zeros_like(logp)))
        if c["entropy"]:
            out["entropy"] = torch.where(live, h, torch.zeros_like(h))
        return out
    m, sums = s["stats"][:, :1], s["stats"][:, 1:]
    y = (z - m) / T
    p = torch.exp(y) / sums
    grad = _plain_logits_grad(p, s["target"], s["dlogp"], T)
    if c["entropy"]:
        inner = y - torch.log(sums) + s["entropy"][:, None]
        grad = grad - torch.where(p > 0, p * inner, torch.zeros_like(p)) * (s["dentropy"][:, None]
                                                                           / T)
    return dict(dlogits=torch.where(live[:, None], grad, torch.zeros_like(grad)).to(s["z"].dtype))


def _plain_logits_grad(p, target, dlogp, T):
    g = (dlogp / T)[:, None]
    grad = -p * g
    return grad.scatter_add_(1, target.long()[:, None], g)


def _token_loss(c, logp, old, ref, adv, entropy, live, off):
    """Loss and statistics, and the gradients by logp and entropy, in logp's type."""
    zero = torch.zeros_like(logp)
    n = logp.numel()
    keep = live.to(logp.dtype)
    d = torch.where(live, logp - old, zero)
    r = torch.exp(d)
    surr = torch.minimum(r * adv, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv)
    surr = torch.where(adv < 0, torch.maximum(surr, DUAL_CLIP * adv), surr)
    # the limits of the ratio, as limits of its logarithm
    over = (adv > 0) & (d > math.log1p(CLIP_HIGH))
    under = (adv < 0) & ((d < math.log1p(-CLIP_LOW)) | (d > math.log(DUAL_CLIP)))
    dpg = torch.where(over | under, zero, -r * adv)
    kl, dkl = zero, zero
    if ref is not None:
        q = torch.where(live, ref - logp, zero)
        kl, dkl = torch.expm1(q) - q, -torch.expm1(q)
    valid = keep.sum()
    S = off.numel() - 1
    if c["reduce"] == "token_mean":
        w = keep / valid.clamp(min=1)
    elif c["reduce"] == "seq_sum":
        w = keep / S
    else:
        seg = _sequences_of(off, n)
        per = torch.zeros(S, dtype=logp.dtype, device=logp.device).index_add_(0, seg, keep)
        w = keep / (S * per.clamp(min=1))[seg]
    clk, ch = (KL_COEF if ref is not None else 0.0), (ENTROPY_COEF if c["entropy"] else 0.0)
    pg_sum, kl_sum = -(w * surr).sum(), (w * kl).sum()
    h_sum = (w * torch.where(live, entropy, zero)).sum() if entropy is not None else zero.sum()
    mean = lambda x: (keep * x).sum() / valid.clamp(min=1)  # noqa: E731
    loss = torch.stack([pg_sum + clk * kl_sum - ch * h_sum, pg_sum, kl_sum, h_sum,
                        mean(over.to(logp.dtype)), mean(under.to(logp.dtype)), mean(r),
                        mean(torch.expm1(d) - d)])
    by = _scale(c)
    return loss, by * w * (dpg + clk * dkl), -ch * by * w


def _live(mask, like):
    return mask.bool() if mask is not None else torch.ones_like(like).bool()


def _plain_policy(s):
    loss, dlogp, dh = _token_loss(s["case"], s["logp"], s["old"], s["ref"], s["adv"],
                                  s["entropy"], _live(s["mask"], s["logp"]), s["off"])
    out = dict(loss=loss, dlogp=dlogp)
    if s["entropy"] is not None:
        out["dentropy"] = dh
    return out


def _rows_loss(c, z, target, mask, off, old, ref, adv):
    live, T = _live(mask, target), c["temperature"]
    logp, h, p, plogq = _plain_stats(z, target, T)
    zero = torch.zeros_like(logp)
    logp, h = torch.where(live, logp, zero), torch.where(live, h, zero)
    loss, dlogp, dh = _token_loss(c, logp, old, ref, adv, h if c["entropy"] else None, live, off)
    grad = _plain_logits_grad(p, target, dlogp, T)
    if c["entropy"]:
        grad = grad - (plogq + p * h[:, None]) * (dh / T)[:, None]
    return loss, logp, torch.where(live[:, None], grad, torch.zeros_like(grad))


def _plain_policy_logits(s):
    loss, logp, grad = _rows_loss(s["case"], s["z"].float(), s["target"], s["mask"], s["off"],
                                  s["old"], s["ref"], s["adv"])
    return dict(loss=loss, logp=logp, dlogits=grad.to(s["z"].dtype))


def _pair_loss(c, off, n, logp, ref, mask, pair):
    S, P = off.numel() - 1, pair.shape[0]
    seg = _sequences_of(off, n)
    keep = _live(mask, logp).to(logp.dtype)
    per = logp.new_zeros(S).index_add_(0, seg, keep)
    x = logp - ref if ref is not None else logp
    ratio = logp.new_zeros(S).index_add_(0, seg, keep * x)
    scale = 1 / per.clamp(min=1) if c["average"] else torch.ones_like(per)
    ratio = ratio * scale
    h = ratio[pair[:, 0]] - ratio[pair[:, 1]]
    d = PREF_BETA * h
    if c["loss"] == "logistic":
        each = torch.log1p(torch.exp(-d.abs())) + torch.clamp(-d, min=0.0)
        g = -PREF_BETA / (1 + torch.exp(d))
    elif c["loss"] == "hinge":
        each = torch.clamp(1 - d, min=0.0)
        g = torch.where(d < 1, -PREF_BETA, 0.0).to(logp.dtype)
    else:
        each = (h - 1 / (2 * PREF_BETA)).square()
        g = 2 * (h - 1 / (2 * PREF_BETA))
    coef = logp.new_zeros(S).index_add_(0, pair[:, 0], g / P).index_add_(0, pair[:, 1], -g / P)
    loss = torch.stack([each.mean(), (d > 0).to(logp.dtype).mean(),
                        PREF_BETA * ratio[pair[:, 0]].mean(),
                        PREF_BETA * ratio[pair[:, 1]].mean()])
    return dict(loss=loss, ratio=ratio, pair_loss=each, dlogp=keep * (coef * scale)[seg])


def _plain_preference(s):
    return _pair_loss(s["case"], s["off"], s["n"], s["logp"], s["ref"], s["mask"], s["pair"])


def _router_loss(c, z, sel, mask):
    N, E = z.shape
    keep = _live(mask, z[:, 0])
    hits = keep[:, None].expand_as(sel).reshape(-1).to(torch.int64)
    counts = torch.zeros(E, dtype=torch.int64, device=z.device).index_add_(
        0, sel.reshape(-1).long(), hits)
    valid = keep.sum().clamp(min=1).to(z.dtype)
    f = counts.to(z.dtype) * E / (sel.shape[1] * valid)
    e = torch.exp(z - z.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True) * keep[:, None].to(z.dtype)
    prob = p.sum(0) / valid
    grad = p * (f - (p * f).sum(1, keepdim=True)) * (_scale(c) * BALANCE_COEF / valid)
    return (BALANCE_COEF * (f * prob).sum()).reshape(1), counts, prob, grad


def _plain_balance(s):
    loss, counts, prob, grad = _router_loss(s["case"], s["z"].float(), s["sel"], s["mask"])
    return dict(loss=loss, dlogits=grad.to(s["z"].dtype), counts=counts, prob=prob)


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["kind"]](state)


# --- work ------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] in ("logprob", "policy_logits"):
        size = 4 if c["dtype"] == "f32" else 2
        live = c["rows"] * c["keep"]
        row = c["vocab"] * size
        rows = c["rows"] * (9 if c["keep"] < 1 else 8)  # target, mask, log-probability
        if c["kind"] == "policy_logits":  # logits in, gradient out, the tokens' scalars
            return {"bytes": live * row + c["rows"] * row + rows +
                    c["rows"] * (12 if c["ref"] else 8), "flops": 8 * live * c["vocab"]}
        if c["back"]:
            return {"bytes": live * row + c["rows"] * row + rows +
                    c["rows"] * (16 if c["entropy"] else 8), "flops": 4 * live * c["vocab"]}
        return {"bytes": live * row + rows + (4 * c["rows"] if c["entropy"] else 0),
                "flops": (5 if c["entropy"] else 3) * live * c["vocab"]}
    if c["kind"] == "policy":
        n = _tokens(c, c["seqs"])
        return {"bytes": n * (16 + 4 * c["ref"] + 8 * c["entropy"] + c["masked"]) +
                8 * c["seqs"] + 40, "flops": 20 * n}
    if c["kind"] == "preference":
        S = c["groups"] * c["size"]
        n, pairs = _tokens(c, S), S - c["groups"]
        # the gradient waits for the sums and needs the mask alone again
        return {"bytes": n * (8 + 4 * c["ref"] + c["masked"]) + 12 * S + 20 * pairs + 24,
                "flops": 2 * n + 20 * pairs}
    size = 4 if c["dtype"] == "f32" else 2
    return {"bytes": c["rows"] * (2 * c["experts"] * size + 4 * c["top"] + c["masked"]) +
            12 * c["experts"] + 4, "flops": 10 * c["rows"] * c["experts"]}


# --- exact: the same from the definitions, in 64 bits ---------------------------------
def _exact_rows(z, target, live, T):
    """(logp, entropy, m, S) of some rows."""
    x = z.double()
    m = x.max(1).values
    y = (x - m[:, None]) / T
    S = y.exp().sum(1)
    h = S.log() - torch.nan_to_num(y, neginf=0.0).mul(y.exp()).sum(1) / S
    logp = y.gather(1, target.long()[:, None])[:, 0] - S.log()
    return logp.masked_fill(~live, 0), h.masked_fill(~live, 0), m, S


def _exact_logits_grad(z, target, live, T, m, lnS, dlogp, h=None, dh=None):
    """dz = (g (1[j = t] - p) - dh p (ln p + h)) / T, row by row, in z's type."""
    logq = (z.double() - m[:, None]) / T - lnS[:, None]
    p = logq.exp()
    grad = -dlogp[:, None] * p
    if h is not None:
        grad -= dh[:, None] * p * (torch.nan_to_num(logq, neginf=0.0) + h[:, None])
    grad[torch.arange(z.shape[0]), target.long()] += dlogp
    return (grad / T).masked_fill(~live[:, None], 0)


def _by_rows(f, n, *arrays):
    """f over runs of rows (a 64-bit copy of all the logits would be large)."""
    parts = [f(*(a[i:i + 512] for a in arrays)) for i in range(0, n, 512)]
    if isinstance(parts[0], tuple):
        return tuple(torch.cat(v) for v in zip(*parts))
    return torch.cat(parts)


def _exact_logprob(c, seed):
    g, z, target, mask = _logits_inputs(c, seed)
    T, R = c["temperature"], c["rows"]
    live = _live(mask, target)
    if not c["back"]:
        logp, h, _, _ = _by_rows(lambda a, t, v: _exact_rows(a, t, v, T), R, z, target, live)
        return dict(logp=logp, entropy=h) if c["entropy"] else dict(logp=logp)
    parts = [_forward_of(part, t, T) for part, t in zip(z.split(512), target.split(512))]
    m, S, h = (torch.cat(v).double() for v in zip(*parts))  # the 32-bit ones that are handed on
    dlogp, dh = _upstream(c, g)
    dlogp = dlogp.double()
    if c["entropy"]:
        return dict(dlogits=_by_rows(
            lambda a, t, v, m, s, d, h, e: _exact_logits_grad(a, t, v, T, m, s, d, h, e), R, z,
            target, live, m, S.log(), dlogp, h, dh.double()))
    return dict(dlogits=_by_rows(lambda a, t, v, m, s, d: _exact_logits_grad(
        a, t, v, T, m, s, d), R, z, target, live, m, S.log(), dlogp))


def _exact_tokens(c, logp, old, ref, adv, entropy, live, off):
    logp, old, adv = logp.double()[live], old.double()[live], adv.double()[live]
    n, S = logp.numel(), off.numel() - 1
    seg = _sequences_of(off, live.numel())[live]
    if c["reduce"] == "token_mean":
        w = torch.full_like(logp, 1 / max(n, 1))
    else:
        per = torch.bincount(seg, minlength=S)
        w = 1 / (S * per[seg].double()) if c["reduce"] == "seq_mean" else \
            torch.full_like(logp, 1 / S)
    d = logp - old
    r = d.exp()
    over = (adv > 0) & (r > 1 + CLIP_HIGH)
    under = (adv < 0) & (r < 1 - CLIP_LOW)
    dual = (adv < 0) & (r > DUAL_CLIP)
    pg, dpg = -r * adv, -r * adv
    for which, at in ((over, 1 + CLIP_HIGH), (under, 1 - CLIP_LOW), (dual, DUAL_CLIP)):
        pg, dpg = torch.where(which, -at * adv, pg), dpg.masked_fill(which, 0.0)
    total, grad = (w * pg).sum(), w * dpg
    parts = [total, torch.zeros_like(total), torch.zeros_like(total)]
    if ref is not None:
        q = ref.double()[live] - logp
        parts[1] = (w * (q.expm1() - q)).sum()
        total, grad = total + KL_COEF * parts[1], grad - KL_COEF * w * q.expm1()
    dh = None
    if entropy is not None:
        parts[2] = (w * entropy.double()[live]).sum()
        total = total - ENTROPY_COEF * parts[2]
        dh = torch.zeros_like(live, dtype=torch.float64)
        dh[live] = -ENTROPY_COEF * w
    k = max(n, 1)
    loss = torch.stack([total, *parts, over.sum() / k, (under | dual).sum() / k, r.sum() / k,
                        (d.expm1() - d).sum() / k])
    dlogp = torch.zeros_like(live, dtype=torch.float64)
    dlogp[live] = grad
    return loss, _scale(c) * dlogp, None if dh is None else _scale(c) * dh


def _exact_policy(c, seed):
    off, n, logp, old, ref, adv, mask, entropy = _token_inputs(c, seed)
    loss, dlogp, dh = _exact_tokens(c, logp, old, ref, adv, entropy, _live(mask, logp), off)
    return dict(loss=loss, dlogp=dlogp, **(dict(dentropy=dh) if c["entropy"] else {}))


def _exact_policy_logits(c, seed):
    z, target, mask, off, old, ref, adv = _row_inputs(c, seed)
    R, T, live = c["rows"], c["temperature"], _live(mask, target)
    logp, h, m, S = _by_rows(lambda a, t, v: _exact_rows(a, t, v, T), R, z, target, live)
    loss, dlogp, dh = _exact_tokens(c, logp, old, ref, adv, h if c["entropy"] else None, live,
                                    off)
    if not c["entropy"]:
        dh = torch.zeros_like(dlogp)
    grad = _by_rows(lambda a, t, v, m, s, d, h, e: _exact_logits_grad(a, t, v, T, m, s, d, h, e),
                    R, z, target, live, m, S.log(), dlogp, h, dh)
    return dict(loss=loss, logp=logp, dlogits=grad)


def _exact_preference(c, seed):
    off, n, logp, ref, mask, pair = _pair_inputs(c, seed)
    S, P = off.numel() - 1, pair.shape[0]
    live = _live(mask, logp)
    seg = _sequences_of(off, n)[live]
    x = (logp.double() - (ref.double() if ref is not None else 0.0))[live]
    count = torch.bincount(seg, minlength=S).clamp(min=1).double()
    sums = torch.zeros(S, dtype=torch.float64, device="cuda").scatter_add_(0, seg, x)
    u = sums / count if c["average"] else sums
    chosen, rejected = u[pair[:, 0]], u[pair[:, 1]]
    h = chosen - rejected
    if c["loss"] == "logistic":
        each = -torch.nn.functional.logsigmoid(PREF_BETA * h)
        g = -PREF_BETA * torch.sigmoid(-PREF_BETA * h)
    elif c["loss"] == "hinge":
        each = (1 - PREF_BETA * h).clamp(min=0)
        g = -PREF_BETA * (PREF_BETA * h < 1).double()
    else:
        each = (h - 0.5 / PREF_BETA)**2
        g = 2 * h - 1 / PREF_BETA
    by = torch.zeros(S, dtype=torch.float64, device="cuda")
    by.scatter_add_(0, pair[:, 0], g / P)
    by.scatter_add_(0, pair[:, 1], -g / P)
    if c["average"]:
        by = by / count
    dlogp = torch.zeros(n, dtype=torch.float64, device="cuda")
    dlogp[live] = by[seg]
    loss = torch.stack([each.sum() / P, (h > 0).sum() / P, PREF_BETA * chosen.sum() / P,
                        PREF_BETA * rejected.sum() / P])
    return dict(loss=loss, ratio=u, pair_loss=each, dlogp=dlogp)


def _exact_balance(c, seed):
    z, sel, mask = _router_inputs(c, seed)
    live = _live(mask, z[:, 0])
    N, E = max(int(live.sum()), 1), c["experts"]
    p = torch.softmax(z.double(), 1) * live[:, None]
    f = torch.bincount(sel[live].reshape(-1).long(), minlength=E).double() * E / (c["top"] * N)
    prob = p.sum(0) / N
    grad = _scale(c) * BALANCE_COEF / N * p * (f - (p @ f)[:, None])
    return dict(loss=BALANCE_COEF * (f * prob).sum().reshape(1), dlogits=grad, counts=None,
                prob=prob)


def exact(case, seed):
    return globals()["_exact_" + case["kind"]](case, seed)
