"""A teacher's lists of likely tokens and the distillation loss on them, as cases
that can be timed.

Beside the losses of a packed batch, a post-training program that learns from a
teacher goes through these operators:

* top     -- the likeliest tokens of each row of logits with their
             log-probabilities, the log-probability of a given token, the entropy
             and the logarithm of what is outside of the list: what an actor reports
             while it generates, and what a teacher leaves for its students;
* distill -- the divergence between a teacher's list and the student's logits,
             reduced over the batch, and the gradient of the logits.

With `own` false the same is computed from elementary torch operations in 32
bits.  Inputs come from the seed alone.
"""
import math

import torch

own = False

DTYPES = dict(bf16=torch.bfloat16, f16=torch.float16, f32=torch.float32)
BETA = 0.5       # weight of the teacher in the mixture
SCALE = 1024.0   # gradients that are kept in 16 bits with 5 bits of exponent


def listed():
    return [
        # serving: an actor samples one token and reports 20 alternatives; some
        # tokens are excluded by its sampler
        dict(name="top_one_token", kind="top", rows=1, vocab=152_064, pad=0, dtype="bf16", top=20,
             keep=1.0, entropy=False, temperature=0.7, banned=64),
        # a decoding step of 256 sequences over a small vocabulary of an odd size
        dict(name="top_step_256", kind="top", rows=256, vocab=32_003, pad=0, dtype="f16", top=8,
             keep=1.0, entropy=True, temperature=0.9, banned=5),
        # a teacher scores a micro-batch of responses; a tenth are prompt tokens
        dict(name="top_teacher_8192", kind="top", rows=8_192, vocab=152_064, pad=0, dtype="bf16",
             top=64, keep=0.9, entropy=True, temperature=1.0, banned=0),
        # long lists from 32-bit logits, rows at every alignment
        dict(name="top_odd_f32", kind="top", rows=777, vocab=32_003, pad=0, dtype="f32", top=128,
             keep=1.0, entropy=False, temperature=1.0, banned=64),
        # one micro-batch of a few short responses: launches and latency
        dict(name="distill_16", kind="distill", rows=16, seqs=2, vocab=32_003, pad=0, dtype="bf16",
             top=20, divergence="forward", rest=False, back=True, keep=1.0,
             reduce="token_mean", temperature=1.0),
        # the learner's step on a micro-batch: the whole of the teacher's distribution,
        # its list and one class for all else
        dict(name="distill_8192", kind="distill", rows=8_192, seqs=12, vocab=152_064, pad=0,
             dtype="bf16", top=64, divergence="forward", rest=True, back=True, keep=0.9,
             reduce="token_mean", temperature=1.0),
        # a teacher's raw top logits at a higher temperature, each response alike
        dict(name="distill_warm_4096", kind="distill", rows=4_096, seqs=9, vocab=152_064, pad=0,
             dtype="f16", top=32, divergence="forward", rest=False, back=True, keep=1.0,
             reduce="seq_mean", temperature=2.0),
        # on the student's own responses: the divergence that avoids what the teacher excludes
        dict(name="distill_reverse_4096", kind="distill", rows=4_096, seqs=16, vocab=152_064,
             pad=0, dtype="bf16", top=128, divergence="reverse", rest=True, back=True, keep=0.9,
             reduce="token_mean", temperature=1.0),
        # between the two, in 32 bits over a small vocabulary of an odd size
        dict(name="distill_mix_odd", kind="distill", rows=515, seqs=9, vocab=32_003, pad=0,
             dtype="f32", top=100, divergence="mix", rest=True, back=True, keep=0.8,
             reduce="seq_sum", temperature=1.0),
        # evaluation of a student: the loss without a gradient
        dict(name="distill_eval_2048", kind="distill", rows=2_048, seqs=7, vocab=152_064, pad=0,
             dtype="bf16", top=20, divergence="forward", rest=True, back=False, keep=1.0,
             reduce="token_mean", temperature=1.0),
    ]


# --- draws ---------------------------------------------------------------------
_LOGITS = 1_245_708_288  # elements of the largest listed logits


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_shape(rng):
    vocab = rng.choice([152_064, 32_000, _log(rng, 500, 262_144), _log(rng, 500, 262_144)])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    most = _LOGITS // vocab // (2 if dtype == "f32" else 1)
    return dict(rows=_log(rng, 1, min(8_192, most)), vocab=vocab, dtype=dtype,
                pad=rng.choice([0, 0, -vocab % 64]), keep=rng.choice([1.0, 0.9, 0.5]),
                top=rng.choice([1, 8, 20, 64, 128, _log(rng, 1, 128)]))


def _draw_top(rng):
    return dict(kind="top", **_draw_shape(rng), entropy=rng.random() < 0.5,
                temperature=rng.choice([1.0, 1.0, 0.7]), banned=rng.choice([0, 0, 1, 64]))


def _draw_distill(rng):
    c = dict(kind="distill", **_draw_shape(rng))
    c["seqs"] = _log(rng, 1, max(1, c["rows"] // 4))
    c["divergence"] = rng.choice(["forward", "forward", "forward", "reverse", "mix"])
    c["rest"] = c["divergence"] != "forward" or rng.random() < 0.5
    c["back"] = rng.random() < 0.8
    c["reduce"] = rng.choice(["token_mean", "seq_mean", "seq_sum"])
    c["temperature"] = rng.choice([1.0, 1.0, 2.0])
    return c


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        c = rng.choice([_draw_top, _draw_distill])(rng)
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


def _bulk(c, g):
    """Logits of a wide bulk, the log-sum of whose exponentials is ln V + 3.1."""
    z = torch.empty(c["rows"], c["vocab"] + c["pad"], dtype=DTYPES[c["dtype"]], device="cuda")
    z.normal_(0.0, 2.5 * c["temperature"], generator=g)
    return z[:, :c["vocab"]]


def _distinct(g, R, V, K):
    """K different tokens a row, in any order: one of each of K stretches of the vocabulary."""
    ends = torch.arange(K + 1, device="cuda") * V // K
    wide = ends[1:] - ends[:-1]
    ids = ends[:-1] + torch.minimum((_uniform(g, R, K) * wide).long(), wide - 1)
    return ids.gather(1, _uniform(g, R, K).argsort(1))


def _mask_of(c, g):
    return (_uniform(g, c["rows"]) < c["keep"]).to(torch.uint8) if c["keep"] < 1 else None


def _top_inputs(c, seed):
    """Logits as a language model gives them (a bulk and some likely tokens, the given
    one most often among them); excluded tokens are at -infinity."""
    g = _gen(seed)
    R, V, T = c["rows"], c["vocab"], c["temperature"]
    z = _bulk(c, g)
    target = torch.randint(0, V, (R,), generator=g, device="cuda")
    z.scatter_(1, _distinct(g, R, V, 12), (T * (math.log(V) + 1 + 2 * _normal(g, R, 12))).to(z.dtype))
    z.scatter_(1, target[:, None], (T * (math.log(V) + 3 + _normal(g, R, 1))).to(z.dtype))
    if c["banned"]:
        ban = torch.randint(0, V, (R, c["banned"]), generator=g, device="cuda")
        ban = torch.where(ban == target[:, None], (ban + 1) % V, ban)
        z.scatter_(1, ban, -math.inf)
    return z, target.to(torch.int32), _mask_of(c, g)


def _distill_inputs(c, seed):
    """A teacher's lists, likeliest token first, and a student's logits that know most of
    it.  One list in eight is shorter than the others (the teacher excluded the rest)."""
    g = _gen(seed)
    R, V, K, T = c["rows"], c["vocab"], c["top"], c["temperature"]
    z = _bulk(c, g)
    ids = _distinct(g, R, V, K)
    steps = 1.3 * torch.log1p(torch.arange(K, device="cuda", dtype=torch.float32))
    value = (-steps + 0.5 * _normal(g, R, K)).sort(1, descending=True)[0]
    z.scatter_(1, ids, (T * (math.log(V) + 4 + value + 0.8 * _normal(g, R, K))).to(z.dtype))
    n = torch.where(_uniform(g, R) < 0.125, (1 + (K - 1) * _uniform(g, R)).long(), K)
    absent = torch.arange(K, device="cuda") >= n[:, None]
    value = value.double().masked_fill(absent, -math.inf)
    rest = None
    if c["rest"]:  # the list's log-probabilities, and the logarithm of what they leave
        rest = -0.3 - 6 * _uniform(g, R).double()
        value = value - torch.logsumexp(value, 1, keepdim=True) + torch.log1p(-rest.exp())[:, None]
        rest = rest.float()
    else:  # logits, as they came out of the teacher
        value = T * (value + 12 + 2 * _normal(g, R, 1))
    ids = ids.masked_fill(absent, -1).to(torch.int32)
    cuts = torch.sort(torch.randint(0, R + 1, (c["seqs"] - 1,), generator=g, device="cuda"))[0]
    off = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), R)])
    return z, ids, value.float(), rest, _mask_of(c, g), off


def _scale(c):
    return SCALE if c["dtype"] == "f16" else 1.0


# --- prepare ---------------------------------------------------------------------
def _like(z):
    return torch.zeros(z.shape[0], z.stride(0), dtype=z.dtype, device="cuda")[:, :z.shape[1]]


def _prepare_top(c, seed):
    z, target, mask = _top_inputs(c, seed)
    R, K = c["rows"], c["top"]
    out = dict(ids=torch.zeros(R, K, dtype=torch.int32, device="cuda"),
               top_logp=torch.zeros(R, K, device="cuda"), logp=torch.zeros(R, device="cuda"),
               rest=torch.zeros(R, device="cuda"))
    if c["entropy"]:
        out["entropy"] = torch.zeros(R, device="cuda")
    return dict(z=z, target=target, mask=mask, out=out)


def _prepare_distill(c, seed):
    z, ids, value, rest, mask, off = _distill_inputs(c, seed)
    out = dict(loss=torch.zeros(1, device="cuda"), row_loss=torch.zeros(c["rows"], device="cuda"))
    if c["back"]:
        out["dlogits"] = _like(z)
    return dict(z=z, ids=ids, value=value, rest=rest, mask=mask, off=off, out=out)


_ring = None


def _ctx():
    """A context of the library; its ring is not used."""
    global _ring
    if _ring is None:
        from paper_2609_24456_gb300 import edp
        cfg = edp.make_config(64, (1, 16, 16), edp.EDP_XFORM_CHW_NORM_BF16)
        _ring = edp.Ring(cfg, action=False, reward=False, done=False)
    return _ring.ctx


def prepare(case, seed):
    s = dict(globals()["_prepare_" + case["kind"]](case, seed), case=case)
    if own:
        _ctx()
    return s


# --- run: the framework's calls ----------------------------------------------------
def _own_top(s):
    from paper_2609_24456_gb300 import edp
    o = s["out"]
    edp.edp_token_top(_ctx(), s["z"], o["ids"], o["top_logp"], target=s["target"],
                      logp=o["logp"], mask=s["mask"], temperature=s["case"]["temperature"],
                      entropy=o.get("entropy"), rest=o["rest"])
    return o


def _own_distill(s):
    from paper_2609_24456_gb300 import edp
    c, o = s["case"], s["out"]
    cfg = edp.make_distill_config(
        kind=getattr(edp, "EDP_DISTILL_" + c["divergence"].upper()),
        reduce=getattr(edp, "EDP_REDUCE_" + c["reduce"].upper()),
        beta=BETA if c["divergence"] == "mix" else 0.0,
        teacher_temperature=1.0 if c["rest"] else c["temperature"], grad_scale=_scale(c))
    edp.edp_distill_loss(_ctx(), cfg, s["z"], s["ids"], s["value"], o["loss"], rest=s["rest"],
                         mask=s["mask"], off=s["off"], n_seq=c["seqs"],
                         temperature=c["temperature"], row_loss=o["row_loss"],
                         dlogits=o.get("dlogits"))
    return o


# --- run: the plain form -------------------------------------------------------------
def _live(mask, rows, device):
    return mask.bool() if mask is not None else torch.ones(rows, dtype=torch.bool, device=device)


def _likeliest(z, k):
    """The k largest of each row, ties to the lowest index: the order of the bits of fp32
    numbers in the upper half of a key, the index counted down in the lower."""
    bits = (z.float() + 0.0).view(torch.int32)  # -0 is 0
    order = bits ^ ((bits >> 31) & 0x7fffffff)
    places = torch.arange(z.shape[1], device=z.device)
    key = (order.long() << 32) | (0xffffffff - places)
    return 0xffffffff - (key.topk(k, 1)[0] & 0xffffffff)


def _log_softmax(x):
    y = x - x.amax(1, keepdim=True)
    return y - torch.log(torch.exp(y).sum(1, keepdim=True))


def _log_sum_exp(x):
    m = x.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    return torch.log(torch.exp(x - m).sum(1)) + m[:, 0]


def _plain_top(s):
    c, z, T = s["case"], s["z"], s["case"]["temperature"]
    live = _live(s["mask"], c["rows"], z.device)
    ids = torch.cat([_likeliest(part, c["top"]) for part in z.split(512)])
    logq = _log_softmax(z.float() / T)
    top_logp = logq.gather(1, ids)
    logp = logq.gather(1, s["target"].long()[:, None])[:, 0]
    zero = torch.zeros_like(logp)
    out = dict(ids=torch.where(live[:, None], ids, -1).to(torch.int32),
               top_logp=torch.where(live[:, None], top_logp, -math.inf),
               logp=torch.where(live, logp, zero))
    if c["entropy"]:
        p = torch.exp(logq)
        h = -torch.where(p > 0, p * logq, torch.zeros_like(p)).sum(1)
        out["entropy"] = torch.where(live, h, zero)
    rest = _log_sum_exp(logq.scatter_(1, ids, -math.inf))
    out["rest"] = torch.where(live, rest, zero)
    return out


def _weights(c, live, off):
    keep, S, n = live.float(), off.numel() - 1, live.numel()
    if c["reduce"] == "token_mean":
        return keep / keep.sum().clamp(min=1)
    if c["reduce"] == "seq_sum":
        return keep / S
    seq = torch.searchsorted(off[1:], torch.arange(n, device=off.device), right=True)
    per = torch.zeros(S, device=off.device).index_add_(0, seq, keep)
    return keep / (S * per.clamp(min=1))[seq]


def _plain_distill(s):
    c, T = s["case"], s["case"]["temperature"]
    live = _live(s["mask"], c["rows"], s["z"].device)
    w = _weights(c, live, s["off"])
    absent = s["ids"] < 0
    first = s["ids"][:, :1].long()
    at = torch.where(absent, first, s["ids"].long())  # the first entry is always there
    if c["rest"]:
        lp, lpr = s["value"], s["rest"]
    else:
        lp, lpr = _log_softmax(s["value"] / T), None
    lp = torch.where(absent, -math.inf, lp)
    p = torch.exp(lp)
    x = s["z"].float() / T
    logq = _log_softmax(x)
    lq = logq.gather(1, at)
    q = torch.where(absent, torch.zeros_like(p), torch.exp(lq))
    lqr = _log_sum_exp(logq.scatter(1, at, -math.inf))
    qr, zero = torch.exp(lqr), torch.zeros_like(p)
    pr = torch.exp(lpr) if lpr is not None else torch.zeros_like(qr)

    def over(weight, log):  # sum of weight log over the classes that weigh
        return torch.where(weight > 0, weight * log, torch.zeros_like(weight))

    # each class's share of the loss, and q f' of its derivative f' by q
    if c["divergence"] == "forward":
        loss = over(p, lp - lq).sum(1)
        if lpr is not None:
            loss = loss + over(pr, lpr - lqr)
        qf, qfr = -p, -pr
    elif c["divergence"] == "reverse":
        each, rest = over(q, lq - lp), over(qr, lqr - lpr)
        loss = each.sum(1) + rest
        qf, qfr = each + q, rest + qr
    else:
        lm, lmr = torch.log(BETA * p + (1 - BETA) * q), torch.log(BETA * pr + (1 - BETA) * qr)
        qf, qfr = (1 - BETA) * over(q, lq - lm), (1 - BETA) * over(qr, lqr - lmr)
        loss = (BETA * over(p, lp - lm) + qf).sum(1) + BETA * over(pr, lpr - lmr) + qfr
    loss = torch.where(live, loss, torch.zeros_like(loss))
    out = dict(loss=(w * loss).sum().reshape(1), row_loss=loss)
    if c["back"]:
        both = qf.sum(1) + qfr
        by = _scale(c) * w / T
        grad = torch.exp(logq) * (by * (qfr / qr - both))[:, None]
        own_grad = by[:, None] * (qf - q * both[:, None])
        grad.scatter_(1, at, torch.where(absent, own_grad[:, :1], own_grad))
        out["dlogits"] = torch.where(live[:, None], grad, torch.zeros_like(grad)).to(s["z"].dtype)
    return out


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["kind"]](state)


# --- work ------------------------------------------------------------------------
def work(case):
    c = case
    row = c["vocab"] * (4 if c["dtype"] == "f32" else 2)
    live = c["rows"] * c["keep"]
    scalars = c["rows"] if c["keep"] < 1 else 0  # the mask
    lists = 8 * c["rows"] * c["top"]
    if c["kind"] == "top":
        scalars += c["rows"] * (16 if c["entropy"] else 12)
        return {"bytes": live * row + lists + scalars,
                "flops": (6 if c["entropy"] else 4) * live * c["vocab"]}
    scalars += c["rows"] * (8 if c["rest"] else 4) + 8 * (c["seqs"] + 1) + 4
    return {"bytes": live * row + (c["rows"] * row if c["back"] else 0) + lists + scalars,
            "flops": (8 if c["back"] else 4) * live * c["vocab"]}


# --- exact: the same from the definitions, in 64 bits ---------------------------------
def _exact_top_rows(z, target, live, c):
    K = c["top"]
    x = z.double()
    order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :K]
    logq = torch.log_softmax(x / c["temperature"], 1)
    q = logq.exp()
    outside = torch.ones_like(q).scatter_(1, order, 0.0)
    entropy = -(q * torch.nan_to_num(logq, neginf=0.0)).sum(1)
    dead = ~live
    return (order.masked_fill(dead[:, None], -1).to(torch.int32),
            logq.gather(1, order).masked_fill(dead[:, None], -math.inf),
            logq.gather(1, target.long()[:, None])[:, 0].masked_fill(dead, 0),
            (q * outside).sum(1).log().masked_fill(dead, 0), entropy.masked_fill(dead, 0))


def _by_rows(f, n, *arrays):
    """f over runs of rows (a 64-bit copy of all the logits would be large)."""
    parts = [f(*(a[i:i + 256] if a is not None else None for a in arrays))
             for i in range(0, n, 256)]
    return tuple(None if v[0] is None else torch.cat(v) for v in zip(*parts))


def _exact_top(c, seed):
    z, target, mask = _top_inputs(c, seed)
    live = torch.ones_like(target).bool() if mask is None else mask > 0
    ids, top_logp, logp, rest, h = _by_rows(lambda a, t, v: _exact_top_rows(a, t, v, c),
                                            c["rows"], z, target, live)
    out = dict(ids=ids, top_logp=top_logp, logp=logp, rest=rest)
    return dict(out, entropy=h) if c["entropy"] else out


def _exact_distill_rows(z, ids, value, rest, live, by, c):
    """The loss of some rows, from the classes' probabilities p and q as two matrices
    (class K is all that is not in the list), and the gradient by the chain rule through
    the softmax: (1/T) (q_j f'_j - q_j sum_i q_i f'_i)."""
    R, K, T = ids.shape[0], ids.shape[1], c["temperature"]
    here = ids >= 0
    rows = torch.arange(R, device=z.device)
    cls = torch.full(z.shape, K, dtype=torch.long, device=z.device)
    where = torch.nonzero(here)
    cls[where[:, 0], ids[here].long()] = where[:, 1]
    q = torch.softmax(z.double() / T, 1)
    Q = torch.zeros(R, K + 1, dtype=torch.float64, device=z.device).scatter_add_(1, cls, q)
    v = value.double().masked_fill(~here, -math.inf)
    if rest is not None:
        P = torch.cat([v, rest.double()[:, None]], 1).exp()
    else:
        P = torch.softmax(torch.cat([v / T, torch.full_like(v[:, :1], -math.inf)], 1), 1)
    if c["divergence"] == "forward":
        terms, d = torch.xlogy(P, P / Q), -P / Q
        terms, d = terms.masked_fill(P == 0, 0), d.masked_fill(P == 0, 0)
    elif c["divergence"] == "reverse":
        terms = torch.xlogy(Q, Q / P).masked_fill(Q == 0, 0)
        d = ((Q / P).log() + 1).masked_fill(Q == 0, 0)
    else:
        M = BETA * P + (1 - BETA) * Q
        terms = BETA * torch.xlogy(P, P / M).masked_fill(P == 0, 0) + \
            (1 - BETA) * torch.xlogy(Q, Q / M).masked_fill(Q == 0, 0)
        d = ((1 - BETA) * (Q / M).log()).masked_fill(Q == 0, 0)
    loss = terms.sum(1).masked_fill(~live, 0)
    if not c["back"]:
        return loss, None
    inner = (Q * d).sum(1)
    grad = q * (d[rows[:, None], cls] - inner[:, None]) * (by / T)[:, None]
    return loss, grad.masked_fill(~live[:, None], 0)


def _exact_distill(c, seed):
    z, ids, value, rest, mask, off = _distill_inputs(c, seed)
    R, S = c["rows"], off.numel() - 1
    live = torch.ones(R, dtype=torch.bool, device="cuda") if mask is None else mask > 0
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), off[1:] - off[:-1])
    if c["reduce"] == "token_mean":
        w = torch.full((R,), 1 / max(int(live.sum()), 1), dtype=torch.float64, device="cuda")
    elif c["reduce"] == "seq_mean":
        w = 1 / (S * torch.bincount(seq[live], minlength=S).clamp(min=1).double())[seq]
    else:
        w = torch.full((R,), 1 / S, dtype=torch.float64, device="cuda")
    w = w * live
    loss, grad = _by_rows(lambda *a: _exact_distill_rows(*a, c), R, z, ids, value, rest, live,
                          _scale(c) * w)
    out = dict(loss=(w * loss).sum().reshape(1), row_loss=loss)
    return dict(out, dlogits=grad) if c["back"] else out


def exact(case, seed):
    return globals()["_exact_" + case["kind"]](case, seed)
