"""The learner's losses over a packed batch, written out from their definitions
in 64 bits (test infrastructure only; the library never uses it).

Inputs are numpy arrays (float64 values of whatever type the caller has);
`keep` is the boolean mask of the tokens that count, `off` the sequences'
offsets.  Gradients are the formulas'; tests/test_oracle_losses.py checks them
against differences of the losses themselves.
"""
import math

import numpy as np

TOKEN_MEAN, SEQ_MEAN, SEQ_SUM = range(3)
K1, K2, K3 = range(3)
LOGISTIC, SQUARE, HINGE = range(3)


def token_logprob(z, target, temperature=1.0):
    """(logp, entropy, m, S) of rows z with a finite logit each."""
    z = np.asarray(z, np.float64)
    m = z.max(1)
    y = (z - m[:, None]) / temperature
    e = np.exp(y)
    S = e.sum(1)
    logp = y[np.arange(len(z)), target] - np.log(S)
    H = np.log(S) - (e * np.where(e > 0, y, 0.0)).sum(1) / S
    return logp, H, m, S


def token_logprob_grad(z, target, dlogp, dentropy=None, temperature=1.0):
    z = np.asarray(z, np.float64)
    _, H, m, S = token_logprob(z, target, temperature)
    lnp = (z - m[:, None]) / temperature - np.log(S)[:, None]
    p = np.exp(lnp)
    d = -np.asarray(dlogp, np.float64)[:, None] * p
    d[np.arange(len(z)), target] += dlogp
    if dentropy is not None:
        d -= np.asarray(dentropy, np.float64)[:, None] * p * (
            np.where(p > 0, lnp, 0.0) + H[:, None])
    return d / temperature


def sequences(off, n):
    """The sequence of each of n tokens, -1 outside all."""
    s = np.full(n, -1)
    for i in range(len(off) - 1):
        s[int(off[i]):min(int(off[i + 1]), n)] = i
    return s


def policy(logp, old, adv, keep, off=None, ref=None, entropy=None, low=0.2, high=0.2, dual=0.0,
           kl_coef=0.0, kl=K3, entropy_coef=0.0, reduce=TOKEN_MEAN, norm=0.0, grad_scale=1.0):
    """(loss[8], dlogp, dentropy)."""
    n = len(logp)
    keep = np.asarray(keep, bool).copy()
    seq = sequences(off, n) if off is not None else np.zeros(n, int)
    keep &= seq >= 0
    n_seq = len(off) - 1 if off is not None else 1
    out, dlogp, dent = np.zeros(8), np.zeros(n), np.zeros(n)
    tokens = int(keep.sum())
    per = np.bincount(seq[keep], minlength=n_seq)
    for t in np.flatnonzero(keep):
        w = 1 / ((norm or n_seq) * per[seq[t]]) if reduce == SEQ_MEAN else \
            1 / (norm or (tokens if reduce == TOKEN_MEAN else n_seq))
        A, d = float(adv[t]), float(logp[t]) - float(old[t])
        r = math.exp(d)
        pg = -min(r * A, min(max(r, 1 - low), 1 + high) * A)
        if dual and A < 0:
            pg = min(pg, -dual * A)
        above = A > 0 and r > 1 + high
        below = A < 0 and (r < 1 - low or (dual > 0 and r > dual))
        g = 0.0 if above or below else -r * A
        k = gk = 0.0
        if ref is not None:
            q = float(ref[t]) - float(logp[t])
            k = (-q, q * q / 2, math.expm1(q) - q)[kl]
            gk = (1.0, -q, -math.expm1(q))[kl]
        h = float(entropy[t]) if entropy is not None else 0.0
        out[:4] += w * np.array([pg + kl_coef * k - entropy_coef * h, pg, k, h])
        out[4:] += np.array([above, below, r, math.expm1(d) - d]) / tokens
        dlogp[t] = grad_scale * w * (g + kl_coef * gk)
        dent[t] = -grad_scale * w * entropy_coef
    return out, dlogp, dent


def preference(logp, ref, keep, off, pair, beta, kind=LOGISTIC, smooth=0.0, margin=0.0,
               average=False, norm=0.0, grad_scale=1.0):
    """(loss[4], u, pair losses, dlogp); a pair with an index out of range adds
    nothing."""
    n, S = len(logp), len(off) - 1
    x = np.asarray(logp, np.float64) - (0.0 if ref is None else np.asarray(ref, np.float64))
    seq = sequences(off, n)
    keep = np.asarray(keep, bool) & (seq >= 0)
    count = np.bincount(seq[keep], minlength=S)
    u = np.array([math.fsum(x[keep & (seq == s)]) for s in range(S)])
    scale = 1 / np.maximum(count, 1) if average else np.ones(S)
    u = u * scale
    each, by, out = np.zeros(len(pair)), np.zeros(S), np.zeros(4)
    norm = norm or len(pair)
    for i, (c, r) in enumerate(pair):
        if not (0 <= c < S and 0 <= r < S):
            continue
        h = u[c] - u[r]
        d = beta * h - margin
        if kind == LOGISTIC:
            up, down = np.logaddexp(0, -d), np.logaddexp(0, d)
            each[i] = (1 - smooth) * up + smooth * down
            # s(-d) (1 - e) - s(d) e
            g = -beta * ((1 - smooth) * math.exp(-down) - smooth * math.exp(-up))
        elif kind == HINGE:
            each[i], g = max(0.0, 1 - d), -beta if d < 1 else 0.0
        else:
            y = h - 1 / (2 * beta)
            each[i], g = y * y, 2 * y
        by[c] += g
        by[r] -= g
        out += np.array([each[i] / norm, (h > 0) / len(pair), beta * u[c] / len(pair),
                         beta * u[r] / len(pair)])
    dlogp = np.where(keep, grad_scale / norm * (by * scale)[seq], 0.0)
    return out, u, each, dlogp


def balance(z, sel, keep, coef, grad_scale=1.0):
    """(loss, counts, prob, dlogits); rows of -infinity alone have p = 0."""
    z = np.asarray(z, np.float64)
    rows, E = z.shape
    keep = np.asarray(keep, bool)
    N = max(int(keep.sum()), 1)
    counts = np.zeros(E, np.int64)
    for t in np.flatnonzero(keep):
        for e in sel[t]:
            if 0 <= e < E:
                counts[e] += 1
    p = np.zeros((rows, E))
    for t in np.flatnonzero(keep):
        m = z[t].max()
        if m > -np.inf:
            e = np.exp(z[t] - m)
            p[t] = e / e.sum()
    f = E * counts / (sel.shape[1] * N)
    prob = p.sum(0) / N
    grad = grad_scale * coef / N * p * (f - (p @ f)[:, None])
    return coef * float(f @ prob), counts, prob, grad


FORWARD, REVERSE, MIX = range(3)


def token_top(z, top, temperature=1.0):
    """(ids, logp, rest) of rows z with a finite logit each: the largest first, ties
    by their index; -1 and -inf where no token with a probability is left."""
    z = np.asarray(z, np.float64)
    ids, logp = np.full((len(z), top), -1), np.full((len(z), top), -np.inf)
    rest = np.full(len(z), -np.inf)
    for t, row in enumerate(z):
        order = np.lexsort((np.arange(len(row)), -row))[:top]
        order = order[row[order] > -np.inf]
        y = (row - row.max()) / temperature
        ln = np.log(np.exp(y).sum())
        ids[t, :len(order)], logp[t, :len(order)] = order, y[order] - ln
        out = np.delete(y, order)
        out = out[out > -np.inf]
        if len(out):  # relative to its own maximum: none of it is lost beside the list
            rest[t] = out.max() + np.log(np.exp(out - out.max()).sum()) - ln
    return ids, logp, rest


def weights(keep, off=None, reduce=TOKEN_MEAN, norm=0.0):
    """What each of the tokens weighs in the batch's loss."""
    keep = np.asarray(keep, bool).copy()
    n = len(keep)
    seq = sequences(off, n) if off is not None else np.zeros(n, int)
    keep &= seq >= 0
    n_seq = len(off) - 1 if off is not None else 1
    per = np.bincount(seq[keep], minlength=n_seq)
    w = np.zeros(n)
    for t in np.flatnonzero(keep):
        w[t] = 1 / ((norm or n_seq) * per[seq[t]]) if reduce == SEQ_MEAN else \
            1 / (norm or (keep.sum() if reduce == TOKEN_MEAN else n_seq))
    return w


def _log_sum(x):
    x = x[x > -np.inf]
    return x.max() + np.log(np.exp(x - x.max()).sum()) if len(x) else -np.inf


def _times(w, log):
    return np.where(w == 0, 0.0, w * np.where(w == 0, 0.0, log))


def distill_row(z, ids, value, rest=None, kind=FORWARD, beta=0.0, temperature=1.0,
                teacher_temperature=1.0):
    """(loss, d loss / d z) of one row with a finite logit."""
    z = np.asarray(z, np.float64)
    x = z / temperature
    lnq = x - _log_sum(x)
    q = np.exp(lnq)
    here = [k for k in range(len(ids)) if ids[k] >= 0 and value[k] > -np.inf]
    at = np.array([ids[k] for k in here], int)
    lp = np.array([value[k] for k in here], np.float64)
    others = np.delete(np.arange(len(z)), at)
    if rest is None:
        lp = lp / teacher_temperature
        lp = lp - _log_sum(lp) if len(lp) else lp
        lp = np.append(lp, -np.inf)
    else:
        lp = np.append(lp, rest)
    lq = np.append(lnq[at], _log_sum(lnq[others]))
    P, Q = np.exp(lp), np.exp(lq)
    cls = np.full(len(z), len(here))
    cls[at] = np.arange(len(here))
    with np.errstate(all="ignore"):
        if kind == FORWARD:
            loss, qf = _times(P, lp - lq).sum(), -P
        elif kind == REVERSE:
            loss = _times(Q, lq - lp).sum()
            qf = _times(Q, lq - lp + 1)
        else:
            m = np.logaddexp(np.log(beta) + lp, np.log1p(-beta) + lq)
            qf = (1 - beta) * _times(Q, lq - m)
            loss = beta * _times(P, lp - m).sum() + qf.sum()
        # q_j f'_b = (q_j / Q_b) (Q_b f'_b): a token's share of its class
        share = np.where(lq[cls] > -np.inf, np.exp(lnq - lq[cls]), 0.0)
        share[at] = 1.0
        return loss, (share * qf[cls] - q * qf.sum()) / temperature


def distill(z, ids, value, rest, keep, off=None, kind=FORWARD, beta=0.0, reduce=TOKEN_MEAN,
            norm=0.0, temperature=1.0, teacher_temperature=1.0, grad_scale=1.0):
    """(loss, row losses, gradient of the logits)."""
    z = np.asarray(z, np.float64)
    w = weights(keep, off, reduce, norm)
    each, grad = np.zeros(len(z)), np.zeros_like(z)
    for t in np.flatnonzero(w):
        each[t], g = distill_row(z[t], ids[t], value[t], None if rest is None else rest[t], kind,
                                 beta, temperature, teacher_temperature)
        grad[t] = grad_scale * w[t] * g
    return float((w * each)[w > 0].sum()), each, grad
