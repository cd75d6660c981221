"""The policy, preference and balance losses on the GPU against the 64-bit oracle.

Bounds, with eps = 2^-24.  Policy: d = logp - old rounds once (eps |d|), e^d is
good to 2 eps and d's error, and a weight and a gradient take a few roundings
more: each token's loss and gradient are within 2e-6 of its terms' sizes, and
so are their sums (kept as pairs of fp32 numbers).  Preference: u is a sum of
at least 44 bits rounded once; the derivative of the logistic loss is good to
(4 + |d|) eps relatively.  Balance: p of E terms to 1e-6 (|z - m| below 20), sums
over rows of fp32 partial sums of at most a few hundred rows, to 1e-5 at worst.
"""
import numpy as np
import pytest
import torch

from gpu_util import cuda, to_np
from oracle import losses as L
from test_gpu_logprob import LEAST, TYPES, UNIT, check_grad, ctx_of, make, view

pytestmark = pytest.mark.gpu


def f32(x):
    return np.asarray(x, np.float32).astype(np.float64)


def offsets(rng, n_seq, lmax, empty=0.1):
    lens = rng.integers(1, lmax + 1, n_seq)
    lens[rng.random(n_seq) < empty] = 0
    if not lens.sum():
        lens[-1] = 1
    return np.concatenate([[0], np.cumsum(lens)])


def policy_case(rng, n, spread=.3):
    old = f32(-rng.exponential(1, n))
    return f32(old + rng.normal(0, spread, n)), old, f32(old + rng.normal(0, .3, n)), \
        f32(rng.normal(0, 1, n)), f32(rng.random(n))


def run_policy(edp, ring, kw, logp, old, adv, n, off=None, keep=None, ref=None, ent=None,
               grads=True, shift=0):
    def dev(x):  # `shift` elements off the storage's start
        if x is None:
            return None
        pad = np.concatenate([np.full(shift, np.nan), x, np.full(4, np.nan)]).astype(np.float32)
        return cuda(pad)[shift:shift + len(x)]

    mask = None
    if keep is not None:
        mask = cuda(np.concatenate([np.zeros(shift), keep, np.zeros(4)]).astype(np.uint8))[
            shift:shift + len(keep)]
    loss = torch.full((8,), 7.0, device="cuda")
    store = torch.full((2, shift + n + 8), 7.0, device="cuda")
    g, h = store[0, shift:shift + n], store[1, shift:shift + n]
    cfg = edp.make_policy_config(
        kw.get("low", .2), kw.get("high", .2), kw.get("dual", 0.0), kw.get("kl_coef", 0.0),
        kw.get("kl", L.K3), kw.get("entropy_coef", 0.0), kw.get("reduce", 0),
        kw.get("norm", 0.0), kw.get("grad_scale", 1.0))
    edp.edp_policy_loss(ring.ctx, cfg, dev(logp), dev(old), dev(adv), n, loss, ref_logp=dev(ref),
                        mask=mask, off=cuda(np.asarray(off, np.uint64)) if off is not None else
                        None, n_seq=len(off) - 1 if off is not None else 0, entropy=dev(ent),
                        dlogp=g if grads else None, dentropy=h if grads else None)
    edp.edp_sync(ring.ctx)
    assert (store[:, :shift] == 7).all() and (store[:, shift + n:] == 7).all()
    return to_np(loss), to_np(g), to_np(h)


def policy_sizes(kw, logp, old, adv, keep, off, ref, ent):
    """Per token: its terms' sizes with its weight; the sums' bounds."""
    n = len(logp)
    keep = np.ones(n, bool) if keep is None else np.asarray(keep, bool)
    seq = L.sequences(off, n) if off is not None else np.zeros(n, int)
    keep = keep & (seq >= 0)
    S = len(off) - 1 if off is not None else 1
    norm, tokens = kw.get("norm", 0.0), max(int(keep.sum()), 1)
    per = np.maximum(np.bincount(seq[keep], minlength=S), 1)
    w = (1 / ((norm or S) * per[seq]) if kw.get("reduce", 0) == L.SEQ_MEAN else
         np.full(n, 1 / (norm or (tokens if kw.get("reduce", 0) == 0 else S)))) * keep
    d = np.where(keep, logp - old, 0.0)
    pg = np.exp(d) * np.abs(adv) * (1 + np.abs(d)) + np.abs(adv)
    k = np.zeros(n)
    if ref is not None:
        q = np.where(keep, ref - logp, 0.0)
        k = (np.exp(q) + np.abs(q) + 1) * np.abs(q) + q * q + (kw.get("kl", L.K3) == L.K1)
    return keep, w, np.where(keep, pg, 0), np.where(keep, k, 0), d


def check_policy(kw, got, logp, old, adv, n, off=None, keep=None, ref=None, ent=None):
    loss, g, h = got
    rl, rg, rh = L.policy(logp, old, adv, np.ones(n) if keep is None else keep, off, ref, ent, **kw)
    live, w, pg, k, d = policy_sizes(kw, logp, old, adv, keep, off, ref, ent)
    ck, ce, gs = kw.get("kl_coef", 0), kw.get("entropy_coef", 0), abs(kw.get("grad_scale", 1))
    assert np.all(np.abs(g - rg) <= 2e-6 * gs * w * (pg + ck * k) + 1e-37)
    assert np.all(np.abs(h - rh) <= 1e-6 * np.abs(rh))
    e = np.where(live, np.abs(ent), 0) if ent is not None else np.zeros(n)
    sums = [(w * pg).sum(), (w * k).sum(), (w * e).sum()]
    bound = [sums[0] + ck * sums[1] + ce * sums[2], *sums, 0.0, 0.0]
    tokens = max(live.sum(), 1)
    r = np.where(live, np.exp(d) * (1 + np.abs(d)), 0).sum() / tokens
    bound += [r, r + 1]
    assert np.all(np.abs(loss - rl) <= 2e-6 * np.array(bound) + 1e-6 * np.abs(rl)), (loss, rl)


@pytest.mark.parametrize("reduce", [0, 1, 2])
@pytest.mark.parametrize("n_seq,lmax", [(1, 1), (1, 5000), (3, 40), (40, 300), (700, 6), (9, 4000)])
@pytest.mark.parametrize("shift", [0, 1])
def test_policy_sizes(edp_lib, reduce, n_seq, lmax, shift):
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(n_seq + lmax)
    off = offsets(rng, n_seq, lmax)
    n = int(off[-1])
    logp, old, ref, adv, ent = policy_case(rng, n)
    for full in (False, True):
        kw = dict(reduce=reduce, low=.2, high=.28)
        extra = dict(off=off)
        if full:
            kw.update(dual=2.0, kl_coef=.1, entropy_coef=.02, norm=17.0, grad_scale=-3.0)
            extra.update(ref=ref, ent=ent, keep=rng.random(n) < .7)
        elif reduce == 0:
            extra = {}
        got = run_policy(edp_lib, ring, kw, logp, old, adv, n, shift=shift, **extra)
        check_policy(kw, got, logp, old, adv, n, **extra)
        only = run_policy(edp_lib, ring, kw, logp, old, adv, n, shift=shift, grads=False, **extra)
        assert np.array_equal(only[0], got[0])
        if "keep" in extra:
            kw["norm"] = 0.0
            got = run_policy(edp_lib, ring, kw, logp, old, adv, n, shift=shift, **extra)
            check_policy(kw, got, logp, old, adv, n, **extra)


@pytest.mark.parametrize("kl", [0, 1, 2])
def test_policy_divergences(edp_lib, kl):
    """Log ratios from 1e-6 to 30, both signs."""
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(kl)
    n = 4000
    logp, old, _, adv, _ = policy_case(rng, n)
    ref = f32(logp + rng.choice([-1, 1], n) * 10.0**rng.uniform(-6, 1.4, n))
    kw = dict(kl_coef=1.0, kl=kl)
    got = run_policy(edp_lib, ring, kw, logp, old, adv, n, ref=ref)
    check_policy(kw, got, logp, old, adv, n, ref=ref)


@pytest.mark.parametrize("reduce", [0, 1, 2])
def test_policy_left_out_and_empty(edp_lib, reduce):
    """Tokens left out hold NaN and infinity; sequences without tokens; tokens
    after the last sequence; nothing left at all."""
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(reduce)
    off = np.array([0, 0, 50, 50, 53, 700, 700])
    n = 900  # room beyond off[-1]
    logp, old, ref, adv, ent = policy_case(rng, n)
    keep = rng.random(n) < .6
    keep[50:53] = False
    out = ~keep | (np.arange(n) >= 700)
    for a, x in zip((logp, old, ref, adv, ent), (np.nan, np.inf, -np.inf, np.nan, np.inf)):
        a[out] = x
    kw = dict(reduce=reduce, dual=3.0, kl_coef=.2, entropy_coef=.1)
    got = run_policy(edp_lib, ring, kw, logp, old, adv, n, off, keep, ref, ent)
    fix = lambda a: np.where(out, 0, a)  # noqa: E731
    check_policy(kw, got, fix(logp), fix(old), fix(adv), n, off, keep, fix(ref), fix(ent))
    assert not got[1][out].any() and not got[2][out].any()
    got = run_policy(edp_lib, ring, kw, logp, old, adv, n, off, np.zeros(n), ref, ent)
    assert not got[0].any() and not got[1].any() and not got[2].any()
    # the call after an empty one starts from its own counts
    got = run_policy(edp_lib, ring, kw, logp, old, adv, n, off, keep, ref, ent)
    check_policy(kw, got, fix(logp), fix(old), fix(adv), n, off, keep, fix(ref), fix(ent))


def test_policy_special_values(edp_lib):
    ring = ctx_of(edp_lib)
    logp = np.array([0.0, -1, -1, 90, -200, np.nan, -1])
    old = np.array([0.0, -1, -90, 0, 0, -1, -1])
    adv = np.array([1.0, 0, 0, 2, -2, 1, -1])
    for i in range(len(logp)):
        loss, g, _ = run_policy(edp_lib, ring, {}, logp[i:i + 1], old[i:i + 1], adv[i:i + 1], 1)
        want = [-1, 0, 0, -2.4, 1.6, np.nan, 1][i]
        dwant = [-1, 0, 0, 0, 0, np.nan, 1][i]
        assert np.isnan(want) and np.isnan(loss[0]) or abs(loss[0] - want) <= 1e-6, i
        assert np.isnan(dwant) and np.isnan(g[0]) or abs(g[0] - dwant) <= 1e-6, i


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(1, 3), (5, 1000), (40, 20_011), (333, 4097), (3, 152_064),
                                        (128, 130), (129, 130), (640, 65), (641, 65),
                                        (5000, 130)])
@pytest.mark.parametrize("reduce", [0, 1])
def test_policy_from_logits(edp_lib, dtype, rows, vocab, reduce):
    """The fused form against the oracle's three steps, in place and not, and
    against the three calls."""
    policy_from_logits(edp_lib, dtype, rows, vocab, reduce)


@pytest.mark.parametrize("dtype,vocab", [("f32", 420_011), ("bf16", 840_007)])
def test_policy_from_logits_beyond_shared_memory(edp_lib, dtype, vocab):
    """Rows whose eighth does not fit shared memory are read twice."""
    policy_from_logits(edp_lib, dtype, 2, vocab, 0)


def policy_from_logits(edp_lib, dtype, rows, vocab, reduce):
    edp, ring = edp_lib, ctx_of(edp_lib)
    rng = np.random.default_rng(rows)
    _, v, target, zd = make(rows, vocab, dtype, rows, banned=vocab > 100)
    off = np.concatenate([[0], np.sort(rng.integers(0, rows + 1, 4)), [rows]])
    keep = rng.random(rows) < .8
    if rows > 4:
        target[3] = -1
    use = keep & (target >= 0)
    T = .8
    tgt = np.maximum(target, 0)
    logp, H, m, S = L.token_logprob(zd, tgt, T)
    old, ref = f32(logp + rng.normal(0, .3, rows)), f32(logp + rng.normal(0, .3, rows))
    adv = f32(rng.normal(0, 1, rows))
    kw = dict(reduce=reduce, dual=3.0, kl_coef=.1, entropy_coef=.05, grad_scale=64.0)
    rl, rg, rh = L.policy(logp, old, adv, use, off, ref, H, **kw)
    cfg = edp.make_policy_config(.2, .2, 3.0, .1, L.K3, .05, reduce, 0.0, 64.0)
    args = dict(ref_logp=cuda(ref.astype(np.float32)), mask=cuda(keep.astype(np.uint8)),
                off=cuda(off.astype(np.uint64)), n_seq=5, temperature=T)
    d_old, d_adv = cuda(old.astype(np.float32)), cuda(adv.astype(np.float32))
    t = cuda(target)
    results = []
    for inplace in (False, True):
        store, out = view(rows, vocab, dtype, vocab + 3, 1)
        if inplace:
            out = v
        loss, lp = torch.full((8,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
        ent = torch.full((rows,), 7.0, device="cuda") if not inplace else None
        if inplace:  # the three calls first, while the logits are there
            lp3, e3, g3, h3 = (torch.zeros(rows, device="cuda") for _ in range(4))
            st, d3, l3 = torch.zeros(rows, 2, device="cuda"), torch.zeros_like(v), torch.zeros(
                8, device="cuda")
            edp.edp_token_logprob(ring.ctx, v, t, lp3, mask=args["mask"], temperature=T,
                                  entropy=e3, stats=st)
            edp.edp_policy_loss(ring.ctx, cfg, lp3, d_old, d_adv, rows, l3,
                                ref_logp=args["ref_logp"], mask=cuda(use.astype(np.uint8)),
                                off=args["off"], n_seq=5, entropy=e3, dlogp=g3, dentropy=h3)
            edp.edp_token_logprob_grad(ring.ctx, v, t, st, g3, d3, mask=args["mask"],
                                       temperature=T, entropy=e3, dentropy=h3)
        edp.edp_policy_loss_logits(ring.ctx, cfg, v, t, d_old, d_adv, loss, lp, out, entropy=ent,
                                   **args)
        edp.edp_sync(ring.ctx)
        results.append((to_np(loss), to_np(lp), to_np(out.double())))
        if not inplace:
            assert np.all(np.abs(to_np(ent)[use] - H[use]) <= 1e-5 + 1e-6 * H[use])
            gap = torch.ones_like(store, dtype=torch.bool)
            gap[1:1 + rows * (vocab + 3)].view(rows, vocab + 3)[:, :vocab] = False
            assert torch.isnan(store[gap]).all()
    (loss, lp, d), (loss2, lp2, d2) = results
    assert np.array_equal(loss, loss2) and np.array_equal(lp, lp2) and np.array_equal(d, d2)
    assert np.all(np.abs(lp[use] - logp[use]) <= 1e-5 + 1e-6 * np.abs(logp[use]))
    assert not lp[~use].any() and not d[~use].any()
    # log-probabilities off by 1e-5 move each term by that much of its size
    live, w, pg, k, _ = policy_sizes(kw, logp, old, adv, use, off, ref, H)
    bound = 2e-5 * np.array([1, 1, 1, 1, 0, 0, 1, 1]) * (1 + (w * (pg + k + H)).sum())
    assert np.all(np.abs(loss - rl) <= bound + 2e-5 * np.abs(rl)), (loss, rl)
    if use.any():
        y = np.where(np.isfinite(zd), (zd - m[:, None]) / T, 0)
        lnp = y - np.log(S)[:, None]
        p = np.where(np.isfinite(zd), np.exp(lnp), 0)
        ref_d = L.token_logprob_grad(zd[use], tgt[use], rg[use], rh[use], T)
        slack = 2e-5 * 64 * (w * (pg + .1 * k))[use][:, None]
        one = np.zeros_like(p[use])
        one[np.arange(int(use.sum())), tgt[use]] = 1
        size = np.abs(rg[use])[:, None] + np.abs(rh[use])[:, None] * (np.abs(lnp[use]) +
                                                                    H[use][:, None])
        bound = ((2e-5 + 4e-7 * np.abs(y[use])) * p[use] * size + slack * (one + p[use])) / T
        bound += UNIT[dtype] * np.abs(ref_d) + 2.0**-22 * one * np.abs(rg[use])[:, None] / T
        assert np.all(np.abs(d[use] - ref_d) <= bound + LEAST[dtype])
        # the three calls: the same numbers up to the last roundings
        assert np.all(np.abs(to_np(l3) - loss) <= 1e-5 * (1 + np.abs(loss)))
        assert np.all(np.abs(to_np(d3.double())[use] - d[use]) <= 2 * bound + 2 * LEAST[dtype] +
                      2 * UNIT[dtype] * np.abs(ref_d))


@pytest.mark.parametrize("vocab", [40, 20_000])
def test_policy_from_logits_special_values(edp_lib, vocab):
    """The type's lowest and largest values, one allowed token, NaN: the fused
    form as the three calls."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    for dtype in ("bf16", "f16", "f32"):
        _, v = view(6, vocab, dtype)
        v.normal_(0, 1)
        v[0, 1:] = torch.finfo(TYPES[dtype]).min
        v[1, :] = torch.finfo(TYPES[dtype]).min
        v[2, 1:] = -torch.inf
        v[3, 5] = float("nan")
        v[4, :] = torch.finfo(TYPES[dtype]).max
        t = cuda(np.array([0, 5, 0, 0, 9, 7], np.int32))
        a, b = torch.ones(6, device="cuda"), -torch.ones(6, device="cuda")
        cfg = edp.make_policy_config(entropy_coef=.1)
        lp, lp3, H, g, h = (torch.zeros(6, device="cuda") for _ in range(5))
        st, loss, d = torch.zeros(6, 2, device="cuda"), torch.zeros(8, device="cuda"), \
            torch.zeros_like(v)
        edp.edp_token_logprob(ring.ctx, v, t, lp3, entropy=H, stats=st)
        edp.edp_policy_loss(ring.ctx, cfg, lp3, b, a, 6, loss, entropy=H, dlogp=g, dentropy=h)
        edp.edp_token_logprob_grad(ring.ctx, v, t, st, g, d, entropy=H, dentropy=h)
        edp.edp_policy_loss_logits(ring.ctx, cfg, v, t, b, a, loss, lp, v)
        edp.edp_sync(ring.ctx)
        fine = [0, 1, 2, 4, 5]
        assert np.all(np.abs(to_np(lp)[fine] - to_np(lp3)[fine]) <= 1e-5)
        assert np.isnan(to_np(lp)[3]) and torch.isnan(v[3]).all() and torch.isnan(d[3]).all()
        got, want = to_np(v.double())[fine], to_np(d.double())[fine]
        # the same up to roundings of the type, and of 1e-5 of a gradient below 1
        assert np.all(np.abs(got - want) <= 2e-5 + 2 * UNIT[dtype] * np.abs(want))


def test_policy_from_logits_rows_without_distribution(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    _, v, target, zd = make(4, 100, "f32", 0)
    v[2] = -torch.inf
    target[1] = 100
    o = torch.zeros(4, device="cuda")
    loss, lp, d = torch.zeros(8, device="cuda"), torch.ones(4, device="cuda"), torch.ones_like(v)
    edp.edp_policy_loss_logits(ring.ctx, edp.make_policy_config(), v, cuda(target), o - 1, o + 1,
                               loss, lp, d)
    status, _ = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID
    assert lp[1] == 0 and lp[2] == 0 and not d[1].any() and not d[2].any()
    # three tokens count: the second, whose target does not exist, is left out
    logp = L.token_logprob(zd, np.minimum(target, 99))[0]
    want = L.policy([logp[0], 0, logp[3]], [-1] * 3, [1] * 3, [1] * 3)[0]
    assert np.all(np.abs(to_np(loss) - want) <= 3e-5 * (1 + np.abs(want)))


# ---- preference ----------------------------------------------------------------

def run_pref(edp, ring, kw, logp, ref, keep, off, pair, n, shift=0):
    def dev(x):
        pad = np.concatenate([np.full(shift, np.nan), x, np.full(4, np.nan)]).astype(np.float32)
        return cuda(pad)[shift:shift + len(x)]

    mask = None
    if keep is not None:
        mask = cuda(np.concatenate([np.zeros(shift), keep, np.zeros(4)]).astype(np.uint8))[
            shift:shift + len(keep)]
    S, P = len(off) - 1, len(pair)
    loss, u = torch.full((4,), 7.0, device="cuda"), torch.full((S,), 7.0, device="cuda")
    each = torch.full((P,), 7.0, device="cuda")
    store = torch.full((shift + n + 8,), 7.0, device="cuda")
    g = store[shift:shift + n]
    cfg = edp.make_preference_config(kw["beta"], kw.get("kind", 0), kw.get("smooth", 0.0),
                                     kw.get("margin", 0.0), kw.get("average", False),
                                     kw.get("norm", 0.0), kw.get("grad_scale", 1.0))
    edp.edp_preference_loss(ring.ctx, cfg, dev(logp), cuda(np.asarray(off, np.uint64)), S, n,
                            cuda(np.asarray(pair, np.int64)), P, loss,
                            ref_logp=dev(ref) if ref is not None else None, mask=mask,
                            seq_ratio=u, pair_loss=each, dlogp=g)
    status = edp.edp_sync_status(ring.ctx)[0]
    assert (store[:shift] == 7).all() and (store[shift + n:] == 7).all()
    return status, to_np(loss), to_np(u), to_np(each), to_np(g)


def check_pref(kw, got, logp, ref, keep, off, pair, n):
    _, loss, u, each, g = got
    rl, ru, re_, rg = L.preference(logp, ref, np.ones(n) if keep is None else keep, off, pair, **kw)
    live = (np.ones(n) if keep is None else np.asarray(keep)) > 0
    seq = L.sequences(off, n)
    S = len(off) - 1
    mass = np.zeros(S)
    live = live & (seq >= 0)
    np.add.at(mass, seq[live], np.abs(logp[live]) + (np.abs(ref[live]) if ref is not None else 0))
    if kw.get("average"):
        mass /= np.maximum(np.bincount(seq[live], minlength=S), 1)
    uerr = 2.0**-44 * 40 * mass  # sums in pairs, long before their rounding
    assert np.all(np.abs(u - ru) <= 2.0**-23 * np.abs(ru) + uerr)
    beta = kw["beta"]
    by = np.zeros(S)
    norm = kw.get("norm", 0) or len(pair)
    total = 0.0
    for i, (c, r) in enumerate(pair):
        if not (0 <= c < S and 0 <= r < S):
            assert each[i] == 0
            continue
        h = ru[c] - ru[r]
        d = abs(beta * h - kw.get("margin", 0))
        e = uerr[c] + uerr[r]
        if kw.get("kind", 0) == L.LOGISTIC:
            b = 1e-6 * (1 + re_[i]) * np.minimum(1 + d, 4) + beta * e
            gb = beta * (4 + d) * 2.0**-22 * (np.exp(-d) + 1e-12 + kw.get("smooth", 0) +
                                             (1 if h < 0 else 0)) + beta * beta * e
        elif kw["kind"] == L.HINGE:
            b, gb = 1e-6 * re_[i] + 2.0**-40 * d + beta * e, 0.0
        else:
            y = abs(h - .5 / beta)
            b, gb = 1e-6 * re_[i] + 2 * y * e + 1e-12, 2.0**-40 * (y + 1) + 2 * e
        assert abs(each[i] - re_[i]) <= b
        total += b / norm
        by[c] += gb
        by[r] += gb
    scale = 1 / np.maximum(np.bincount(seq[live], minlength=S), 1) if kw.get("average") else \
        np.ones(S)
    bound = abs(kw.get("grad_scale", 1)) / norm * (by * scale)[np.maximum(seq, 0)]
    assert np.all(np.abs(g - rg)[live] <= (bound + 2.0**-23 * np.abs(rg) + 1e-18)[live])
    assert not g[~live].any()
    assert abs(loss[0] - rl[0]) <= total + 1e-6 * abs(rl[0])
    assert np.all(np.abs(loss[1:] - rl[1:]) <= 1e-6 * (np.abs(rl[1:]) + 2.0**-20 * beta *
                                                       mass.max()))


@pytest.mark.parametrize("kind,smooth,margin", [(0, 0, 0), (0, .1, .25), (1, 0, 0), (2, 0, .5)])
@pytest.mark.parametrize("n_seq,lmax", [(1, 1), (2, 9), (2, 20_000), (33, 100), (500, 4), (64, 3000)])
@pytest.mark.parametrize("average,shift", [(False, 0), (True, 3)])
def test_preference_sizes(edp_lib, kind, smooth, margin, n_seq, lmax, average, shift):
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(n_seq + lmax)
    off = offsets(rng, n_seq, lmax)
    n = int(off[-1])
    ref = f32(-rng.exponential(1, n))
    logp = f32(ref + rng.normal(0, .1, n))
    # sequences in many pairs, in none, and against themselves
    pair = rng.integers(0, n_seq, (max(1, n_seq // 2), 2))
    keep = rng.random(n) < .9
    kw = dict(beta=.3, kind=kind, smooth=smooth, margin=margin, average=average)
    got = run_pref(edp_lib, ring, kw, logp, ref, keep, off, pair, n, shift)
    assert got[0] == edp_lib.EDP_OK
    check_pref(kw, got, logp, ref, keep, off, pair, n)
    kw.update(norm=5.0, grad_scale=128.0)
    got = run_pref(edp_lib, ring, kw, logp, None, None, off, pair, n, shift)
    check_pref(kw, got, logp, None, None, off, pair, n)


def test_preference_shared_sequences_and_order(edp_lib):
    """One sequence in thousands of pairs: its gradient is the sum, the same
    bits whatever the pairs' order."""
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(3)
    S = 300
    off = np.arange(S + 1) * 3
    n = 3 * S
    logp, ref = f32(-rng.exponential(1, n)), f32(-rng.exponential(1, n))
    pair = np.stack([np.zeros(5000, int), rng.integers(1, S, 5000)], 1)
    kw = dict(beta=.7)
    got = run_pref(edp_lib, ring, kw, logp, ref, None, off, pair, n)
    check_pref(kw, got, logp, ref, None, off, pair, n)
    again = run_pref(edp_lib, ring, kw, logp, ref, None, off, pair[::-1].copy(), n)
    assert np.array_equal(got[4], again[4]) and np.array_equal(got[2], again[2])


def test_preference_bad_pairs_masks_and_tail(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    rng = np.random.default_rng(4)
    off = np.array([0, 4, 4, 10, 200, 203])
    n = 230
    ref = f32(-rng.exponential(1, n))
    logp = f32(ref + rng.normal(0, .5, n))
    keep = rng.random(n) < .5
    keep[200:203] = False  # a sequence without tokens
    out = ~keep | (np.arange(n) >= 203)
    pair = [(0, 2), (3, 4), (5, 0), (-1, 2), (1, 3), (2, 1 << 40)]
    bad = logp.copy(), ref.copy()
    bad[0][out], bad[1][out] = np.nan, np.inf
    for average in (False, True):
        kw = dict(beta=.5, average=average)
        got = run_pref(edp, ring, kw, *bad, keep, off, pair, n)
        assert got[0] == edp.EDP_ERR_INVALID
        check_pref(kw, got, logp, ref, keep, off, pair, n)
    # NaN in a token that counts: its pairs and sequences, no others
    logp[int(np.flatnonzero(keep & (np.arange(n) < 4))[0])] = np.nan
    _, loss, u, each, g = run_pref(edp, ring, dict(beta=.5), logp, ref, keep, off, [(0, 2), (3, 2)],
                                   n)
    assert np.isnan(loss[0]) and np.isnan(u[0]) and np.isnan(each[0]) and not np.isnan(each[1])
    seq = L.sequences(off, n)
    for s, nan in ((0, True), (2, True), (3, False)):
        assert np.isnan(g[keep & (seq == s)]).all() == nan


# ---- balance -------------------------------------------------------------------

def run_balance(edp, ring, v, sel, keep, coef, scale, out):
    E = v.shape[1]
    loss, counts = torch.full((1,), 7.0, device="cuda"), torch.full((E,), 7, dtype=torch.int64,
                                                                   device="cuda")
    prob = torch.full((E,), 7.0, device="cuda")
    edp.edp_balance_loss(ring.ctx, v, cuda(sel), coef, loss, counts,
                         mask=cuda(keep.astype(np.uint8)) if keep is not None else None,
                         prob=prob, dlogits=out, grad_scale=scale)
    status = edp.edp_sync_status(ring.ctx)[0]
    return status, float(loss[0]), to_np(counts), to_np(prob)


def check_balance(got, d, zd, sel, keep, coef, scale, dtype):
    _, loss, counts, prob = got
    rows, E = zd.shape
    live = np.ones(rows, bool) if keep is None else keep
    rl, rc, rp, rg = L.balance(zd, sel, live, coef, scale)
    assert np.array_equal(counts, rc)
    assert np.all(np.abs(prob - rp) <= 1e-5 * rp + 2.0**-34)
    f = E * rc / (sel.shape[1] * max(live.sum(), 1))
    assert abs(loss - rl) <= 1e-5 * abs(coef) * (f @ rp) + 1e-9 * abs(coef) * f.sum()
    if d is None:
        return
    z = np.where(live[:, None], zd, 0.0)
    m = np.max(z, 1, keepdims=True)
    y = np.where(np.isfinite(z), z - np.where(np.isfinite(m), m, 0), -np.inf)
    e = np.exp(y)
    p = e / np.maximum(e.sum(1, keepdims=True), 1e-300) * live[:, None]
    size = abs(scale * coef) / max(live.sum(), 1) * p * (f + (p @ f)[:, None])
    rel = 4e-6 + 4e-7 * np.abs(np.where(np.isfinite(y), y, 0))
    assert np.all(np.abs(d - rg) <= rel * size + UNIT[dtype] * np.abs(rg) + LEAST[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,E,top", [(1, 1, 1), (1, 8, 2), (7, 3, 2), (300, 60, 6), (1000, 128, 8),
                                        (513, 257, 4), (90, 1000, 3), (64, 1024, 8), (5000, 8, 1),
                                        (777, 512, 64)])
def test_balance_sizes(edp_lib, dtype, rows, E, top):
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(rows + E)
    for shift, stride, masked in ((0, E, False), (1, E + 5, True), (0, E + 8 - E % 8, True)):
        _, v = view(rows, E, dtype, stride, shift)
        v.normal_(0, 2)
        zd = to_np(v.double())
        sel = rng.integers(-1 if masked else 0, E, (rows, top)).astype(np.int32)
        keep = rng.random(rows) < .7 if masked else None
        if masked:
            v[torch.from_numpy(~keep).cuda()] = float("nan")
        store, out = view(rows, E, dtype, stride, shift, 7.0)
        got = run_balance(edp_lib, ring, v, sel, keep, .01, 512.0, out)
        assert got[0] == edp_lib.EDP_OK
        check_balance(got, to_np(out.double()), zd, sel, keep, .01, 512.0, dtype)
        gap = torch.ones_like(store, dtype=torch.bool)
        gap[shift:shift + rows * stride].view(rows, stride)[:, :E] = False
        assert torch.isnan(store[gap]).all()
        # the loads alone; and in place
        none = run_balance(edp_lib, ring, v, sel, keep, .01, 512.0, None)
        assert none[1] == got[1] and np.array_equal(none[3], got[3])
        run_balance(edp_lib, ring, v, sel, keep, .01, 512.0, v)
        assert torch.equal(v, out)


def test_balance_many_rows(edp_lib):
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(9)
    rows, E = 60_001, 64
    _, v = view(rows, E, "bf16")
    v.normal_(0, 1)
    sel = rng.integers(0, E, (rows, 6)).astype(np.int32)
    keep = rng.random(rows) < .9
    out = torch.zeros_like(v)
    got = run_balance(edp_lib, ring, v, sel, keep, 1.0, 1.0, out)
    check_balance(got, to_np(out.double()), to_np(v.double()), sel, keep, 1.0, 1.0, "bf16")
    again = run_balance(edp_lib, ring, v, sel, keep, 1.0, 1.0, out)
    assert got[1] == again[1] and np.array_equal(got[3], again[3])


def test_balance_special_rows(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    rng = np.random.default_rng(2)
    _, v = view(6, 40, "f32")
    v.normal_(0, 1)
    v[1, 2:] = -torch.inf
    v[2] = torch.finfo(torch.float32).min
    sel = rng.integers(0, 40, (6, 2)).astype(np.int32)
    out = torch.zeros_like(v)
    got = run_balance(edp, ring, v, sel, None, 1.0, 1.0, out)
    assert got[0] == edp.EDP_OK
    check_balance(got, to_np(out.double()), to_np(v.double()), sel, None, 1.0, 1.0, "f32")
    v[3] = -torch.inf  # no distribution: p = 0, reported
    got = run_balance(edp, ring, v, sel, None, 1.0, 1.0, out)
    assert got[0] == edp.EDP_ERR_INVALID
    check_balance(got, to_np(out.double()), to_np(v.double()), sel, None, 1.0, 1.0, "f32")
    sel[4, 1] = 40  # not an expert: not counted, reported
    got = run_balance(edp, ring, v, sel, None, 1.0, 1.0, out)
    assert got[0] == edp.EDP_ERR_INVALID
    check_balance(got, to_np(out.double()), to_np(v.double()), sel, None, 1.0, 1.0, "f32")
    sel[4, 1] = 0
    v[5, 7] = float("nan")
    got = run_balance(edp, ring, v, sel, None, 1.0, 1.0, out)
    assert np.isnan(got[1]) and np.isnan(got[3]).all()
    d = to_np(out)
    assert np.isnan(d[5]).all() and np.isfinite(d[:5]).all()
    keep = np.zeros(6, bool)
    got = run_balance(edp, ring, v, sel, keep, 1.0, 1.0, out)
    assert got[1] == 0 and not got[2].any() and not got[3].any() and not to_np(out).any()


# ---- all -----------------------------------------------------------------------

def test_losses_on_streams_and_in_a_graph(edp_lib):
    """The same bits on another stream, from a graph and again, with the calls
    that share their scratch between them."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    rng = np.random.default_rng(5)
    off = offsets(rng, 50, 200)
    n = int(off[-1])
    arrs = [cuda(x.astype(np.float32)) for x in policy_case(rng, n)]
    d_off, pair = cuda(off.astype(np.uint64)), cuda(rng.integers(0, 50, (40, 2)))
    mask = cuda((rng.random(n) < .8).astype(np.uint8))
    cfgs = [edp.make_policy_config(kl_coef=.1, entropy_coef=.1, reduce=r) for r in range(3)]
    pcfg = edp.make_preference_config(.2)
    z = torch.randn(n, 48, device="cuda").to(torch.bfloat16)
    sel = cuda(rng.integers(0, 48, (n, 4)).astype(np.int32))

    def outputs():
        return [torch.zeros(8, device="cuda") for _ in range(3)] + [
            torch.zeros(n, device="cuda") for _ in range(4)] + [
            torch.zeros(4, device="cuda"), torch.zeros(1, device="cuda"),
            torch.zeros(48, dtype=torch.int64, device="cuda"), torch.zeros_like(z)]

    def go(o, stream=None):
        for r in range(3):
            edp.edp_policy_loss(ring.ctx, cfgs[r], arrs[0], arrs[1], arrs[3], n, o[r],
                                ref_logp=arrs[2], mask=mask, off=d_off, n_seq=50,
                                entropy=arrs[4], dlogp=o[3 + r], stream=stream)
        edp.edp_preference_loss(ring.ctx, pcfg, arrs[0], d_off, 50, n, pair, 40, o[7],
                                ref_logp=arrs[2], mask=mask, dlogp=o[6], stream=stream)
        edp.edp_balance_loss(ring.ctx, z, sel, .1, o[8], o[9], mask=mask, dlogits=o[10],
                             stream=stream)

    a, b, c = outputs(), outputs(), outputs()
    torch.cuda.synchronize()
    go(a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    go(b, side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        go(c)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for x, y, w in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, w)
    edp.edp_sync(ring.ctx)


def test_losses_between_calls_that_share_their_scratch(edp_lib):
    """Advantages, packing and each loss in turn on one stream, without waiting
    between them, give the bits that each gives on its own."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    rng = np.random.default_rng(8)
    off = offsets(rng, 60, 300)
    n = int(off[-1])
    logp, old, ref, adv, _ = (cuda(x.astype(np.float32)) for x in policy_case(rng, n))
    d_off, pair = cuda(off.astype(np.uint64)), cuda(rng.integers(0, 60, (50, 2)))
    tokens = cuda(rng.integers(0, 9, n).astype(np.int32))
    idx = torch.arange(60, device="cuda")
    mask = cuda((rng.random(n) < .8).astype(np.uint8))
    T, E = 64, 200
    r, v = torch.randn(T, E, device="cuda"), torch.randn(T + 1, E, device="cuda")
    d = torch.zeros(T, E, dtype=torch.uint8, device="cuda")
    z = torch.randn(n, 64, device="cuda")
    sel = cuda(rng.integers(0, 64, (n, 2)).astype(np.int32))
    seq = edp.make_policy_config(reduce=edp.EDP_REDUCE_SEQ_MEAN)
    one = edp.make_policy_config()
    pref = edp.make_preference_config(.2)

    def calls(wait):
        out = [torch.zeros(T, E, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"),
               torch.zeros(61, dtype=torch.int64, device="cuda")]
        out += [torch.zeros(n, device="cuda") for _ in range(3)]
        out += [torch.zeros(8, device="cuda") for _ in range(2)]
        out += [torch.zeros(4, device="cuda"), torch.zeros(1, device="cuda"),
                torch.zeros(64, dtype=torch.int64, device="cuda"), torch.zeros_like(z)]
        todo = [
            lambda: edp.edp_policy_loss(ring.ctx, seq, logp, old, adv, n, out[6], mask=mask,
                                        off=d_off, n_seq=60, dlogp=out[3]),
            lambda: edp.edp_gae(ring.ctx, r, v, d, T, E, .99, .95, adv_norm=out[0]),
            lambda: edp.edp_preference_loss(ring.ctx, pref, logp, d_off, 60, n, pair, 50, out[8],
                                            ref_logp=ref, mask=mask, dlogp=out[4]),
            lambda: edp.edp_pack_deliver(ring.ctx, tokens, d_off, 60, idx, 60, out[1], out[2], n),
            lambda: edp.edp_balance_loss(ring.ctx, z, sel, .1, out[9], out[10], mask=mask,
                                         dlogits=out[11]),
            lambda: edp.edp_policy_loss(ring.ctx, one, logp, old, adv, n, out[7], mask=mask,
                                        dlogp=out[5])]
        for f in todo:
            f()
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return out

    want = calls(True)
    for _ in range(5):
        for a, b in zip(calls(False), want):
            assert torch.equal(a, b)
    edp.edp_sync(ring.ctx)


def test_capture_before_the_scratch_is_there(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    n = 1 << 20
    x, loss = torch.zeros(n, device="cuda"), torch.zeros(8, device="cuda")
    off = torch.arange(0, n + 1, device="cuda")
    cfg = edp.make_policy_config(reduce=edp.EDP_REDUCE_SEQ_MEAN)
    mask = torch.ones(n, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        with pytest.raises(edp.EdpError) as e:
            edp.edp_policy_loss(ring.ctx, cfg, x, x, x, n, loss, mask=mask, off=off, n_seq=n)
        assert e.value.status == edp.EDP_ERR_STATE
        x.add_(0.0)
    edp.edp_policy_loss(ring.ctx, cfg, x, x, x, n, loss, mask=mask, off=off, n_seq=n)
    edp.edp_sync(ring.ctx)


def test_refusals(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    x = torch.zeros(6, device="cuda")
    off = torch.tensor([0, 2, 6], device="cuda")
    pair = torch.tensor([[0, 1]], device="cuda")
    loss, host = torch.zeros(8, device="cuda"), torch.zeros(6)
    z = torch.zeros(3, 4, device="cuda")
    sel = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    cnt = torch.zeros(4, dtype=torch.int64, device="cuda")

    def refused(f, *a, **k):
        with pytest.raises(edp.EdpError) as e:
            f(ring.ctx, *a, **k)
        assert e.value.status == edp.EDP_ERR_INVALID
        assert f.__name__ in str(e.value)

    P, Q = edp.make_policy_config, edp.make_preference_config
    for cfg in [P(-.1), P(1.0), P(float("nan")), P(.2, -1), P(.2, .2, 1.0), P(.2, .2, -2.0),
                P(kl_coef=-1), P(kl_coef=.1), P(entropy_coef=.1), P(entropy_coef=-1), P(kl=3),
                P(reduce=3), P(reduce=1), P(reduce=2), P(norm=-1), P(norm=float("inf")),
                P(grad_scale=float("nan"))]:
        refused(edp.edp_policy_loss, cfg, x, x, x, 6, loss)
    bad = P()
    bad.reserved[1] = 1
    refused(edp.edp_policy_loss, bad, x, x, x, 6, loss)
    refused(edp.edp_policy_loss, P(), x, x, x, 0, loss)
    refused(edp.edp_policy_loss, P(), x, x, x, 1 << 40, loss)
    refused(edp.edp_policy_loss, P(), x, x, x, 6, loss, off=off)
    refused(edp.edp_policy_loss, P(), x, x, x, 6, loss, n_seq=2)
    for i in range(3):
        a = [x, x, x]
        a[i] = None
        refused(edp.edp_policy_loss, P(), *a, 6, loss)
        a[i] = host
        refused(edp.edp_policy_loss, P(), *a, 6, loss)
    refused(edp.edp_policy_loss, P(), x, x, x, 6, None)
    for k in ("ref_logp", "entropy", "dlogp", "dentropy"):
        refused(edp.edp_policy_loss, P(), x, x, x, 6, loss, **{k: host})
    t = torch.zeros(3, dtype=torch.int32, device="cuda")
    F = edp.edp_policy_loss_logits
    refused(F, P(reduce=1), z, t, x, x, loss, x, z)
    refused(F, P(kl_coef=.1), z, t, x, x, loss, x, z)
    refused(F, P(), z, None, x, x, loss, x, z)
    refused(F, P(), z, t, x, x, loss, None, z)
    refused(F, P(), z, t, x, x, loss, x, None)
    refused(F, P(), z[:0], t, x, x, loss, x, z[:0])
    refused(F, P(), z, t, x, x, loss, x, z, temperature=0.0)
    for cfg in [Q(0.0), Q(-1.0), Q(.1, 3), Q(.1, 0, .5), Q(.1, 1, .1), Q(.1, 2, .1), Q(.1, 0, -.1),
                Q(.1, 1, 0.0, 1.0), Q(.1, margin=float("inf")), Q(.1, norm=-1.0),
                Q(.1, grad_scale=float("inf"))]:
        refused(edp.edp_preference_loss, cfg, x, off, 2, 6, pair, 1, loss)
    D = edp.edp_preference_loss
    refused(D, Q(.1), None, off, 2, 6, pair, 1, loss)
    refused(D, Q(.1), x, None, 2, 6, pair, 1, loss)
    refused(D, Q(.1), x, off, 0, 6, pair, 1, loss)
    refused(D, Q(.1), x, off, 2, 0, pair, 1, loss)
    refused(D, Q(.1), x, off, 2, 6, None, 1, loss)
    refused(D, Q(.1), x, off, 2, 6, pair, 0, loss)
    refused(D, Q(.1), x, off, 2, 6, pair, (1 << 20) + 1, loss)
    refused(D, Q(.1), x, off, 2, 6, pair.cpu(), 1, loss)
    refused(D, Q(.1), host, off, 2, 6, pair, 1, loss)
    B = edp.edp_balance_loss
    refused(B, z, sel, float("nan"), loss, cnt)
    refused(B, z, sel, .1, loss, cnt, grad_scale=float("inf"))
    refused(B, z, sel, .1, None, cnt)
    refused(B, z, sel, .1, loss, None)
    refused(B, z[:0], sel, .1, loss, cnt)
    refused(B, torch.zeros(3, 1025, device="cuda"), sel, .1, loss, cnt)
    refused(B, z, torch.zeros(3, 65, dtype=torch.int32, device="cuda"), .1, loss, cnt)
    refused(B, z, sel.cpu(), .1, loss, cnt)
    refused(B, z, sel, .1, loss, cnt.cpu())
    with pytest.raises(ValueError):
        B(ring.ctx, z, sel.t(), .1, loss, cnt)
    # a refused call leaves the context as it was
    edp.edp_policy_loss(ring.ctx, P(), x, x, x, 6, loss)
    edp.edp_sync(ring.ctx)
    for f in ("edp_token_logprob", "edp_policy_loss", "edp_preference_loss", "edp_balance_loss"):
        fn = getattr(edp.lib(), f)
        args = [0] * len(fn.argtypes)
        args = [None if a in (edp._VP,) or "LP_" in a.__name__ else 0 for a in fn.argtypes]
        assert fn(*args) == edp.EDP_ERR_INVALID
