"""16-bit logits over the whole range that the calls accept: temperatures from
1e-6, largest logits from 1 to far beyond, lower ones that stand for a mask.

Bounds: those of test_gpu_logprob.py and of the form from logits in
test_gpu_losses.py, and a 2^y below 2^-126 is 0, which takes as much of a
gradient's size.  Gradients by the log-probabilities are scaled with the
temperature, so that those of the logits fit their type.
"""
import numpy as np
import pytest
import torch

from gpu_util import cuda, to_np
from oracle import losses as L
from test_gpu_logprob import LEAST, TYPES, UNIT, check_forward, ctx_of, run_grad, view
from test_gpu_losses import f32, policy_sizes

pytestmark = pytest.mark.gpu

TOPS = {"bf16": [0.0, 1.0, 20, 37.25, 60, 72.5, 101, 3e4, 1e6, 4e8, 1e20, -60, -1e4, -1e6, -1e9,
                 -1e20],
        "f16": [0.0, 1.0, 20, 37.25, 60, 72.5, 101, 3e4, -60, -3e4]}
LOWS = {"bf16": [-1e4, -1e9, -1e10, -1e20, -9e28, -3.38e38], "f16": [-2e4, -65504.0]}


def rows_of(dtype, vocab, T, seed):
    """For each largest logit: all equal, a few steps apart with excluded ones,
    and with one half of the row at a finite number that stands for a mask."""
    rng = np.random.default_rng(seed)
    wide = 2 * min(T, 50.0)  # within float16
    digits = {"bf16": 2.0**-7, "f16": 2.0**-10}[dtype]
    z, low = [], 0
    for M in TOPS[dtype]:
        z.append(np.full(vocab, M))
        step = 2.0**np.floor(np.log2(abs(M))) * digits if M else T
        y = M - step * rng.integers(0, 4, vocab) + wide * rng.normal(0, 1, vocab)
        y[rng.random(vocab) < .3] = -np.inf
        y[rng.integers(vocab)] = M
        z.append(y)
        if M >= -100:
            y = M - step * rng.integers(0, 4, vocab) + wide * rng.normal(0, 1, vocab)
            half = slice(0, vocab // 2) if low % 2 else slice(vocab // 2, vocab)
            y[half] = LOWS[dtype][low % len(LOWS[dtype])]
            low += 1
            z.append(y)
    store, v = view(len(z), vocab, dtype)
    v.copy_(torch.from_numpy(np.array(z)))
    zd = to_np(v.double())
    # a token that is not excluded: any of those near the top, or the top itself
    near = np.isfinite(zd) & (zd > zd.max(1, keepdims=True) - 20 * T -
                              8 * digits * np.abs(zd.max(1, keepdims=True)))
    some = np.array([rng.choice(np.flatnonzero(r)) for r in near], np.int32)
    return v, zd, some, zd.argmax(1).astype(np.int32)


def terms(zd, T):
    m = zd.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        y = np.where(np.isfinite(zd), (zd - m) / T, 0)
    lnp = y - np.log(np.where(np.isfinite(zd), np.exp(y), 0).sum(1))[:, None]
    return y, lnp, np.where(np.isfinite(zd), np.exp(lnp), 0)


def finite(zd):
    """-infinity as a number whose power of 2 is 0 all the same (the oracle's
    differences are then numbers)."""
    return np.where(np.isfinite(zd), zd, -1e300)


@pytest.mark.parametrize("T", [1e-6, 1e-5, 1e-4, 1e-3, 1e-2, 0.3, 1.0, 50.0, 1e6])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 3000, 40_000])
def test_logprob(edp_lib, T, dtype, vocab):
    ring = ctx_of(edp_lib)
    v, zd, target, _ = rows_of(dtype, vocab, T, vocab)
    rows = len(zd)
    zd = finite(zd)
    _, H, st = check_forward(edp_lib, ring, v, zd, target, T)
    check_forward(edp_lib, ring, v, zd, target, T, entropy=False)
    rng = np.random.default_rng(vocab)
    g, h = (f32(T * rng.normal(0, 1, rows)) for _ in range(2))
    _, ent, m, S = L.token_logprob(zd, target, T)
    exact = cuda(np.stack([m, S], 1).astype(np.float32)), cuda(ent.astype(np.float32))
    y, lnp, p = terms(to_np(v.double()), T)
    at = np.zeros_like(zd)
    at[np.arange(rows), target] = np.abs(g) / T
    for hh in (None, h):
        ah = np.zeros(rows) if hh is None else np.abs(hh)
        size = (np.abs(g)[:, None] + ah[:, None] * (np.abs(lnp) + ent[:, None])) / T
        ref = L.token_logprob_grad(zd, target, g, hh, T)
        bound = (1e-5 + 4e-7 * np.abs(y)) * p * size + UNIT[dtype] * np.abs(ref) + \
            2.0**-22 * at + 2.0**-126 * np.where(p > 0, size, 0) + LEAST[dtype]
        for stats, e in ((st, H), exact):
            _, out = view(rows, vocab, dtype)
            run_grad(edp_lib, ring, v, target, stats, e, g, hh, T, out)
            err = np.abs(to_np(out.double()) - ref)
            assert np.all(err <= bound), np.argwhere(~(err <= bound))[:5]


@pytest.mark.parametrize("T", [1e-6, 1e-5, 1e-4, 1e-3, 1e-2, 1.0])
@pytest.mark.parametrize("dtype,vocab", [("bf16", 40), ("f16", 40), ("bf16", 3000), ("f16", 3000),
                                         ("bf16", 40_000), ("f16", 40_000)])
def test_policy_from_logits(edp_lib, T, dtype, vocab):
    v, zd, _, target = rows_of(dtype, vocab, T, vocab + 1)
    policy_case(edp_lib, v, zd, target, dtype, T)


@pytest.mark.parametrize("T", [1e-6, 1e-3, 1.0])
def test_policy_from_logits_beyond_shared_memory(edp_lib, T):
    """Rows whose eighth does not fit shared memory are read twice."""
    v, zd, _, target = rows_of("bf16", 840_007, T, 5)
    pick = np.array([10, 13, 16, 20, 30, 41])
    w = v[torch.from_numpy(pick).cuda()].contiguous()
    policy_case(edp_lib, w, zd[pick], target[pick], "bf16", T)


def policy_case(edp, v, zd, target, dtype, T):
    ring = ctx_of(edp)
    rows, vocab = zd.shape
    rng = np.random.default_rng(rows)
    y, lnp, p = terms(zd, T)
    zd = finite(zd)
    logp, H, m, S = L.token_logprob(zd, target, T)
    old, ref = (f32(logp - rng.uniform(-.1, .1, rows)) for _ in range(2))
    adv = f32(rng.normal(0, 1, rows))
    kw = dict(reduce=0, kl_coef=.1, entropy_coef=.05, grad_scale=T)
    keep = np.ones(rows)
    rl, rg, rh = L.policy(logp, old, adv, keep, None, ref, H, **kw)
    cfg = edp.make_policy_config(kl_coef=.1, entropy_coef=.05, grad_scale=T)
    loss, lp, ent = (torch.full((n,), 7.0, device="cuda") for n in (8, rows, rows))
    _, out = view(rows, vocab, dtype)
    edp.edp_policy_loss_logits(ring.ctx, cfg, v, cuda(target), cuda(old.astype(np.float32)),
                               cuda(adv.astype(np.float32)), loss, lp, out,
                               ref_logp=cuda(ref.astype(np.float32)), temperature=T, entropy=ent)
    edp.edp_sync(ring.ctx)
    assert np.all(np.abs(to_np(lp) - logp) <= 1e-5 + 1e-6 * np.abs(logp))
    assert np.all(np.abs(to_np(ent) - H) <= 1e-5 + 1e-6 * H)
    _, w, pg, k, _ = policy_sizes(kw, logp, old, adv, keep, None, ref, H)
    bound = 2e-5 * np.array([1, 1, 1, 1, 0, 0, 1, 1]) * (1 + (w * (pg + k + H)).sum())
    assert np.all(np.abs(to_np(loss) - rl) <= bound + 2e-5 * np.abs(rl)), (loss, rl)
    ref_d = L.token_logprob_grad(zd, target, rg, rh, T)
    one = np.zeros_like(p)
    one[np.arange(rows), target] = 1
    size = np.abs(rg)[:, None] + np.abs(rh)[:, None] * (np.abs(lnp) + H[:, None])
    slack = 2e-5 * T * (w * (pg + .1 * k))[:, None]
    bound = ((2e-5 + 4e-7 * np.abs(y)) * p * size + slack * (one + p)) / T
    bound += UNIT[dtype] * np.abs(ref_d) + 2.0**-22 * one * np.abs(rg)[:, None] / T
    bound += 2.0**-126 * np.where(p > 0, size, 0) / T + LEAST[dtype]
    err = np.abs(to_np(out.double()) - ref_d)
    assert np.all(err <= bound), np.argwhere(~(err <= bound))[:5]
