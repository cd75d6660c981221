"""Pins of the 64-bit losses: hand-worked values, invariants, and every gradient
against central differences of its own loss."""
import math

import numpy as np
import pytest

from oracle import losses as L

H = 1e-5  # step; the error of a central difference is of the order of H^2 = 1e-10


def _diff(f, x):
    """Central differences of f by each element of x."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += H
        b[i] -= H
        g[i] = (f(a) - f(b)) / (2 * H)
    return g


def test_logprob_by_hand():
    z = np.array([[0.0, math.log(2), math.log(5)], [1.0, 1.0, -np.inf]])
    logp, ent, m, S = L.token_logprob(z, [1, 0])
    assert np.allclose(logp, [math.log(2 / 8), -math.log(2)], atol=1e-15)
    p = np.array([1, 2, 5]) / 8
    assert np.allclose(ent, [-(p * np.log(p)).sum(), math.log(2)], atol=1e-15)
    assert np.allclose(m, [math.log(5), 1]) and np.allclose(S, [8 / 5, 2])
    # two equal halves at any temperature, and the limit of a low one
    assert np.allclose(L.token_logprob(z[1:], [1], 0.3)[0], -math.log(2))
    assert L.token_logprob(z[:1], [2], 1e-3)[0][0] > -1e-12


@pytest.mark.parametrize("T", [1.0, 0.6])
def test_logprob_gradient_against_differences(T):
    rng = np.random.default_rng(0)
    z, t = rng.normal(0, 2, (3, 5)), np.array([0, 4, 2])
    g, h = rng.normal(0, 1, 3), rng.normal(0, 1, 3)

    def f(z):
        logp, ent, _, _ = L.token_logprob(z, t, T)
        return g @ logp + h @ ent

    assert np.allclose(L.token_logprob_grad(z, t, g, h, T), _diff(f, z), atol=1e-8)
    # a row's gradient sums to 0: a shift of the logits changes nothing
    assert np.allclose(L.token_logprob_grad(z, t, g, h, T).sum(1), 0, atol=1e-14)


def test_policy_by_hand():
    one = [True]
    # ratio 2: clipped at 1.2 for a positive advantage, not for a negative one
    l, g, _ = L.policy([math.log(2)], [0.0], [3.0], one)
    assert np.isclose(l[0], -3.6) and g[0] == 0 and l[4] == 1 and l[5] == 0
    l, g, _ = L.policy([math.log(2)], [0.0], [-3.0], one)
    assert np.isclose(l[0], 6.0) and np.isclose(g[0], 6.0) and l[5] == 0
    l, g, _ = L.policy([math.log(4)], [0.0], [-3.0], one, dual=3.0)
    assert np.isclose(l[0], 9.0) and g[0] == 0 and l[5] == 1
    l, g, _ = L.policy([math.log(.5)], [0.0], [-3.0], one)
    assert np.isclose(l[0], 2.4) and g[0] == 0 and l[5] == 1
    # weights: sequences of 1 and 3 tokens, the second with one left out
    logp, z = np.zeros(4), np.zeros(4)
    adv, keep, off = np.array([1.0, 2, 9, 4]), np.array([1, 1, 0, 1]), [0, 1, 4]
    assert np.isclose(L.policy(logp, z, adv, keep, off)[0][0], -7 / 3)
    assert np.isclose(L.policy(logp, z, adv, keep, off, reduce=L.SEQ_MEAN)[0][0], -(1 + 3) / 2)
    assert np.isclose(L.policy(logp, z, adv, keep, off, reduce=L.SEQ_SUM)[0][0], -7 / 2)
    assert np.isclose(L.policy(logp, z, adv, keep, off, norm=10)[0][0], -.7)
    # nothing left: all 0
    assert not L.policy(logp, z, adv, 0 * keep, off)[0].any()


@pytest.mark.parametrize("reduce", [0, 1, 2])
@pytest.mark.parametrize("kl", [0, 1, 2])
def test_policy_gradient_against_differences(reduce, kl):
    rng = np.random.default_rng(reduce + 3 * kl)
    n, off = 12, [0, 3, 3, 10, 12]
    old, ref = -rng.exponential(1, n), -rng.exponential(1, n)
    logp = old + rng.normal(0, .4, n)
    adv, ent, keep = rng.normal(0, 1, n), rng.random(n), rng.random(n) < .8
    kw = dict(off=off, ref=ref, dual=1.5, kl_coef=.3, kl=kl, entropy_coef=.2, reduce=reduce)
    _, g, h = L.policy(logp, old, adv, keep, entropy=ent, **kw)
    assert np.allclose(g, _diff(lambda x: L.policy(x, old, adv, keep, entropy=ent, **kw)[0][0],
                                logp), atol=1e-8)
    assert np.allclose(h, _diff(lambda x: L.policy(logp, old, adv, keep, entropy=x, **kw)[0][0],
                                ent), atol=1e-8)


def test_preference_by_hand():
    logp, ref = np.array([-1.0, -2, -3, -4, -7]), np.array([-1.5, -2, -4, -1, 0])
    off, keep = [0, 2, 4, 5], np.array([1, 1, 1, 0, 1])
    out, u, each, g = L.preference(logp, ref, keep, off, [(0, 1)], 0.5)
    assert np.allclose(u, [.5, 1, -7])
    s = 1 / (1 + math.exp(-.25))  # s(-d) for d = -1/4
    assert np.isclose(each[0], math.log(1 + math.exp(.25))) and out[1] == 0
    assert np.allclose(g, [-.5 * s, -.5 * s, .5 * s, 0, 0])
    # indices out of range add nothing; the divisor stays
    out2, _, each2, g2 = L.preference(logp, ref, keep, off, [(0, 1), (0, 3), (-1, 1)], .5)
    assert np.allclose(each2, [each[0], 0, 0]) and np.allclose(g2, g / 3)


@pytest.mark.parametrize("kind,smooth,margin", [(0, 0, 0), (0, .1, .3), (1, 0, 0), (2, 0, .2)])
@pytest.mark.parametrize("average", [False, True])
def test_preference_gradient_against_differences(kind, smooth, margin, average):
    rng = np.random.default_rng(kind)
    off, n = [0, 3, 4, 4, 9, 12], 12
    logp, ref, keep = -rng.exponential(1, n), -rng.exponential(1, n), rng.random(n) < .8
    pair = [(0, 1), (0, 3), (4, 0), (2, 3), (1, 1)]
    kw = dict(beta=.7, kind=kind, smooth=smooth, margin=margin, average=average)
    g = L.preference(logp, ref, keep, off, pair, **kw)[3]
    assert np.allclose(g, _diff(lambda x: L.preference(x, ref, keep, off, pair, **kw)[0][0],
                                logp), atol=1e-7)


def test_balance_by_hand_and_against_differences():
    rng = np.random.default_rng(1)
    # equal loads and probabilities: the loss is its coefficient
    sel = np.array([[0, 1], [2, 3]])
    loss, counts, prob, g = L.balance(np.zeros((2, 4)), sel, [1, 1], .01)
    assert np.isclose(loss, .01) and list(counts) == [1] * 4 and np.allclose(prob, .25)
    assert np.allclose(g, 0)
    z, sel = rng.normal(0, 1, (6, 5)), rng.integers(-1, 5, (6, 3))
    keep = np.array([1, 1, 0, 1, 1, 1])
    loss, counts, prob, g = L.balance(z, sel, keep, 2.0)
    assert counts.sum() == (sel[keep > 0] >= 0).sum() and np.isclose(prob.sum(), 1)
    assert np.allclose(g, _diff(lambda x: L.balance(x, sel, keep, 2.0)[0], z), atol=1e-8)
    assert not g[2].any()
