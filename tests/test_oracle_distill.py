"""Pins of the 64-bit lists and of the distillation loss: values worked by hand, limits,
and every gradient against central differences of its own loss."""
import math

import numpy as np
import pytest

from oracle import losses as L

H = 1e-5  # step; the error of a central difference is of the order of H^2 = 1e-10


def test_top_by_hand():
    z = np.log([[1.0, 4.0, 1.0, 2.0], [3.0, 3.0, 3.0, 3.0]])
    z = np.concatenate([z, [[-np.inf, 0.0, -np.inf, -np.inf]]])
    ids, logp, rest = L.token_top(z, 2)
    assert ids.tolist() == [[1, 3], [0, 1], [1, -1]]
    assert np.allclose(logp[:2], np.log([[.5, .25], [.25, .25]]), atol=1e-15)
    assert logp[2].tolist() == [0.0, -np.inf]
    assert np.allclose(rest[:2], np.log([.25, .5]), atol=1e-15) and rest[2] == -np.inf
    # the list and the rest are a distribution at any temperature
    z = np.random.default_rng(0).normal(0, 3, (5, 40))
    for T in (0.3, 1.0, 4.0):
        _, logp, rest = L.token_top(z, 7, T)
        assert np.allclose(np.exp(logp).sum(1) + np.exp(rest), 1, atol=1e-14)


def test_distill_by_hand():
    z = np.log([[1.0, 2.0, 1.0, 4.0]])  # q = 1/8, 1/4, 1/8, 1/2
    ids, value, rest = np.array([[3, 1]]), np.log([[.5, .125]]), np.log([.375])
    P, Q = np.array([.5, .125, .375]), np.array([.5, .25, .25])
    M = .3 * P + .7 * Q
    want = {L.FORWARD: (P * np.log(P / Q)).sum(), L.REVERSE: (Q * np.log(Q / P)).sum(),
            L.MIX: .3 * (P * np.log(P / M)).sum() + .7 * (Q * np.log(Q / M)).sum()}
    for kind, w in want.items():
        loss, each, grad = L.distill(z, ids, value, rest, [1], kind=kind,
                                     beta=.3 if kind == L.MIX else 0.0)
        assert math.isclose(loss, w, abs_tol=1e-15) and math.isclose(each[0], w, abs_tol=1e-15)
        assert np.allclose(grad.sum(), 0, atol=1e-15)
        if kind == L.FORWARD:  # q - p by classes, the others by their share
            assert np.allclose(grad, [[.125 - .1875, .125, .125 - .1875, 0]], atol=1e-15)
    # raw values at a temperature: only their softmax counts
    _, _, grad = L.distill(z, ids, 2 * value + 5, None, [1], teacher_temperature=2.0)
    assert np.allclose(grad, [[.125, .25 - .2, .125, .5 - .8]], atol=1e-15)
    # the same distribution: no loss, no gradient
    for kind in want:
        loss, _, grad = L.distill(z, ids, np.log([[.5, .25]]), np.log([.25]), [1], kind=kind,
                                  beta=.3 if kind == L.MIX else 0.0)
        assert abs(loss) < 1e-15 and np.abs(grad).max() < 1e-15
    # an absent entry is none
    a = L.distill(z, np.array([[3, -1, 1]]), np.array([[-.7, 9.0, -2.0]]), rest, [1])
    b = L.distill(z, np.array([[3, 0, 1]]), np.array([[-.7, -np.inf, -2.0]]), rest, [1])
    c = L.distill(z, ids, np.array([[-.7, -2.0]]), rest, [1])
    assert a[0] == b[0] == c[0] and np.array_equal(a[2], c[2]) and np.array_equal(b[2], c[2])


def test_classes_beyond_the_smallest_probability():
    """q of the rest is 0 in 64 bits: its tokens still share its pull, by their own odds."""
    _, _, grad = L.distill([[1000.0, 0.0, math.log(3)]], [[0]], [[math.log(.9)]], [math.log(.1)],
                           [1])
    assert np.allclose(grad, [[.1, -.025, -.075]], atol=1e-15)


@pytest.mark.parametrize("reduce", [L.TOKEN_MEAN, L.SEQ_MEAN, L.SEQ_SUM])
@pytest.mark.parametrize("kind,rest", [(L.FORWARD, True), (L.FORWARD, False), (L.REVERSE, True),
                                       (L.MIX, True)])
def test_distill_gradient_against_differences(kind, rest, reduce):
    rng = np.random.default_rng(5)
    n, V, K = 6, 9, 4
    z, off = rng.normal(0, 2, (n, V)), np.array([0, 2, 2, 5])
    ids = np.array([rng.permutation(V)[:K] for _ in range(n)])
    ids[1, 2] = -1
    ids[4] = -1
    value, r = rng.normal(-1, 1, (n, K)), rng.normal(-1, .5, n) if rest else None
    keep = np.array([1, 1, 0, 1, 1, 1], bool)
    kw = dict(off=off, kind=kind, beta=.4 if kind == L.MIX else 0.0, reduce=reduce,
              temperature=1.3, teacher_temperature=1.0 if rest else .8)
    _, _, grad = L.distill(z, ids, value, r, keep, grad_scale=3.0, **kw)
    assert not grad[2].any() and not grad[5].any()  # masked, outside of the sequences
    num = np.zeros_like(z)
    for i in np.ndindex(*z.shape):
        a, b = z.copy(), z.copy()
        a[i] += H
        b[i] -= H
        num[i] = (L.distill(a, ids, value, r, keep, **kw)[0] -
                  L.distill(b, ids, value, r, keep, **kw)[0]) / (2 * H)
    assert np.allclose(grad, 3 * num, atol=3e-8)


def test_weights_by_hand():
    off = [1, 3, 3, 6]
    keep = [1, 1, 0, 1, 1, 1, 1]
    third = 1 / 3
    assert np.allclose(L.weights(keep, off), [0, .25, 0, .25, .25, .25, 0])
    assert np.allclose(L.weights(keep, off, L.SEQ_MEAN), [0, third, 0] + [third / 3] * 3 + [0])
    assert np.allclose(L.weights(keep, off, L.SEQ_SUM), [0, third, 0] + [third] * 3 + [0])
    assert np.allclose(L.weights(keep, off, norm=8.0)[3], 1 / 8)
    assert np.allclose(L.weights(keep), np.array(keep) / 6)
