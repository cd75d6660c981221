"""The policy loss's tokens that do not count, and tokens whose log-probability
is -infinity, against the 64-bit oracle (bounds: test_gpu_losses.py)."""
import numpy as np
import pytest

from oracle import losses as L
from test_gpu_logprob import ctx_of
from test_gpu_losses import check_policy, policy_case, run_policy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kl", [L.K1, L.K2, L.K3])
@pytest.mark.parametrize("reduce", [0, 1, 2])
@pytest.mark.parametrize("n", [900, 4096, 4097, 9001])
@pytest.mark.parametrize("shift", [0, 1])
def test_left_out_by_every_divergence(edp_lib, kl, reduce, n, shift):
    """Tokens left out by the mask, before the first sequence and after the
    last: no gradient, whatever the divergence's own derivative is at 0."""
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(n + kl)
    cut = np.sort(rng.integers(7, n - 9, 3))
    off = np.array([7, 7, *cut, n - 9, n - 9])
    logp, old, ref, adv, ent = policy_case(rng, n)
    keep = rng.random(n) < .6
    keep[cut[0]:cut[1]] = False
    out = ~keep | (np.arange(n) < 7) | (np.arange(n) >= n - 9)
    clean = [a.copy() for a in (logp, old, adv, ref, ent)]
    for a, x in zip((logp, old, ref, adv, ent), (np.nan, np.inf, -np.inf, np.nan, np.inf)):
        a[out] = x
    for a in clean:
        a[out] = 0
    kw = dict(reduce=reduce, dual=3.0, kl_coef=.2, kl=kl, entropy_coef=.1, grad_scale=2.0)
    got = run_policy(edp_lib, ring, kw, logp, old, adv, n, off, keep, ref, ent, shift=shift)
    assert not got[1][out].any() and not got[2][out].any()
    check_policy(kw, got, *clean[:3], n, off, keep, *clean[3:])
