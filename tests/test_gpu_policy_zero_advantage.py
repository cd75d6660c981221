"""A token that its policy now excludes (log-probability -infinity) in a group
without advantages: its ratio is 0, and so is its part of the loss."""
import numpy as np
import pytest
import torch

from gpu_util import cuda, to_np
from oracle import losses as L
from test_gpu_logprob import ctx_of, view
from test_gpu_losses import run_policy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dual", [0.0, 3.0])
@pytest.mark.parametrize("adv", [0.0, 1.5, -1.5])
@pytest.mark.parametrize("n", [5, 5000])
def test_excluded_token(edp_lib, dual, adv, n):
    ring = ctx_of(edp_lib)
    logp, old = np.full(n, -1.0), np.full(n, -1.0)
    a = np.full(n, .25)
    logp[2], a[2] = -np.inf, adv
    kw = dict(dual=dual)
    loss, g, _ = run_policy(edp_lib, ring, kw, logp, old, a, n)
    # by hand: -min(0 A, 0.8 A) at a ratio of 0
    want = (-.25 * (n - 1) + (0.8 * 1.5 if adv < 0 else 0.0)) / n
    assert abs(loss[0] - want) <= 1e-6 and abs(loss[1] - want) <= 1e-6
    assert abs(loss[6] - (n - 1) / n) <= 1e-6 and loss[7] == np.inf
    assert g[2] == 0 and np.all(np.abs(np.delete(g, 2) + .25 / n) <= 1e-6 / n)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_excluded_token_from_logits(edp_lib, dtype):
    edp, ring = edp_lib, ctx_of(edp_lib)
    _, v = view(3, 50, dtype)
    v.normal_(0, 1)
    v[1, 7] = -torch.inf
    zd = to_np(v.double())
    target = np.array([3, 7, 9], np.int32)
    adv, old = np.array([1.0, 0, -1]), np.full(3, -4.0)
    loss, lp, d = torch.zeros(8, device="cuda"), torch.zeros(3, device="cuda"), torch.ones_like(v)
    edp.edp_policy_loss_logits(ring.ctx, edp.make_policy_config(9.0 / 10, 1e6), v, cuda(target),
                               cuda(old.astype(np.float32)), cuda(adv.astype(np.float32)), loss,
                               lp, d)
    edp.edp_sync(ring.ctx)
    logp = L.token_logprob(zd, target)[0]
    assert lp[1] == -torch.inf
    r = np.exp(logp[[0, 2]] + 4)
    want = (-r[0] + max(r[1], .1)) / 3
    assert abs(float(loss[0]) - want) <= 3e-5 * (1 + r.sum())
    assert torch.isfinite(d).all() and not d[1].any() and d[0].any()
