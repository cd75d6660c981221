"""What edp_sync says of a batch with mistakes of several kinds: each kind has the number of
its own first row, or its own index."""
import numpy as np
import pytest
import torch

from gpu_util import cuda

pytestmark = pytest.mark.gpu


def ctx_of(edp):
    cfg = edp.make_config(64, (1, 16, 16), edp.EDP_XFORM_CHW_NORM_BF16)
    return edp.Ring(cfg, action=False, reward=False, done=False)


def report(edp, ring):
    status, msg = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID
    edp.edp_sync(ring.ctx)  # and it is said once
    return msg


@pytest.mark.parametrize("rows,vocab", [(40, 200), (2_000, 200), (300, 40_000)])
@pytest.mark.parametrize("gradient", [True, False])
def test_kinds_apart(edp_lib, rows, vocab, gradient):
    edp, ring = edp_lib, ctx_of(edp_lib)
    z = torch.randn(rows, vocab, device="cuda")
    ids = torch.arange(8, dtype=torch.int32, device="cuda").repeat(rows, 1)
    value = torch.full((rows, 8), -3.0, device="cuda")
    d, loss = torch.zeros_like(z) if gradient else None, torch.zeros(1, device="cuda")
    none, twice, strange = (np.arange(a, rows, b) for a, b in ((7, 5), (13, 10), (26, 20)))
    z[torch.from_numpy(none).cuda()] = -torch.inf
    ids[cuda(twice), 5] = 1
    ids[cuda(strange), 2] = vocab + 11

    def run(keep):
        mask = np.zeros(rows, np.uint8)
        for k in keep:
            mask[k] = 1
        edp.edp_distill_loss(ring.ctx, edp.make_distill_config(), z, ids, value, loss,
                             mask=cuda(mask), dlogits=d)
        return report(edp, ring)

    for _ in range(5):
        msg = run((none, twice))
        assert "twice (first row 13" in msg
        assert "twice (first row 23" in run((none, twice[1:]))
        msg = run((none, strange))
        assert "out of range (first offender %d" % (vocab + 11) in msg
        msg = run((none, twice, strange))
        assert "out of range (first offender %d" % (vocab + 11) in msg
        msg = run((none[2:],))
        assert "-infinity (first row 17" in msg


def test_rows_of_log_probabilities(edp_lib):
    """The first of many rows, in the other operators too."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    z = torch.randn(5_000, 300, device="cuda")
    target = torch.zeros(5_000, dtype=torch.int32, device="cuda")
    z[1_234:] = -torch.inf
    target[2_000::7] = 300
    lp = torch.zeros(5_000, device="cuda")
    ids = torch.zeros(5_000, 4, dtype=torch.int32, device="cuda")
    tp = torch.zeros(5_000, 4, device="cuda")
    for _ in range(3):
        edp.edp_token_logprob(ring.ctx, z[:2_000], target[:2_000], lp)
        assert "-infinity (first row 1234" in report(edp, ring)
        edp.edp_token_top(ring.ctx, z[:2_000], ids[:2_000], tp[:2_000])
        assert "-infinity (first row 1234" in report(edp, ring)
        edp.edp_token_logprob(ring.ctx, z, target, lp)
        assert "out of range (first offender 300" in report(edp, ring)
