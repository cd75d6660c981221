"""A sequence of more tokens than 32 bits count.  The arrays hold one number, so that
the answers are known beforehand."""
import pytest
import torch

from test_gpu_logprob import ctx_of

pytestmark = pytest.mark.gpu

MORE = 2**32 + 2048


def test_a_long_sequence_by_its_mean(edp_lib):
    """The mean over a sequence's tokens: policy and preference loss."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    n = MORE + 5
    x = torch.ones(n, device="cuda")
    mask = torch.ones(n, dtype=torch.uint8, device="cuda")
    off = torch.tensor([0, MORE, n], device="cuda")
    loss = torch.zeros(8, device="cuda")
    cfg = edp.make_policy_config(reduce=edp.EDP_REDUCE_SEQ_MEAN)
    for m in (None, mask):  # ratio and advantage 1
        edp.edp_policy_loss(ring.ctx, cfg, x, x, x, n, loss, mask=m, off=off, n_seq=2)
        edp.edp_sync(ring.ctx)
        assert abs(float(loss[0]) + 1) <= 1e-6 and abs(float(loss[6]) - 1) <= 1e-6
    pair = torch.tensor([[0, 1]], device="cuda")
    u, out = torch.zeros(2, device="cuda"), torch.zeros(4, device="cuda")
    edp.edp_preference_loss(ring.ctx, edp.make_preference_config(1.0, average=True), x, off, 2, n,
                            pair, 1, out, mask=mask, seq_ratio=u)
    edp.edp_sync(ring.ctx)
    assert u.tolist() == [1, 1] and out[2] == 1 and out[3] == 1
    assert abs(float(out[0]) - 0.693147180559945) <= 1e-6
