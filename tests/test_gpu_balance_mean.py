"""The mean of a router's probabilities over so many rows that a plain fp32 sum of
them loses digits."""
import pytest
import torch

from test_gpu_logprob import ctx_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2**24, 2**26])
@pytest.mark.parametrize("E", [7, 8])
def test_equal_probabilities(edp_lib, rows, E):
    """p = 1/(E - 1) on all experts but the last.  Partial sums are those of a few
    hundred rows, whose roundings, all in one direction, stay below 300 of 2^-24."""
    ring = ctx_of(edp_lib)
    z = torch.zeros(rows, E, dtype=torch.float16, device="cuda")
    z[:, E - 1] = -torch.inf
    sel = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    loss = torch.zeros(1, device="cuda")
    counts = torch.zeros(E, dtype=torch.int64, device="cuda")
    prob = torch.zeros(E, device="cuda")
    edp_lib.edp_balance_loss(ring.ctx, z, sel, 1.0, loss, counts, prob=prob)
    edp_lib.edp_sync(ring.ctx)
    assert (prob[:-1].double() * (E - 1) - 1).abs().max() <= 300 * 2.0**-24 and prob[-1] == 0
    assert abs(float(loss) * (E - 1) / E - 1) <= 320 * 2.0**-24
