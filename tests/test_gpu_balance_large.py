"""The router's sums where they are large, with answers known beforehand."""
import pytest
import torch

from test_gpu_logprob import ctx_of

pytestmark = pytest.mark.gpu


def outputs(E):
    return (torch.full((1,), 7.0, device="cuda"),
            torch.full((E,), 7, dtype=torch.int64, device="cuda"),
            torch.full((E,), 7.0, device="cuda"))


@pytest.mark.parametrize("rows", [2**23, 2**24, 2**24 + 5, 2**26])
def test_probabilities_of_many_rows(edp_lib, rows):
    """All of the probability on one of eight experts: its sum is the number of
    rows, the mean 1, the loss 8."""
    ring = ctx_of(edp_lib)
    z = torch.full((rows, 8), -torch.inf, dtype=torch.bfloat16, device="cuda")
    z[:, 3] = 1.0
    sel = torch.full((rows, 1), 3, dtype=torch.int32, device="cuda")
    loss, counts, prob = outputs(8)
    for _ in range(2):  # the second call starts from sums that the first left at 0
        edp_lib.edp_balance_loss(ring.ctx, z, sel, 1.0, loss, counts, prob=prob)
        edp_lib.edp_sync(ring.ctx)
        assert prob.tolist() == [0, 0, 0, 1, 0, 0, 0, 0]
        assert counts.tolist() == [0, 0, 0, rows, 0, 0, 0, 0]
        assert abs(float(loss) - 8) <= 1e-5


def test_one_expert(edp_lib):
    ring = ctx_of(edp_lib)
    rows = 2**24 + 3
    z = torch.randn(rows, 1, device="cuda")
    sel = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    loss, counts, prob = outputs(1)
    edp_lib.edp_balance_loss(ring.ctx, z, sel, .5, loss, counts, prob=prob)
    edp_lib.edp_sync(ring.ctx)
    assert float(prob) == 1 and int(counts) == rows and abs(float(loss) - .5) <= 1e-6
