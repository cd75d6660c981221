"""More choices of one expert than 32 bits count."""
import pytest
import torch

from test_gpu_logprob import ctx_of

pytestmark = pytest.mark.gpu


def test_choices_of_one_expert(edp_lib):
    ring = ctx_of(edp_lib)
    rows, top = 2**26 + 3, 64
    z = torch.zeros(rows, 2, dtype=torch.bfloat16, device="cuda")
    sel = torch.zeros(rows, top, dtype=torch.int32, device="cuda")
    loss = torch.zeros(1, device="cuda")
    counts = torch.zeros(2, dtype=torch.int64, device="cuda")
    edp_lib.edp_balance_loss(ring.ctx, z, sel, 1.0, loss, counts)
    edp_lib.edp_sync(ring.ctx)
    assert counts.tolist() == [rows * top, 0]
    # f = (2, 0) and p = 1/2
    assert abs(float(loss) - 1) <= 1e-5
