"""Lists that the student hardly knows: the largest of their logits lies 60 to 95 nats below the
logarithm of the row's sum, which the sums relative to it reach 2^87 to 2^137 with, over rows
in 1 to 8 parts.  The bounds are those of test_gpu_distill.py."""
import numpy as np
import pytest
import torch

from gpu_util import to_np
from oracle import losses as L
from test_gpu_distill import KINDS, Case, ctx_of, view

pytestmark = pytest.mark.gpu

TOP = 20


def below(rows, vocab, dtype, kind, rest, first, T=1.0, **kw):
    """Row t's list lies first + t nats below the sum of the others (which is spread evenly
    over the row); rows from 18 on are left out."""
    keep = np.arange(rows) < 18
    c = Case(rows, vocab, TOP, dtype, kind, rest, first, T=T, absent=False,
             keep=keep if rows > 18 else None, **kw)
    for t in range(18):
        x = c.zd[t] / T
        lse = L._log_sum(np.delete(x, c.ids[t]))
        c.zd[t, c.ids[t]] = T * (lse - first - t - np.arange(TOP) / 30)
    c.v.copy_(torch.from_numpy(c.zd))
    c.zd = to_np(c.v.double())
    return c


# as parts of a row: 8, 4, 2 and 1 with the loss alone, by the rows and the row's size
ROWS = [(18, *k) for k in KINDS] + [(n, L.FORWARD, True) for n in (30, 60, 90)]


@pytest.mark.parametrize("dtype,vocab", [("f32", 66_000), ("bf16", 132_000), ("f16", 132_000)])
@pytest.mark.parametrize("rows,kind,rest", ROWS)
@pytest.mark.parametrize("first", [60, 78])
def test_loss_alone(edp_lib, dtype, vocab, rows, first, kind, rest):
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = below(rows, vocab, dtype, kind, rest, first)
    loss, each = c.run(edp, ring)
    edp.edp_sync(ring.ctx)
    assert torch.isfinite(each).all()
    c.check(loss, each)
