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


@pytest.mark.parametrize("vocab", [3_001, 66_000, 240_000])
@pytest.mark.parametrize("first", [60, 78])
@pytest.mark.parametrize("kind,rest", KINDS)
@pytest.mark.parametrize("scale,norm,T", [(1.0, 8_192.0, 1.0), (1e-3, 1_000.0, 1.0),
                                          (1.0, 1e6, 0.1)])
def test_small_gradients(edp_lib, vocab, first, kind, rest, scale, norm, T):
    """In fp32, whose bits the other tokens' factor has to have: held in shared memory, and
    (240,000 columns) from a second reading."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = below(18, vocab, "f32", kind, rest, first, T=T, scale=scale, norm=norm)
    _, d = view(18, vocab, "f32")
    loss, each = c.run(edp, ring, d)
    edp.edp_sync(ring.ctx)
    c.check(loss, each, d)


@pytest.mark.parametrize("dtype,vocab", [("bf16", 3_001), ("f16", 70_001), ("bf16", 470_000)])
@pytest.mark.parametrize("first", [60, 78])
def test_gradients_of_16_bits(edp_lib, dtype, vocab, first):
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = below(18, vocab, dtype, L.MIX, True, first)
    _, d = view(18, vocab, dtype)
    loss, each = c.run(edp, ring, d)
    edp.edp_sync(ring.ctx)
    c.check(loss, each, d)
