"""NaN and infinities in a teacher's lists: a row that has any is NaN whole, its loss and every
number of its gradient, whatever the student's probabilities are; the other rows are as without
it."""
import numpy as np
import pytest
import torch

from gpu_util import to_np
from oracle import losses as L
from test_gpu_distill import LEAST, UNIT, Case, ctx_of, view

pytestmark = pytest.mark.gpu

WITH_REST = [L.FORWARD, L.REVERSE, L.MIX]
SIZES = [("f32", 60), ("bf16", 60), ("f16", 40_001), ("bf16", 40_001), ("f32", 240_000)]


def near_rows(c, rows, each, got):
    """The row losses and gradients of `rows`, of a batch whose mean is over all."""
    (be, bg), want, grad = c.expect_rows(rows)
    e = to_np(each.double())[rows]
    assert np.all(np.abs(e - want) <= be + 1e-6 * np.abs(want))
    if got is not None:
        g = to_np(got.double())[rows]
        assert np.all(np.abs(g - grad) <= bg + UNIT[c.dtype] * (np.abs(grad) + bg) +
                      LEAST[c.dtype])


def exclude(c, t, places):
    c.zd[t, places] = -np.inf


@pytest.mark.parametrize("dtype,vocab", SIZES)
@pytest.mark.parametrize("kind", WITH_REST)
@pytest.mark.parametrize("top", [6, 40])
def test_nan_and_infinity_in_lists(edp_lib, dtype, vocab, kind, top):
    edp, ring = edp_lib, ctx_of(edp_lib)
    n, inf = 12, float("inf")
    c = Case(n, vocab, top, dtype, kind, True, 4, absent=False)
    c.value[0, 1] = inf
    c.rest[1] = inf
    c.rest[2] = np.nan
    for t, x in ((3, np.nan), (4, inf), (5, np.nan)):   # where the student has no probability
        c.zd[t, c.ids[t, 2]] = -300 if t < 5 else -inf
        c.value[t, 2] = x
    for t in (6, 7, 8):                                 # all others are excluded
        exclude(c, t, np.setdiff1d(np.arange(vocab), c.ids[t]))
    c.value[6, 0], c.rest[7] = np.nan, np.nan
    c.zd[8, c.ids[8, 1]] = np.nan                       # of the student
    c.value[9, top - 1], c.rest[9] = inf, inf
    c.v.copy_(torch.from_numpy(c.zd))
    c.zd = to_np(c.v.double())
    _, d = view(n, vocab, dtype)
    loss, each = c.run(edp, ring, d)
    edp.edp_sync(ring.ctx)
    assert torch.isnan(loss[0]) and torch.isnan(each[:10]).all()
    assert torch.isnan(d[:10]).all()
    near_rows(c, [10, 11], each, d)
    loss, each = c.run(edp, ring)
    edp.edp_sync(ring.ctx)
    assert torch.isnan(loss[0]) and torch.isnan(each[:10]).all()
    near_rows(c, [10, 11], each, None)


@pytest.mark.parametrize("dtype,vocab", SIZES)
@pytest.mark.parametrize("top", [6, 40])
def test_nan_and_infinity_in_lists_without_rest(edp_lib, dtype, vocab, top):
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = Case(6, vocab, top, dtype, L.FORWARD, False, 4, absent=False)
    c.value[0, 1] = np.nan
    c.value[1, top - 1] = np.inf
    c.zd[2, c.ids[2, 3]], c.value[2, 3] = -300, np.inf
    exclude(c, 3, np.setdiff1d(np.arange(vocab), c.ids[3]))
    c.value[3, 2] = np.nan
    c.v.copy_(torch.from_numpy(c.zd))
    c.zd = to_np(c.v.double())
    _, d = view(6, vocab, dtype)
    for out in (d, None):
        loss, each = c.run(edp, ring, out)
        edp.edp_sync(ring.ctx)
        assert torch.isnan(loss[0]) and torch.isnan(each[:4]).all()
        near_rows(c, [4, 5], each, out)
    assert torch.isnan(d[:4]).all()


@pytest.mark.parametrize("dtype,vocab", SIZES)
def test_reverse_where_the_teacher_excludes_the_rest(edp_lib, dtype, vocab):
    """The loss is infinite, and the row's gradient NaN throughout: at the entries, at those
    that the student gives nothing, and at all others."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = Case(4, vocab, 12, dtype, L.REVERSE, True, 4, absent=False)
    c.rest[:2] = -np.inf
    c.zd[1, c.ids[1, 2]], c.zd[1, c.ids[1, 3]] = -300, -np.inf
    exclude(c, 2, np.setdiff1d(np.arange(vocab), c.ids[2]))  # nothing is left to exclude
    c.rest[2] = -np.inf
    c.v.copy_(torch.from_numpy(c.zd))
    c.zd = to_np(c.v.double())
    _, d = view(4, vocab, dtype)
    for out in (d, None):
        loss, each = c.run(edp, ring, out)
        edp.edp_sync(ring.ctx)
        assert loss[0] == float("inf") and (each[:2] == float("inf")).all()
        near_rows(c, [2, 3], each, out)
    assert torch.isnan(d[:2]).all()


@pytest.mark.parametrize("top", [1, 20, 33, 128])
@pytest.mark.parametrize("vocab", [130, 33_001])
@pytest.mark.parametrize("with_rest", [True, False])
def test_a_broken_teacher(edp_lib, top, vocab, with_rest):
    """A teacher's row with NaN or +infinity is the student's, too: edp_token_top marks it by
    ids of -1 and NaN, and the loss does not pass over it as over a row without a list."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    t = torch.randn(6, vocab, device="cuda")
    t[0, 5], t[1, vocab - 1] = float("nan"), float("inf")
    s = torch.randn(6, vocab, device="cuda")
    mask = torch.tensor([1, 1, 0, 1, 1, 1], dtype=torch.uint8, device="cuda")
    ids = torch.zeros(6, top, dtype=torch.int32, device="cuda")
    lp, rest = torch.zeros(6, top, device="cuda"), torch.zeros(6, device="cuda")
    edp.edp_token_top(ring.ctx, t, ids, lp, mask=mask, rest=rest)
    ids[4], lp[4], rest[4] = -1, -float("inf"), -float("inf")  # a row without a list
    # places without a token hold anything, unless it is NaN alone
    ids[3, 1:], lp[3, 1:] = -1, float("nan")
    ids[5], lp[5], rest[5] = -1, float("nan"), -float("inf")
    lp[5, top // 2] = 3.0
    loss, each = torch.zeros(1, device="cuda"), torch.zeros(6, device="cuda")
    d = torch.full_like(s, 7.0)
    for out in (d, None):
        edp.edp_distill_loss(ring.ctx, edp.make_distill_config(), s, ids, lp, loss,
                             rest=rest if with_rest else None, mask=mask, row_loss=each,
                             dlogits=out)
        edp.edp_sync(ring.ctx)
        assert torch.isnan(loss).all() and torch.isnan(each[:2]).all()
        assert not each[[2, 4, 5]].any() and torch.isfinite(each[3])
    assert torch.isnan(d[:2]).all()
    assert not d[[2, 4, 5]].any() and torch.isfinite(d[3]).all()
