"""Sums of rows of millions of alike numbers, whose roundings would all go one way: a row is
one CTA's, a lane has ten thousands of its numbers.  Logarithms are good to the 1e-5 + 1e-6 of
them that test_gpu_top.py has for short rows; far below the list's maximum to three roundings
of numbers up to 128 more."""
import math

import numpy as np
import pytest
import torch

from gpu_util import to_np

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = [("bf16", 8_388_608), ("f16", 8_388_001), ("f32", 4_194_304)]
LIKELY = 1_000


def ctx_of(edp):
    cfg = edp.make_config(64, (1, 16, 16), edp.EDP_XFORM_CHW_NORM_BF16)
    return edp.Ring(cfg, action=False, reward=False, done=False)


def long_row(vocab, dtype, shape, rows):
    """(logits with one row in use, its index, mask, columns of the likely tokens); of rows
    that are not given more than half of the SMs, so that none is split.  flat: all but the likely tokens are alike;
    rising: each is a little above the one before."""
    rows = rows or torch.cuda.get_device_properties(0).multi_processor_count // 2 + 1
    z = torch.empty(rows, vocab, dtype=TYPES[dtype], device="cuda")
    at = rows - 2
    z[at] = -0.3 if shape == "flat" else torch.linspace(-6.3, -0.3, vocab, device="cuda")
    columns = torch.arange(LIKELY, device="cuda") * (vocab // LIKELY) + 3
    z[at, columns] = 0.0
    mask = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    mask[at] = 1
    return z, at, mask, columns


def sums(z, inside):
    """(logarithm of the list's sum, of the others', entropy) in 64 bits."""
    x = z.double()
    ln = torch.logsumexp(x, 0)
    rest = x.clone()
    rest[inside] = -math.inf
    return float(torch.logsumexp(x[inside], 0)), float(torch.logsumexp(rest, 0)), \
        float(ln - ((x - ln).exp() * x).sum())


@pytest.mark.parametrize("dtype,vocab", SIZES)
@pytest.mark.parametrize("shape", ["flat", "rising"])
@pytest.mark.parametrize("high", [0.0, 100.0])
@pytest.mark.parametrize("top", [64, 128])
def test_lists_of_long_rows(edp_lib, dtype, vocab, shape, high, top, rows=None):
    """high 100: the list lies so far above all others that these are summed relative to
    their own maximum."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    z, at, mask, columns = long_row(vocab, dtype, shape, rows)
    inside = columns[:top]
    z[at, inside] = high
    rows = len(z)
    ids = torch.zeros(rows, top, dtype=torch.int32, device="cuda")
    lp = torch.zeros(rows, top, device="cuda")
    rest, H = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    edp.edp_token_top(ring.ctx, z, ids, lp, mask=mask, rest=rest, entropy=H)
    edp.edp_sync(ring.ctx)
    assert torch.equal(ids[at].long(), inside)
    of_list, of_rest, entropy = sums(z[at], inside)
    ln = float(np.logaddexp(of_list, of_rest))
    far = (high > 0) * 3 * 128 * 2.0**-24
    for got, want, more in ((lp[at], high - ln, 0), (rest[at], of_rest - ln, far),
                            (H[at], entropy, 0)):
        got = to_np(got.double())
        assert np.all(np.abs(got - want) <= 1e-5 + 1e-6 * min(abs(want), 40) + more), \
            (got.reshape(-1)[0], want)


@pytest.mark.parametrize("dtype,vocab", SIZES)
@pytest.mark.parametrize("shape", ["flat", "rising"])
@pytest.mark.parametrize("high", [0.0, 100.0, -60.0])
def test_distillation_of_long_rows(edp_lib, dtype, vocab, shape, high, rows=None):
    """sum p ln(p/q) with p = 1/20 at entries and 1/2 in all for the others, so that the
    loss has ln q of the list and of the others, and the gradient their sum.  The list lies
    at the others' likely tokens, far above and far below."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    z, at, mask, columns = long_row(vocab, dtype, shape, rows)
    n = 10
    inside = columns[-n:]
    z[at, inside] = high
    rows = len(z)
    ids = inside.to(torch.int32).repeat(rows, 1)
    value = torch.full((rows, n), -math.log(20.0), device="cuda")
    rest = torch.full((rows,), -math.log(2.0), device="cuda")
    loss = torch.zeros(1, device="cuda")
    of_list, of_rest, _ = sums(z[at], inside)
    ln = float(np.logaddexp(of_list, of_rest))
    lq, lqr = high - ln, of_rest - ln
    want = .5 * (-math.log(20) - lq) + .5 * (-math.log(2) - lqr)
    # both logarithms' bounds, and roundings of the logarithms of p and of the loss
    far = (high != 0) * 3 * 128 * 2.0**-24
    bound = 1e-5 + .5e-6 * (min(abs(lq), 40) + min(abs(lqr), 40)) + far
    d = torch.full_like(z, 7.0)
    for out in (None, d):
        edp.edp_distill_loss(ring.ctx, edp.make_distill_config(), z, ids, value, loss, rest=rest,
                             mask=mask, dlogits=out)
        edp.edp_sync(ring.ctx)
        assert abs(float(loss) - want) <= bound, (float(loss), want)
    eps = torch.finfo(TYPES[dtype]).eps / 2
    x = z[at].double()
    q, share = (x - ln).exp(), (x - of_rest).exp()
    q[inside] = share[inside] = 0
    # q and a token's share of its class, each to 1.2e-5 of itself, rounded to the type
    grad = q - .5 * share
    err = 1.2e-5 * (q + .5 * share) + eps * grad.abs() + (2.0**-24 if dtype == "f16" else 1e-37)
    off = (d[at].double() - grad).abs() - err
    off[inside] = 0
    assert off.max() <= 0, (float(off.max()), int(off.argmax()))


@pytest.mark.parametrize("dtype,vocab,rows", [("bf16", 8_388_608, 3), ("f32", 4_194_301, 5),
                                              ("f16", 700_001, 200), ("f32", 300_007, 160),
                                              ("bf16", 600_000, 400), ("f32", 270_000, 350)])
@pytest.mark.parametrize("high", [0.0, 100.0])
def test_other_shapes(edp_lib, dtype, vocab, rows, high):
    """Rows in parts, and more rows than SMs (one and two of them to an SM)."""
    test_lists_of_long_rows(edp_lib, dtype, vocab, "rising", high, 64, rows)
    test_distillation_of_long_rows(edp_lib, dtype, vocab, "flat", high, rows)


def test_rows_that_are_not_split(edp_lib):
    """77 rows are more than half of the SMs, so that each is one CTA's, as the test of the
    longest rows' ties (test_gpu_top.py) and those here need it."""
    assert 2 * 77 > torch.cuda.get_device_properties(0).multi_processor_count
