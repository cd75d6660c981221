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


def long_row(vocab, dtype, high):
    """(logits with one row in use, its index, mask, columns of the likely tokens, the
    others' logit): more rows than half of the SMs, so that none is split."""
    rows = torch.cuda.get_device_properties(0).multi_processor_count // 2 + 1
    z = torch.empty(rows, vocab, dtype=TYPES[dtype], device="cuda")
    at = rows - 2
    z[at] = -0.3
    low = float(z[at, 0])
    columns = torch.arange(LIKELY, device="cuda") * (vocab // LIKELY) + 3
    z[at, columns] = high
    mask = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    mask[at] = 1
    return z, at, mask, columns, low


@pytest.mark.parametrize("dtype,vocab", SIZES)
@pytest.mark.parametrize("high", [0.0, 100.0])
@pytest.mark.parametrize("top", [64, 128])
def test_lists_of_long_rows(edp_lib, dtype, vocab, high, top):
    """high 100: the list lies so far above all others that these are summed relative to
    their own maximum."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    z, at, mask, columns, low = long_row(vocab, dtype, 0.0)
    z[at, columns[:top]] = high
    rows = len(z)
    ids = torch.zeros(rows, top, dtype=torch.int32, device="cuda")
    lp = torch.zeros(rows, top, device="cuda")
    rest, H = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    edp.edp_token_top(ring.ctx, z, ids, lp, mask=mask, rest=rest, entropy=H)
    edp.edp_sync(ring.ctx)
    assert torch.equal(ids[at].long(), columns[:top])
    few, many = LIKELY - top, vocab - LIKELY
    outside = few + many * math.exp(low)
    S = top + outside * math.exp(-high)                 # relative to the largest
    ln_s = math.log(S)
    U = few * -high + many * math.exp(low) * (low - high)
    for got, want, most in ((lp[at], -ln_s, 0), (rest[at], math.log(outside) - high - ln_s, high),
                            (H[at], ln_s - U * math.exp(-high) / S, 0)):
        got = to_np(got.double())
        assert np.all(np.abs(got - want) <= 1e-5 + 1e-6 * min(abs(want), 40) +
                      (most > 0) * 3 * 128 * 2.0**-24), (got.reshape(-1)[0], want)


@pytest.mark.parametrize("dtype,vocab", SIZES)
@pytest.mark.parametrize("high", [0.0, 100.0])
def test_distillation_of_long_rows(edp_lib, dtype, vocab, high):
    """sum p ln(p/q) with p = 1/20 at entries and 1/2 in all for the others, so that the
    loss has ln q of the list and of the others, and the gradient their sum."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    z, at, mask, columns, low = long_row(vocab, dtype, 0.0)
    n = 10
    z[at, columns[-n:]] = high
    rows = len(z)
    ids = columns[-n:].to(torch.int32).repeat(rows, 1)
    value = torch.full((rows, n), -math.log(20.0), device="cuda")
    rest = torch.full((rows,), -math.log(2.0), device="cuda")
    loss = torch.zeros(1, device="cuda")
    outside = LIKELY - n + (vocab - LIKELY) * math.exp(low)
    S = n + outside * math.exp(-high)
    lq, lqr = -math.log(S), math.log(outside) - high - math.log(S)
    want = .5 * (-math.log(20) - lq) + .5 * (-math.log(2) - lqr)
    # both logarithms' bounds, and roundings of the logarithms of p and of the loss
    bound = 1e-5 + .5e-6 * (abs(lq) + min(abs(lqr), 40)) + (high > 0) * 3 * 128 * 2.0**-24
    d = torch.full_like(z, 7.0)
    for out in (None, d):
        edp.edp_distill_loss(ring.ctx, edp.make_distill_config(), z, ids, value, loss, rest=rest,
                             mask=mask, dlogits=out)
        edp.edp_sync(ring.ctx)
        assert abs(float(loss) - want) <= bound, (float(loss), want)
    eps = torch.finfo(TYPES[dtype]).eps / 2
    free = torch.ones(vocab, dtype=torch.bool, device="cuda")
    free[columns] = False
    for got, y, tol in ((d[at, free], low, 1.2e-5), (d[at, columns[:-n]], 0.0, 1.2e-5)):
        q = math.exp(y - high) / S
        grad = q - .5 * math.exp(y) / outside
        # q and a token's share of its class, each to 1.2e-5 of itself (and e^-100 of nothing)
        err = tol * (q + .5 * math.exp(y) / outside) + eps * abs(grad) + \
            (2.0**-24 if dtype == "f16" else 1e-37)
        assert (got.double() - grad).abs().max() <= err, (float(got[0]), grad)
