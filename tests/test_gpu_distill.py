"""The distillation loss against the 64-bit oracle on the same (rounded) inputs.

Bounds, with y = (z - m) / T: a log-probability of the student, of a token or of the class
of all others, is good to 1e-5 + 1e-6 of it (as those of the lists), a teacher's from a
list's softmax better; a probability q to (1e-5 + 4e-7 |y|) of itself, the teacher's
exp(value) to 2^-21.  With d_b = 1.2e-5 + 3e-6 (|ln p_b| + |ln q_b|) for the logarithm of a
class's ratio:
  loss of a row:  sum_b (p_b + q_b) (d_b + 1.2e-5 |ln p_b - ln q_b|)
  gradient:       (scale w / T) [(1.2e-5 + 4e-7 |y|) (q_j |G| + s_j |q_b f'_b|)
                                 + s_j (p_b + q_b) (d_b + the loss's bound)]
                  + the rounding to the output's type,
G the sum of all q_b f'_b and s_j the token's share of its class.
"""
import gc

import numpy as np
import pytest
import torch

from gpu_util import cuda, to_np
from oracle import losses as L

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {k: torch.finfo(t).eps / 2 for k, t in TYPES.items()}  # 2^-24, 2^-8, 2^-11
LEAST = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0**-24}
KINDS = [(L.FORWARD, True), (L.FORWARD, False), (L.REVERSE, True), (L.MIX, True)]
BETA = 0.3


def ctx_of(edp):
    cfg = edp.make_config(64, (1, 16, 16), edp.EDP_XFORM_CHW_NORM_BF16)
    return edp.Ring(cfg, action=False, reward=False, done=False)


def view(rows, vocab, dtype, stride=None, shift=0, fill=float("nan")):
    stride = stride or vocab
    store = torch.full((shift + rows * stride + 16,), fill, dtype=TYPES[dtype], device="cuda")
    return store, store[shift:shift + rows * stride].view(rows, stride)[:, :vocab]


class Case:
    """Logits, lists (some shorter than others, in any order) and what they weigh."""

    def __init__(self, rows, vocab, top, dtype, kind, rest, seed, T=1.0, reduce=L.TOKEN_MEAN,
                 off=None, keep=None, norm=0.0, scale=1.0, stride=None, shift=0, spread=2.0,
                 absent=True, tt=None):
        rng = np.random.default_rng(seed)
        z = rng.normal(0, spread, (rows, vocab)) * T
        self.ids = np.full((rows, top), -1, np.int32)
        self.value = rng.normal(-1, 1, (rows, top))
        n = min(top, vocab)
        for t in range(rows):
            self.ids[t, :n] = rng.permutation(vocab)[:n]
            z[t, self.ids[t, :n]] += T * (np.log(vocab) + rng.normal(-2, 1, n))
            if absent and t % 3 == 2:
                self.ids[t, rng.random(top) < .3] = -1
                self.value[t, rng.random(top) < .2] = -np.inf
        self.rest = None
        if rest:
            self.rest = -.3 - 4 * rng.random(rows)
            v = np.where(self.ids >= 0, self.value, -np.inf)
            s = np.log(np.maximum(np.exp(v).sum(1), 1e-300))
            self.value = np.where(np.isfinite(s)[:, None] & (s > -600)[:, None],
                                  self.value - s[:, None], self.value) + \
                np.log1p(-np.exp(self.rest))[:, None]
            self.rest = self.rest.astype(np.float32)
        else:
            self.value = 3 + 2 * self.value
        self.value = self.value.astype(np.float32)
        self.store, self.v = view(rows, vocab, dtype, stride, shift)
        self.v.copy_(torch.from_numpy(z))
        self.zd = to_np(self.v.double())
        self.keep = np.ones(rows, bool) if keep is None else keep
        self.masked = keep is not None
        self.off, self.T, self.dtype, self.kind, self.reduce = off, T, dtype, kind, reduce
        self.norm, self.scale, self.beta = norm, scale, BETA if kind == L.MIX else 0.0
        self.tt = 1.0 if rest else (1.7 if tt is None else tt)

    def config(self, edp):
        return edp.make_distill_config(self.kind, self.reduce, self.beta, self.tt, self.norm,
                                       self.scale)

    def arrays(self):
        return dict(ids=cuda(self.ids), value=cuda(self.value),
                    rest=cuda(self.rest) if self.rest is not None else None,
                    mask=cuda(self.keep.astype(np.uint8)) if self.masked else None,
                    off=cuda(np.asarray(self.off, np.int64)) if self.off is not None else None)

    def run(self, edp, ring, dlogits=None, row_loss=True, stream=None):
        rows = len(self.ids)
        a = self.arrays()
        loss = torch.full((2,), 7.0, device="cuda")
        each = torch.full((rows + 2,), 7.0, device="cuda") if row_loss else None
        edp.edp_distill_loss(ring.ctx, self.config(edp), self.v, a["ids"], a["value"], loss,
                             rest=a["rest"], mask=a["mask"], off=a["off"],
                             n_seq=len(self.off) - 1 if self.off is not None else 0,
                             temperature=self.T, row_loss=each, dlogits=dlogits, stream=stream)
        return loss, each

    def expect(self):
        return L.distill(self.zd, self.ids, self.value.astype(np.float64),
                         None if self.rest is None else self.rest.astype(np.float64), self.keep,
                         self.off, self.kind, self.beta, self.reduce, self.norm, self.T, self.tt,
                         self.scale)

    def bounds(self):
        """(of the row losses, of the gradient before its type's rounding)."""
        rows, V = self.zd.shape
        w = L.weights(self.keep, self.off, self.reduce, self.norm)
        each, grad = np.zeros(rows), np.zeros((rows, V))
        for t in np.flatnonzero(w):
            x = self.zd[t] / self.T
            lnq = x - L._log_sum(x)
            here = (self.ids[t] >= 0) & (self.value[t] > -np.inf)
            at = self.ids[t][here].astype(int)
            lp = self.value[t][here].astype(np.float64)
            if self.rest is None:
                lp = lp / self.tt
                lp = lp - (L._log_sum(lp) if len(lp) else 0)
                lp = np.append(lp, -np.inf)
            else:
                lp = np.append(lp, float(self.rest[t]))
            lq = np.append(lnq[at], L._log_sum(np.delete(lnq, at)))
            P, Q = np.exp(lp), np.exp(lq)
            flp, flq = (np.where(np.isfinite(a), a, 0) for a in (lp, lq))
            both = np.isfinite(lp) & np.isfinite(lq)
            d = 1.2e-5 + 3e-6 * (np.abs(flp) + np.abs(flq))
            ratio = np.where(both, np.abs(flp - flq), 0)
            each[t] = ((P + Q) * (d + 1.2e-5 * ratio)).sum()
            if self.kind == L.FORWARD:
                qf = P
            else:
                qf = Q * (ratio + 1)
            cls = np.full(V, len(at))
            cls[at] = np.arange(len(at))
            share = np.where(np.isfinite(lq[cls]), np.exp(lnq - flq[cls]), 0.0)
            share[at] = 1.0  # an entry is its class, one that the student excludes too
            y = np.where(np.isfinite(x), np.abs(x - x.max()), 0)
            grad[t] = abs(self.scale) * w[t] / self.T * (
                (1.2e-5 + 4e-7 * y) * (np.exp(lnq) * qf.sum() + share * qf[cls]) +
                share * (P + Q)[cls] * (d[cls] + each[t]))
        return each, grad

    def check(self, loss, each, got=None):
        want, rows_want, grad = self.expect()
        be, bg = self.bounds()
        w = L.weights(self.keep, self.off, self.reduce, self.norm)
        loss = to_np(loss.double())
        assert loss[0] == want or abs(loss[0] - want) <= (w * be).sum() + 1e-6 * (
            w * np.abs(rows_want)).sum()
        assert loss[1] == 7
        if each is not None:
            e = to_np(each.double())
            assert (e[len(rows_want):] == 7).all()
            e = e[:len(rows_want)]
            same = e == rows_want  # infinite where the student excludes the rest
            off = np.abs(np.where(same, 0, e) - np.where(same, 0, rows_want))
            assert np.all(off <= be + 1e-6 * np.abs(np.where(same, 0, rows_want)))
            assert not e[w == 0].any()
        if got is not None:
            g = to_np(got.double())
            err = np.abs(g - grad) - (bg + UNIT[self.dtype] * (np.abs(grad) + bg) +
                                      LEAST[self.dtype])
            assert err.max() <= 0, (err.max(), np.unravel_index(err.argmax(), err.shape))
            assert not g[w == 0].any()

    def all(self, edp, ring):
        store, d = view(*self.zd.shape, self.dtype)
        loss, each = self.run(edp, ring, d)
        edp.edp_sync(ring.ctx)
        self.check(loss, each, d)
        assert torch.isnan(store[self.zd.size:]).all()
        alone, _ = self.run(edp, ring, None, row_loss=False)  # the loss alone
        edp.edp_sync(ring.ctx)
        self.check(alone, None)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind,rest", KINDS)
@pytest.mark.parametrize("vocab", [1, 2, 9, 65, 515, 4_099, 33_001])
@pytest.mark.parametrize("rows,top", [(1, 1), (5, 20), (3, 33), (7, 64), (2, 128)])
def test_sizes(edp_lib, dtype, kind, rest, vocab, rows, top):
    c = Case(rows, vocab, top, dtype, kind, rest, vocab + rows, T=0.8 if vocab % 2 else 1.0)
    c.all(edp_lib, ctx_of(edp_lib))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,rest", KINDS)
@pytest.mark.parametrize("vocab,rows,top", [(152_064, 3, 64), (50_257, 160, 20), (20_011, 330, 5),
                                            (70_003, 200, 100)])
def test_parts_of_rows(edp_lib, dtype, kind, rest, vocab, rows, top):
    """Every number of CTAs per row; rows left out hold NaN, their lists anything."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    rng = np.random.default_rng(rows)
    keep = rng.random(rows) < (.1 if rows > 100 else .9)  # few: the oracle's time
    keep[1] = True
    c = Case(rows, vocab, top, dtype, kind, rest, rows, keep=keep, scale=-3.0)
    dead = torch.from_numpy(~keep).cuda()
    c.v[dead] = float("nan")
    c.ids[~keep] = 1 << 30
    c.value[~keep] = np.nan
    _, d = view(rows, vocab, dtype)
    loss, each = c.run(edp, ring, d)
    edp.edp_sync(ring.ctx)
    c.check(loss, each, d)
    # the loss alone, twice: the same numbers whatever order the threads ran in
    alone, one = c.run(edp, ring)
    edp.edp_sync(ring.ctx)
    c.check(alone, one)
    alone2, one2 = c.run(edp, ring)
    assert torch.equal(alone, alone2) and torch.equal(one, one2)
    # the same with the gradient, and in the logits' place
    again, each2 = c.run(edp, ring, c.v)
    edp.edp_sync(ring.ctx)
    assert torch.equal(loss, again) and torch.equal(each, each2) and torch.equal(d, c.v)


@pytest.mark.parametrize("reduce", [L.TOKEN_MEAN, L.SEQ_MEAN, L.SEQ_SUM])
@pytest.mark.parametrize("norm", [0.0, 50.0])
@pytest.mark.parametrize("rows,masked", [(40, False), (40, True), (700, True), (1_500, True),
                                         (1_500, False)])
def test_reductions(edp_lib, reduce, norm, rows, masked):
    """Sequences of every length, some empty or left out whole, tokens outside of all."""
    rng = np.random.default_rng(rows)
    off = np.sort(np.concatenate([[2, 5, 5], rng.integers(2, rows - 3, 6), [rows - 3]]))
    keep = rng.random(rows) < .7 if masked else None
    if masked:
        keep[off[4]:off[5]] = False
    c = Case(rows, 300, 8, "f32", L.FORWARD, True, rows, reduce=reduce, norm=norm, off=off,
             keep=keep)
    c.all(edp_lib, ctx_of(edp_lib))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift,stride,oshift,ostride",
                         [(1, 1003, 1, 1003), (3, 1008, 5, 1001), (0, 1024, 0, 1000),
                          (7, 1001, 0, 1003)])
def test_strides_and_alignments(edp_lib, dtype, shift, stride, oshift, ostride):
    edp, ring = edp_lib, ctx_of(edp_lib)
    rows, vocab = 9, 1000
    c = Case(rows, vocab, 20, dtype, L.REVERSE, True, 3, stride=stride, shift=shift)
    store, d = view(rows, vocab, dtype, ostride, oshift)
    loss, each = c.run(edp, ring, d)
    edp.edp_sync(ring.ctx)
    c.check(loss, each, d)
    free = torch.ones_like(store, dtype=torch.bool)
    free[oshift:oshift + rows * ostride].view(rows, ostride)[:, :vocab] = False
    assert torch.isnan(store[free]).all()


@pytest.mark.parametrize("kind,rest", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows_that_count(edp_lib, kind, rest, dtype):
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = Case(5, 200, 4, dtype, kind, rest, 1, keep=np.zeros(5, bool))
    _, d = view(5, 200, dtype)
    loss, each = c.run(edp, ring, d)
    edp.edp_sync(ring.ctx)
    assert loss.tolist() == [0, 7] and each.tolist() == [0] * 5 + [7] * 2 and not d.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind,rest", KINDS)
@pytest.mark.parametrize("vocab,top", [(24, 24), (100, 100), (128, 128), (1, 1)])
def test_lists_of_the_whole_vocabulary(edp_lib, dtype, kind, rest, vocab, top):
    """The class of all other tokens is empty: with rest = -infinity its share is 0."""
    c = Case(4, vocab, top, dtype, kind, rest, 9, absent=False)
    if rest:
        c.rest[:] = -np.inf
    c.all(edp_lib, ctx_of(edp_lib))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [60, 40_001])
@pytest.mark.parametrize("kind,rest", KINDS)
def test_excluded_tokens(edp_lib, dtype, vocab, kind, rest):
    """Tokens at -infinity outside of the list, all of those outside, and (with a
    probability that the student excludes) in it."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = Case(3, vocab, 7, dtype, kind, rest, 4, absent=False)
    for t in range(2):
        others = np.setdiff1d(np.arange(vocab), c.ids[t])
        c.zd[t, others[::3] if t == 0 else others] = -np.inf
    if rest:
        c.rest[1] = -np.inf
    c.v.copy_(torch.from_numpy(c.zd))
    c.keep[2] = False
    c.masked = True
    c.all(edp, ring)
    c.keep[:] = [False, False, True]
    c.zd[2, c.ids[2, 3]] = -np.inf
    c.v.copy_(torch.from_numpy(c.zd))
    _, d = view(3, vocab, dtype)
    loss, each = c.run(edp, ring, d)
    alone, one = c.run(edp, ring)
    edp.edp_sync(ring.ctx)
    if kind == L.FORWARD:
        assert each[2] == float("inf") and loss[0] == float("inf")
        assert one[2] == float("inf") and alone[0] == float("inf")
        _, bg = c.bounds()
        _, _, grad = c.expect()
        assert np.all(np.abs(to_np(d.double()) - grad) <=
                      bg + UNIT[dtype] * (np.abs(grad) + bg) + LEAST[dtype])
    else:
        c.check(loss, each, d)
        c.check(alone, one)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind,rest", KINDS)
@pytest.mark.parametrize("how", ["list below", "list far below", "list far above", "neighbours"])
@pytest.mark.parametrize("rows,vocab", [(2, 3_001), (3, 70_000), (160, 9_000)])
def test_lists_beside_the_row(edp_lib, dtype, kind, rest, how, rows, vocab):
    """Lists whose tokens are not the likely ones, and lists of tokens side by side (several
    to a vector, at the row's ends too)."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    keep = np.arange(rows) < 3
    c = Case(rows, vocab, 90, dtype, kind, rest, 5, absent=False, keep=keep)
    if how == "neighbours":
        for t in range(rows):
            a = [0, vocab - 90, vocab // 2][t % 3]
            c.ids[t] = np.random.default_rng(t).permutation(np.arange(a, a + 90))
    else:
        by = {"list below": -20, "list far below": -150, "list far above": 130}[how]
        for t in range(rows):
            c.zd[t, c.ids[t]] = by + np.arange(90) / 30
    c.v.copy_(torch.from_numpy(c.zd))
    c.zd = to_np(c.v.double())
    c.all(edp, ring)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [60, 40_001])
@pytest.mark.parametrize("kind,rest", KINDS)
def test_special_values(edp_lib, dtype, vocab, kind, rest):
    """NaN and infinities, a token twice, an id beyond the vocabulary, no distribution:
    each in its own row, the others as they are."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    top = 40
    c = Case(10, vocab, top, dtype, kind, rest, 4, absent=False)
    others = np.setdiff1d(np.arange(vocab), c.ids[2])
    c.v[0, others[3]] = float("nan")
    c.v[1, int(c.ids[1, 2])] = float("nan")
    c.v[2, others[-1]] = float("inf")
    c.v[3, int(c.ids[3, 0])] = float("inf")
    c.value[4, 1] = np.nan
    c.ids[5, 33] = c.ids[5, 2]
    c.ids[6, 35] = vocab
    c.v[7] = -torch.inf
    c.ids[8] = -1
    _, d = view(10, vocab, dtype)
    loss, each = c.run(edp, ring, d)
    status, msg = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID and "out of range" in msg
    e, g = to_np(each.double())[:10], to_np(d.double())
    assert np.isnan(e[:5]).all() and np.isnan(to_np(loss)[0])
    assert np.isnan(g[:5]).all()
    assert not e[5:8].any() and not g[5:8].any()
    _, alone = c.run(edp, ring)
    status, msg = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID and "out of range" in msg
    alone = to_np(alone.double())[:10]
    assert np.isnan(alone[:5]).all() and not alone[5:8].any()
    want, rows_want, grad = c.expect_rows([8, 9])
    be, bg = want
    assert np.all(np.abs(e[8:] - rows_want) <= be + 1e-6 * np.abs(rows_want))
    assert np.all(np.abs(alone[8:] - rows_want) <= be + 1e-6 * np.abs(rows_want))
    assert np.all(np.abs(g[8:] - grad) <= bg + UNIT[dtype] * (np.abs(grad) + bg) + LEAST[dtype])
    for rows, word in (([5, 9], "twice"), ([7, 9], "-infinity")):
        c.keep = np.isin(np.arange(10), rows)
        c.masked = True
        for out in (d, None):
            c.run(edp, ring, out)
            status, msg = edp.edp_sync_status(ring.ctx)
            assert status == edp.EDP_ERR_INVALID and word in msg and "row %d" % rows[0] in msg
        assert not d[rows[0]].any()
    c.keep = np.arange(10) == 9
    loss, each = c.run(edp, ring, d)
    edp.edp_sync(ring.ctx)
    assert np.isfinite(to_np(loss)[0])


def _expect_rows(self, rows):
    sub = Case.__new__(Case)
    sub.__dict__.update(self.__dict__)
    n = len(self.ids)
    sub.zd = self.zd[rows]
    sub.ids, sub.value = self.ids[rows], self.value[rows]
    sub.rest = None if self.rest is None else self.rest[rows]
    sub.keep, sub.norm = np.ones(len(rows), bool), float(n)
    _, each, grad = sub.expect()
    return sub.bounds(), each, grad


Case.expect_rows = _expect_rows


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind,rest", KINDS)
@pytest.mark.parametrize("T,vocab", [(1e-3, 600), (1e-3, 60_001), (1e3, 600)])
def test_range_of_temperatures(edp_lib, dtype, kind, rest, T, vocab):
    """Logits whose product with log2(e) / T leaves what the fused form takes."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = Case(3, vocab, 12, dtype, kind, rest, 2, absent=False)
    c.zd = c.zd if T > 1 else c.zd * 40
    c.v.copy_(torch.from_numpy(c.zd))
    c.zd = to_np(c.v.double())
    c.T = T
    c.scale = 1.0 if T > 1 else 1e-3
    c.all(edp, ring)


@pytest.mark.parametrize("dtype,vocab", [("bf16", 327_600), ("f16", 500_001), ("f32", 163_900),
                                         ("f32", 393_216)])
@pytest.mark.parametrize("kind,rest", KINDS)
def test_large_vocabularies(edp_lib, dtype, vocab, kind, rest):
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = Case(4, vocab, 128, dtype, kind, rest, 1, shift=3, keep=np.array([1, 0, 1, 1], bool))
    c.v[1] = float("nan")
    c.all(edp, ring)
    _, d = view(4, vocab, dtype, shift=1)  # at other alignments, and in place
    loss, each = c.run(edp, ring, d)
    again, each2 = c.run(edp, ring, c.v)
    edp.edp_sync(ring.ctx)
    assert torch.equal(loss, again) and torch.equal(each, each2) and torch.equal(d, c.v)


@pytest.mark.parametrize("dtype,vocab,rows", [("bf16", 8_388_608, 1), ("f32", 4_194_303, 1),
                                              ("f32", 4_194_304, 100),
                                              ("bf16", 8_388_608, 160)])
def test_largest_vocabularies(edp_lib, dtype, vocab, rows):
    """One row that counts, of one and of many (a CTA then has the whole of it)."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = Case(1, vocab, 128, dtype, L.REVERSE, True, 1)
    if rows == 1:
        c.all(edp, ring)
        _, more = view(1, vocab + 8, dtype)
        c.v = more
        with pytest.raises(edp.EdpError, match="16 MiB"):
            c.run(edp, ring)
        return
    want, _, grad = c.expect()
    be, bg = c.bounds()
    at = rows - 2
    ids = torch.zeros(rows, 128, dtype=torch.int32, device="cuda")
    value = torch.zeros(rows, 128, device="cuda")
    rest, mask = torch.zeros(rows, device="cuda"), torch.zeros(rows, dtype=torch.uint8,
                                                               device="cuda")
    ids[at], value[at], rest[at], mask[at] = cuda(c.ids)[0], cuda(c.value)[0], cuda(c.rest)[0], 1
    z = torch.empty(rows, vocab, dtype=TYPES[dtype], device="cuda")
    z[at] = c.v[0]
    loss, d = torch.zeros(1, device="cuda"), torch.full_like(z, 7.0)
    for out in (None, d):
        edp.edp_distill_loss(ring.ctx, c.config(edp), z, ids, value, loss, rest=rest, mask=mask,
                             dlogits=out)
        edp.edp_sync(ring.ctx)
        assert abs(float(loss) - want) <= be[0] + 1e-6 * abs(want)
    assert np.all(np.abs(to_np(d[at].double()) - grad[0]) <=
                  bg[0] + UNIT[dtype] * (np.abs(grad[0]) + bg[0]) + LEAST[dtype])
    assert not d[:at].any() and not d[at + 1:].any()


def test_offsets_beyond_32_bits(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    stride = (1 << 31) + 5
    c = Case(3, 1000, 10, "bf16", L.FORWARD, True, 6)
    store = torch.empty(2 * stride + 1000, dtype=torch.bfloat16, device="cuda")
    v = store.as_strided((3, 1000), (stride, 1))
    v.copy_(c.v)
    c.v = v
    loss, each = c.run(edp, ring, v)
    edp.edp_sync(ring.ctx)
    c.check(loss, each, v)
    del store, v, c
    gc.collect()


@pytest.mark.parametrize("rows", [30, 1_400])
def test_streams_graphs_and_other_calls(edp_lib, rows):
    """Captured and replayed with other inputs, between calls that share the scratch."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    keep = np.arange(rows) % 5 > 0
    off = np.array([0, rows // 3, rows // 3, rows - 1])
    make = lambda seed: Case(rows, 515, 12, "bf16", L.FORWARD, True, seed,  # noqa: E731
                             reduce=L.SEQ_MEAN, off=off, keep=keep)
    c, other = make(1), make(2)
    a = c.arrays()
    loss = torch.full((2,), 7.0, device="cuda")
    each = torch.full((rows + 2,), 7.0, device="cuda")
    d = torch.zeros(rows, 515, dtype=torch.bfloat16, device="cuda")
    ploss = torch.zeros(8, device="cuda")
    lp = torch.randn(rows, device="cuda")
    pc = edp.make_policy_config()
    s = torch.cuda.Stream()

    def calls():
        edp.edp_policy_loss(ring.ctx, pc, lp, lp, lp, rows, ploss, mask=a["mask"])
        edp.edp_distill_loss(ring.ctx, c.config(edp), c.v, a["ids"], a["value"], loss,
                             rest=a["rest"], mask=a["mask"], off=a["off"], n_seq=3,
                             row_loss=each, dlogits=d)
        edp.edp_policy_loss(ring.ctx, pc, lp, lp, lp, rows, ploss, mask=a["mask"])

    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls()
    edp.edp_sync(ring.ctx, stream=s)
    c.check(loss, each, d)
    first = ploss.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        calls()
    b = other.arrays()
    c.v.copy_(other.v)
    for k in ("ids", "value", "rest"):
        a[k].copy_(b[k])
    d.fill_(3.0)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    other.check(loss, each, d)
    assert torch.equal(ploss, first)


def test_gradient_against_differences(edp_lib):
    """The kernel's gradient against differences of its own losses, in fp32: the step h and
    losses near 1, each off by a few 2^-24 of itself (up to 1e-6), bound the error by
    1e-6 / h and h^2 times a third derivative below 1."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    h = 0.02
    for kind, rest in KINDS:
        c = Case(1, 12, 5, "f32", kind, rest, 7, absent=False)
        _, d = view(1, 12, "f32")
        c.run(edp, ring, d)
        wide = Case(24, 12, 5, "f32", kind, rest, 7)
        wide.ids[:], wide.value[:] = c.ids, c.value
        if rest:
            wide.rest[:] = c.rest
        z = np.repeat(c.zd, 24, 0)
        z[np.arange(24), np.arange(24) // 2] += np.where(np.arange(24) % 2, -h, h)
        wide.v.copy_(torch.from_numpy(z))
        exact = to_np(wide.v.double())
        step = exact[::2] - exact[1::2]
        step = step[np.arange(12), np.arange(12)]
        _, each = wide.run(edp, ring)
        edp.edp_sync(ring.ctx)
        e = to_np(each.double())[:24]
        assert np.all(np.abs((e[::2] - e[1::2]) / step - to_np(d)[0]) <= 2e-6 / h + h * h)


def test_refusals(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    c = Case(4, 100, 8, "bf16", L.FORWARD, True, 0, off=[0, 2, 4])
    a = c.arrays()
    loss, each = torch.zeros(1, device="cuda"), torch.zeros(5, device="cuda")
    d = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")

    def call(cfg=None, z=c.v, **kw):
        args = dict(ids=a["ids"], value=a["value"], loss=loss, rest=a["rest"], off=a["off"],
                    n_seq=2, row_loss=each[:4], dlogits=d[:, :100])
        args.update(kw)
        edp.edp_distill_loss(ring.ctx, cfg or edp.make_distill_config(), z, **args)

    call()
    m = edp.make_distill_config
    nan, inf = float("nan"), float("inf")
    reserved = m()
    reserved.reserved[1] = 1
    bad = [dict(cfg=x) for x in (
        m(kind=3), m(reduce=3), m(beta=.5), m(kind=edp.EDP_DISTILL_MIX, beta=0.0),
        m(kind=edp.EDP_DISTILL_MIX, beta=1.0), m(kind=edp.EDP_DISTILL_MIX, beta=nan),
        m(teacher_temperature=2.0), m(norm=-1.0), m(norm=inf), m(grad_scale=nan), reserved)]
    bad += [dict(cfg=m(teacher_temperature=x), rest=None) for x in (0.0, nan, 1e7)]
    bad += [dict(cfg=m(kind=k, beta=b), rest=None) for k, b in ((1, 0.0), (2, .5))]
    bad += [dict(temperature=0.0), dict(off=None), dict(n_seq=0), dict(value=None),
            dict(loss=None), dict(loss=torch.zeros(1)), dict(ids=a["ids"].cpu()),
            dict(row_loss=each.data_ptr() + 2), dict(off=a["off"].data_ptr() + 4),
            dict(off=None, n_seq=0, cfg=m(reduce=edp.EDP_REDUCE_SEQ_SUM)),
            dict(z=c.v[:0], ids=a["ids"][:0], dlogits=None),
            dict(ids=torch.zeros(4, 129, dtype=torch.int32, device="cuda"),
                 value=torch.zeros(4, 129, device="cuda")),
            dict(ids=torch.zeros(4, 0, dtype=torch.int32, device="cuda")),
            dict(z=c.v[:2], ids=a["ids"][:2],
                 dlogits=c.store[:400].view(2, 200)[:, :100])]  # the logits' array, other stride
    for kw in bad:
        with pytest.raises(edp.EdpError) as e:
            call(**kw)
        assert e.value.status == edp.EDP_ERR_INVALID, kw
    call()
    edp.edp_sync(ring.ctx)
