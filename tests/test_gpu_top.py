"""The likeliest tokens of rows of logits, against the 64-bit oracle on the same (rounded)
inputs.

Ids are compared exactly (equal logits go by their index).  Bounds, with eps = 2^-24 and
y = (z - m) / T: log2(e)/T, the difference and the product round y to 4 eps |y|, 2^x is good
to 2^-22, and the sums of a row's parts (at most about 600 terms one after another in a
thread, then a tree) lose eps sqrt(600) at random and 600 eps at the worst, so that the
logarithm of a sum is good to 8e-6.  With the |y| of a value and of its maximum below 40 and
a last rounding,
  top_logp, logp, entropy, rest:  |error| <= 1e-5 + 1e-6 |value|,  S: 1e-5 of it.
"""
import numpy as np
import pytest
import torch

from gpu_util import cuda, to_np
from oracle import losses as L

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def ctx_of(edp):
    cfg = edp.make_config(64, (1, 16, 16), edp.EDP_XFORM_CHW_NORM_BF16)
    return edp.Ring(cfg, action=False, reward=False, done=False)


def view(rows, vocab, dtype, stride=None, shift=0):
    """A [rows][vocab] view, `shift` elements into its storage, with rows `stride` apart;
    everything around it holds NaN."""
    stride = stride or vocab
    store = torch.full((shift + rows * stride + 16,), float("nan"), dtype=TYPES[dtype],
                       device="cuda")
    return store, store[shift:shift + rows * stride].view(rows, stride)[:, :vocab]


def make(rows, vocab, dtype, seed, stride=None, shift=0, banned=0, scale=3.0):
    rng = np.random.default_rng(seed)
    z = rng.normal(0, scale, (rows, vocab))
    for t in range(rows):
        z[t, rng.permutation(vocab)[:min(banned, vocab - 1)]] = -np.inf
    target = rng.integers(0, vocab, rows).astype(np.int32)
    _, v = view(rows, vocab, dtype, stride, shift)
    v.copy_(torch.from_numpy(z))
    return v, target, to_np(v.double())


def outputs(rows, top, pad=3):
    f = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
    return dict(ids=torch.full((rows + pad, top), 77, dtype=torch.int32, device="cuda")[:rows],
                top_logp=f(rows + pad, top)[:rows], logp=f(rows + pad)[:rows],
                entropy=f(rows + pad)[:rows], rest=f(rows + pad)[:rows],
                stats=f(rows + pad, 2)[:rows])


def near(got, want):
    with np.errstate(invalid="ignore"):
        return np.all((got == want) | (np.abs(got - want) <= 1e-5 + 1e-6 * np.abs(want)))


def check(o, zd, target, top, T=1.0, live=None):
    rows = len(zd)
    live = np.ones(rows, bool) if live is None else live
    ids, logp, rest = L.token_top(zd[live], top, T)
    assert np.array_equal(to_np(o["ids"])[live], ids)
    assert near(to_np(o["top_logp"])[live], logp)
    assert near(to_np(o["rest"])[live], rest)
    lp, H, m, S = L.token_logprob(zd[live], target[live], T)
    for k, want in (("logp", lp), ("entropy", H)):
        if k in o:
            assert near(to_np(o[k])[live], want), k
            assert not to_np(o[k])[~live].any()
    if "stats" in o:
        s = to_np(o["stats"])
        assert np.array_equal(s[live, 0], m.astype(np.float32)) and not s[~live].any()
        assert np.all(np.abs(s[live, 1] - S) <= 1e-5 * S)
    assert (to_np(o["ids"])[~live] == -1).all() and not to_np(o["rest"])[~live].any()
    assert np.isneginf(to_np(o["top_logp"])[~live]).all()
    for x in o.values():  # what is behind the last row is left as it was
        n = x.numel()
        behind = x.new_empty(0).set_(x.untyped_storage(), x.storage_offset() + n,
                                     (x.untyped_storage().nbytes() // x.element_size() - n,))
        assert ((behind == 7) | (behind == 77)).all()


def run(edp, ring, v, target, o, T=1.0, mask=None, stream=None):
    edp.edp_token_top(ring.ctx, v, o["ids"], o["top_logp"],
                      target=cuda(target) if target is not None else None, logp=o.get("logp"),
                      mask=cuda(mask) if mask is not None else None, temperature=T,
                      entropy=o.get("entropy"), rest=o.get("rest"), stats=o.get("stats"),
                      stream=stream)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 9, 65, 130, 515, 2_000, 4_099, 33_001])
@pytest.mark.parametrize("rows,top", [(1, 1), (5, 8), (1, 33), (3, 64), (2, 128), (4, 127)])
def test_sizes(edp_lib, dtype, vocab, rows, top):
    ring = ctx_of(edp_lib)
    T = 0.7 if vocab % 2 else 1.0
    v, target, zd = make(rows, vocab, dtype, vocab + top, banned=5 if vocab > 100 else 0)
    target = np.where(np.isneginf(zd[np.arange(rows), target]), zd.argmax(1), target)
    target = target.astype(np.int32)
    o = outputs(rows, top)
    run(edp_lib, ring, v, target, o, T)
    edp_lib.edp_sync(ring.ctx)
    check(o, zd, target, top, T)
    less = {k: x for k, x in outputs(rows, top).items() if k in ("ids", "top_logp", "rest")}
    run(edp_lib, ring, v, None, less, T)  # the list alone, without a target
    edp_lib.edp_sync(ring.ctx)
    check(less, zd, target, top, T)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,rows,top", [(999, 3_001, 7), (2_047, 1_500, 32), (300, 801, 64),
                                            (2_100, 2_000, 32), (152_064, 1, 20),
                                            (152_064, 3, 128), (50_257, 160, 64),
                                            (20_011, 400, 5), (262_147, 2, 100),
                                            (70_003, 330, 128)])
def test_parts_of_rows(edp_lib, dtype, vocab, rows, top):
    """Every number of CTAs per row, with masks and targets that leave rows out (they hold
    NaN)."""
    ring = ctx_of(edp_lib)
    v, target, zd = make(rows, vocab, dtype, rows, scale=2.0)
    rng = np.random.default_rng(rows)
    mask = (rng.random(rows) < .8).astype(np.uint8)
    mask[0] = 1
    target[1:][rng.random(rows - 1) < .1] = -1
    live = (mask > 0) & (target >= 0)
    v[torch.from_numpy(~live).cuda()] = float("nan")
    if rows > 100:  # the oracle sorts: enough of them
        live_few = live & (np.arange(rows) % 8 < 2)
    else:
        live_few = live
    o = outputs(rows, top)
    run(edp_lib, ring, v, target, o, mask=mask)
    edp_lib.edp_sync(ring.ctx)
    few = np.flatnonzero(live_few)
    pick = {k: x[torch.from_numpy(few).cuda()] for k, x in o.items()}
    check_rows = np.ones(len(few), bool)
    ids, logp, rest = L.token_top(zd[few], top)
    assert np.array_equal(to_np(pick["ids"]), ids) and near(to_np(pick["top_logp"]), logp)
    assert near(to_np(pick["rest"]), rest) and check_rows.all()
    lp, H, _, _ = L.token_logprob(zd[few], target[few])
    assert near(to_np(pick["logp"]), lp) and near(to_np(pick["entropy"]), H)
    dead = torch.from_numpy(~live).cuda()
    assert (o["ids"][dead] == -1).all() and torch.isneginf(o["top_logp"][dead]).all()
    for k in ("logp", "entropy", "rest", "stats"):
        assert not o[k][dead].any()
    # the same numbers whatever order the threads ran in
    again = outputs(rows, top)
    run(edp_lib, ring, v, target, again, mask=mask)
    edp_lib.edp_sync(ring.ctx)
    for k in o:
        assert torch.equal(o[k], again[k]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift,stride", [(1, 1003), (3, 1008), (0, 1024), (7, 1001)])
def test_strides_and_alignments(edp_lib, dtype, shift, stride):
    ring = ctx_of(edp_lib)
    v, target, zd = make(9, 1000, dtype, 3, stride, shift)
    o = outputs(9, 24)
    run(edp_lib, ring, v, target, o)
    edp_lib.edp_sync(ring.ctx)
    check(o, zd, target, 24)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 1_000, 1_900, 5_000, 40_000, 152_064])
@pytest.mark.parametrize("top", [3, 32, 100])
def test_ties(edp_lib, dtype, vocab, top):
    """Rows of equal logits, by the thousand: the lowest indexes come first."""
    ring = ctx_of(edp_lib)
    rng = np.random.default_rng(vocab)
    z = np.zeros((9, vocab))
    z[1] = -3.25
    z[2] = np.where(np.arange(vocab) % 2, -0.0, 0.0)    # both zeros are one number
    z[3] = rng.integers(0, 2, vocab)                    # two values
    z[4, ::3] = 1.0
    z[5] = float(torch.finfo(TYPES[dtype]).min)         # masked by the lowest value
    z[5, vocab // 2] = 1.0
    z[6] = -np.inf                                      # fewer tokens than the list has room for
    z[6, [vocab - 1, 3]] = 2.0
    z[7] = float(torch.finfo(TYPES[dtype]).max)
    z[8, vocab - 1], z[8, 0] = 1.0, 1.0
    _, v = view(9, vocab, dtype)
    v.copy_(torch.from_numpy(z))
    zd = to_np(v.double())
    target = np.full(9, 3, np.int32)
    o = outputs(9, top)
    run(edp_lib, ring, v, target, o)
    edp_lib.edp_sync(ring.ctx)
    got = to_np(o["ids"])
    for t in range(9):
        order = np.lexsort((np.arange(vocab), -zd[t]))
        order = order[zd[t, order] > -np.inf][:top]
        want = np.full(top, -1)
        want[:len(order)] = order
        assert np.array_equal(got[t], want), t
    rows = [0, 1, 2, 3, 4, 6, 7, 8]  # row 5: differences of 1e38 in the oracle's rest
    check({k: x[torch.tensor(rows).cuda()].clone() for k, x in o.items()}, zd[rows],
          target[rows], top)
    low = to_np(o["top_logp"])[5]
    assert low[0] == 0 and (low[1:] < -60_000).all() and to_np(o["rest"])[5] < -60_000


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1e-6, 1e-3, 1e3])
@pytest.mark.parametrize("vocab", [17, 600, 60_001])
def test_range_of_temperatures(edp_lib, dtype, T, vocab):
    """Logits whose product with log2(e) / T leaves what the fused form takes."""
    ring = ctx_of(edp_lib)
    v, target, zd = make(4, vocab, dtype, 11, scale=30.0)
    target = zd.argmax(1).astype(np.int32)
    o = outputs(4, 16)
    run(edp_lib, ring, v, target, o, T)
    edp_lib.edp_sync(ring.ctx)
    ids, logp, rest = L.token_top(zd, 16, T)
    assert np.array_equal(to_np(o["ids"]), ids)
    # y itself is rounded: by 4 eps = 2.4e-7 of it
    for k, want in (("top_logp", logp), ("rest", rest)):
        assert near(to_np(o[k]).astype(np.float64), want), k
    assert near(to_np(o["logp"]), L.token_logprob(zd, target, T)[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 900, 5_000, 40_000, 200_000])
def test_special_values(edp_lib, dtype, vocab):
    edp, ring = edp_lib, ctx_of(edp_lib)
    _, v = view(8, vocab, dtype)
    v.normal_(0, 1)
    v[0, 1:] = -torch.inf               # one token has all the probability
    v[1] = -torch.inf                   # reported, an empty list
    v[2, vocab // 2] = float("nan")
    v[3, vocab - 1] = torch.inf
    v[4] = float("nan")
    v[5] = -torch.inf
    v[5, 7] = float("nan")
    v[6, 3] = -torch.inf                # the target itself
    target = np.array([0, 0, 0, 0, 0, 0, 3, vocab], np.int32)
    o = outputs(8, 9)
    run(edp, ring, v, target, o)
    status, msg = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID and "out of range" in msg
    ids, lp = to_np(o["ids"]), to_np(o["top_logp"])
    assert ids[0].tolist() == [0] + [-1] * 8 and abs(lp[0, 0]) <= 1e-6
    assert np.isneginf(lp[0, 1:]).all() and np.isneginf(to_np(o["rest"])[0])
    assert abs(to_np(o["entropy"])[0]) <= 1e-6 and abs(to_np(o["logp"])[0]) <= 1e-6
    for t in (1, 7):
        assert (ids[t] == -1).all() and np.isneginf(lp[t]).all()
        for k in ("logp", "entropy", "rest", "stats"):
            assert not to_np(o[k])[t].any()
    for t in (2, 3, 4, 5):
        assert (ids[t] == -1).all() and np.isnan(lp[t]).all()
        for k in ("logp", "entropy", "rest"):
            assert np.isnan(to_np(o[k])[t]).all(), (t, k)
    assert (ids[6] >= 0).all() and to_np(o["logp"])[6] == -np.inf
    assert np.isfinite(to_np(o["entropy"])[6])
    one = outputs(2, 9)
    run(edp, ring, v[1:2], target[1:2], {k: x[:1] for k, x in one.items()})
    status, msg = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID and "-infinity" in msg and "row 0" in msg


@pytest.mark.parametrize("dtype,vocab", [("bf16", 786_432), ("f16", 786_431), ("f32", 393_216),
                                         ("f32", 1_500_001), ("bf16", 3_000_007)])
def test_large_vocabularies(edp_lib, dtype, vocab):
    edp, ring = edp_lib, ctx_of(edp_lib)
    v, target, zd = make(2, vocab, dtype, 1, shift=3)
    o = outputs(2, 128)
    run(edp, ring, v, target, o)
    edp.edp_sync(ring.ctx)
    check(o, zd, target, 128)


def skewed(rows, vocab, how, seed):
    """Rows whose sample says little, or the wrong thing, about the rest."""
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 1, (rows, vocab))
    if how == "rising":
        z = np.sort(z, 1)
    elif how == "falling":
        z = -np.sort(z, 1)
    elif how == "block":    # all that counts is in one stretch
        z[:, vocab // 3:vocab // 3 + 400] += 30
    elif how == "few":      # as many likely tokens as the list has, nothing near them
        for t in range(rows):
            z[t] -= 300
            z[t, rng.permutation(vocab)[:100]] += 300
    elif how == "comb":     # every 64th token, which are a few threads' alone
        z[:, 5::64] += 20
    elif how == "steps":    # a few values, hundreds of each
        z = np.round(2 * z) / 2
    return z


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("how", ["rising", "falling", "block", "few", "comb", "steps"])
@pytest.mark.parametrize("rows,vocab,top", [(50, 1_024, 20), (7, 2_040, 31), (700, 900, 20),
                                            (1_300, 1_999, 9), (3, 3_000, 40),
                                            (2, 30_011, 128), (2, 100_003, 100),
                                            (160, 40_000, 20)])
def test_skewed_rows(edp_lib, dtype, how, rows, vocab, top):
    ring = ctx_of(edp_lib)
    _, v = view(rows, vocab, dtype)
    few = min(rows, 3)
    z = skewed(few, vocab, how, vocab)
    v.copy_(torch.from_numpy(z).repeat((rows + few - 1) // few, 1)[:rows])
    zd = to_np(v[:few].double())
    target = np.full(rows, 7, np.int32)
    o = outputs(rows, top)
    run(edp_lib, ring, v, target, o)
    edp_lib.edp_sync(ring.ctx)
    check({k: x[:few].clone() for k, x in o.items()}, zd, target[:few], top)
    # the same rows at other alignments, whose sums go in another order: each within its bound
    for x in o.values():
        rest = x[few:few + (rows - few) // few * few].double()
        want = x[:few].double().repeat((len(rest) // few,) + (1,) * (x.dim() - 1))
        assert torch.all((rest == want) | ((rest - want).abs() <= 2e-5 + 2e-6 * want.abs()) |
                         (rest - want).isnan())
    ids = o["ids"][:rows // few * few].view(-1, few, top)
    assert (ids == ids[0]).all()


def test_offsets_beyond_32_bits(edp_lib):
    ring = ctx_of(edp_lib)
    stride = (1 << 31) + 5
    store = torch.empty(2 * stride + 1000, dtype=torch.bfloat16, device="cuda")
    v = store.as_strided((3, 1000), (stride, 1))
    v.normal_(0, 3)
    target = np.array([1, 2, 3], np.int32)
    o = outputs(3, 10)
    run(edp_lib, ring, v, target, o)
    edp_lib.edp_sync(ring.ctx)
    check(o, to_np(v.double()), target, 10)


@pytest.mark.parametrize("top", [1, 64])
def test_equal_at_the_end_of_the_longest_rows(edp_lib, top):
    """Equal numbers, more than a row's candidates may be, at the end of 2^29 columns and more:
    the search for the last of them passes sizes whose eighth part fits 29 bits.  One row of 77
    is in use (with fewer the row would be split)."""
    ring = ctx_of(edp_lib)
    rows, vocab, n = 77, (1 << 29) + 3, 1_500
    if torch.cuda.mem_get_info()[0] < 2 * rows * vocab + (4 << 30):
        pytest.skip("too little memory is free")
    z = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
    z[-2].fill_(float("-inf"))
    z[-2, -n:] = 1.0
    mask = np.zeros(rows, np.uint8)
    mask[-2] = 1
    o = {k: x for k, x in outputs(rows, top).items() if k in ("ids", "top_logp", "rest")}
    run(edp_lib, ring, z, None, o, mask=mask)
    edp_lib.edp_sync(ring.ctx)
    del z
    torch.cuda.empty_cache()
    live = mask != 0
    ids, logp, rest = (to_np(o[k]) for k in ("ids", "top_logp", "rest"))
    assert np.array_equal(ids[live][0], vocab - n + np.arange(top))
    assert near(logp[live], np.full((1, top), -np.log(n))) and near(rest[live], np.log1p(-top / n))
    assert (ids[~live] == -1).all() and np.isneginf(logp[~live]).all() and not rest[~live].any()


def test_stream_and_graph(edp_lib):
    """On a stream of its own, and captured: replays read what the arrays then hold."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    v, target, zd = make(40, 33_001, "bf16", 8)
    o, s = outputs(40, 20), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    tgt = cuda(target)
    call = lambda: edp.edp_token_top(  # noqa: E731
        ring.ctx, v, o["ids"], o["top_logp"], target=tgt, logp=o["logp"], entropy=o["entropy"],
        rest=o["rest"], stats=o["stats"])
    with torch.cuda.stream(s):
        call()
    edp.edp_sync(ring.ctx, stream=s)
    check(o, zd, target, 20)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call()
    v2, target2, zd2 = make(40, 33_001, "bf16", 9)
    v.copy_(v2)
    tgt.copy_(cuda(target2))
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    check(o, zd2, target2, 20)


def test_refusals(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    v, target, _ = make(4, 100, "bf16", 0)
    o, tgt = outputs(4, 8), cuda(target)
    call = lambda ids=o["ids"], lp=o["top_logp"], z=v, **kw: edp.edp_token_top(  # noqa: E731
        ring.ctx, z, ids, lp, **kw)
    call()
    bad = dict(logp=o["logp"]), dict(temperature=0.0), dict(temperature=float("nan")), \
        dict(ids=torch.zeros(4, 129, dtype=torch.int32, device="cuda"),
             lp=torch.zeros(4, 129, device="cuda")), \
        dict(ids=torch.zeros(4, 0, dtype=torch.int32, device="cuda")), dict(lp=None), \
        dict(rest=torch.zeros(4)), dict(target=target.ctypes.data), \
        dict(entropy=o["entropy"].data_ptr() + 2), dict(mask=torch.ones(4, dtype=torch.uint8))
    for kw in bad:
        with pytest.raises(edp.EdpError) as e:
            call(**kw)
        assert e.value.status == edp.EDP_ERR_INVALID, kw
    call(target=tgt, logp=o["logp"])
    edp.edp_token_top(ring.ctx, v[:0], o["ids"][:0], o["top_logp"][:0])
    edp.edp_sync(ring.ctx)
