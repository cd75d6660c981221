"""Log-probabilities of given tokens and the gradient of the logits, against the
64-bit oracle on the same (rounded) inputs.

Bounds, with eps = 2^-24 and y = (z - m) / T: the constant log2(e)/T, the
difference (fp32 logits) and the product round y to 4 eps |y|, 2^x is good to
2^-22, and the sums of a row's parts (at most about 600 terms one after
another in a thread, then a tree) lose eps sqrt(600) at random and 600 eps at
the worst.  With the p-weighted |y| of the rows here below 20:
  logp, entropy:  |error| <= 1e-5 + 1e-6 |value| (S to about 8e-6, and a last rounding)
  gradient:       |error| <= (1e-5 + 4e-7 |y|) p (|g| + |h| (|ln p| + |H|)) / T
                  + the rounding of the sum and of the output's type.
"""
import numpy as np
import pytest
import torch

from gpu_util import cuda, to_np
from oracle import losses as L

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {k: torch.finfo(t).eps / 2 for k, t in TYPES.items()}  # 2^-24, 2^-8, 2^-11
LEAST = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0**-24}


def ctx_of(edp):
    cfg = edp.make_config(64, (1, 16, 16), edp.EDP_XFORM_CHW_NORM_BF16)
    return edp.Ring(cfg, action=False, reward=False, done=False)


def view(rows, vocab, dtype, stride=None, shift=0, fill=0.0):
    """A [rows][vocab] view, `shift` elements into its storage, with rows
    `stride` apart; everything around it holds NaN."""
    stride = stride or vocab
    store = torch.full((shift + rows * stride + 16,), float("nan"), dtype=TYPES[dtype],
                       device="cuda")
    v = store[shift:shift + rows * stride].view(rows, stride)[:, :vocab]
    v.fill_(fill)
    return store, v


def make(rows, vocab, dtype, seed, stride=None, shift=0, banned=0):
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 3, (rows, vocab))
    target = rng.integers(0, vocab, rows).astype(np.int32)
    z[np.arange(rows), target] += rng.normal(2, 3, rows)
    for _ in range(banned):
        col = rng.integers(0, vocab, rows)
        col = np.where(col == target, (col + 1) % vocab, col)
        z[np.arange(rows), col] = np.where(col == target, z[np.arange(rows), col], -np.inf)
    store, v = view(rows, vocab, dtype, stride, shift)
    v.copy_(torch.from_numpy(z))
    return store, v, target, to_np(v.double())


def check_forward(edp, ring, v, zd, target, T=1.0, live=None, entropy=True, stats=True, mask=None):
    rows = v.shape[0]
    out = [torch.full((rows,), 7.0, device="cuda") for _ in range(2)]
    st = torch.full((rows, 2), 7.0, device="cuda")
    edp.edp_token_logprob(ring.ctx, v, cuda(target), out[0], mask=mask, temperature=T,
                          entropy=out[1] if entropy else None, stats=st if stats else None)
    edp.edp_sync(ring.ctx)
    live = np.ones(rows, bool) if live is None else live
    logp, H, m, S = L.token_logprob(zd[live], target[live], T)
    got = to_np(out[0])
    assert np.all(np.abs(got[live] - logp) <= 1e-5 + 1e-6 * np.abs(logp))
    assert not got[~live].any()
    if entropy:
        assert np.all(np.abs(to_np(out[1])[live] - H) <= 1e-5 + 1e-6 * H)
        assert not to_np(out[1])[~live].any()
    if stats:
        s = to_np(st)
        assert np.array_equal(s[live, 0], m.astype(np.float32)) and not s[~live].any()
        assert np.all(np.abs(s[live, 1] - S) <= 1e-5 * S)
    return out[0], out[1], st


def check_grad(zd, target, g, h, T, got, dtype):
    logp, H, m, S = L.token_logprob(zd, target, T)
    ref = L.token_logprob_grad(zd, target, g, h, T)
    y = (zd - m[:, None]) / T
    y = np.where(np.isfinite(y), y, 0)
    lnp = y - np.log(S)[:, None]
    p = np.where(np.isfinite(zd), np.exp(lnp), 0)
    ah = np.zeros(len(g)) if h is None else np.abs(h)
    size = (np.abs(g)[:, None] + ah[:, None] * (np.abs(lnp) + H[:, None])) / T
    bound = (1e-5 + 4e-7 * np.abs(y)) * p * size
    at = np.zeros_like(zd)
    at[np.arange(len(g)), target] = np.abs(g) / T
    bound += UNIT[dtype] * np.abs(ref) + 2.0**-22 * at + LEAST[dtype]
    err = np.abs(got - ref)
    assert np.all(err <= bound), float((err - bound).max())


def run_grad(edp, ring, v, target, st, H, g, h, T, out, mask=None):
    edp.edp_token_logprob_grad(ring.ctx, v, cuda(target), st, cuda(g.astype(np.float32)), out,
                               mask=mask, temperature=T, entropy=H if h is not None else None,
                               dentropy=cuda(h.astype(np.float32)) if h is not None else None)
    edp.edp_sync(ring.ctx)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 65, 515, 4096, 4099, 33_001])
@pytest.mark.parametrize("rows", [1, 5])
def test_sizes(edp_lib, dtype, vocab, rows):
    ring = ctx_of(edp_lib)
    T = 0.7 if vocab % 2 else 1.0
    _, v, target, zd = make(rows, vocab, dtype, vocab + rows, banned=vocab > 100)
    rng = np.random.default_rng(vocab)
    g, h = (rng.normal(0, 1, rows).astype(np.float32).astype(np.float64) for _ in range(2))
    _, H, st = check_forward(edp_lib, ring, v, zd, target, T)
    check_forward(edp_lib, ring, v, zd, target, T, entropy=False, stats=False)
    for hh in (None, h):
        store, out = view(rows, vocab, dtype)
        run_grad(edp_lib, ring, v, target, st, H, g, hh, T, out)
        check_grad(zd, target, g, hh, T, to_np(out.double()), dtype)
        assert torch.isnan(store[rows * vocab:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift,stride,oshift,ostride",
                         [(1, 1003, 1, 1003), (3, 1008, 5, 1001), (0, 1024, 0, 1000),
                          (7, 1001, 0, 1003)])
def test_strides_and_alignments(edp_lib, dtype, shift, stride, oshift, ostride):
    """Rows at every alignment, gradients at the same and at others; nothing
    around the rows is read (it holds NaN) or written."""
    ring = ctx_of(edp_lib)
    rows, vocab = 9, 1000
    _, v, target, zd = make(rows, vocab, dtype, 3, stride, shift)
    g = np.linspace(-1, 1, rows).astype(np.float32).astype(np.float64)
    _, H, st = check_forward(edp_lib, ring, v, zd, target)
    store, out = view(rows, vocab, dtype, ostride, oshift)
    run_grad(edp_lib, ring, v, target, st, H, g, g, 1.0, out)
    check_grad(zd, target, g, g, 1.0, to_np(out.double()), dtype)
    free = torch.ones_like(store, dtype=torch.bool)
    free[oshift:oshift + rows * ostride].view(rows, ostride)[:, :vocab] = False
    assert torch.isnan(store[free]).all()


@pytest.mark.parametrize("rows", [3, 150, 400])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_masks_and_many_rows(edp_lib, rows, dtype):
    """Any number of CTAs per row; rows left out by mask or target hold NaN."""
    ring = ctx_of(edp_lib)
    vocab = 20_011
    _, v, target, zd = make(rows, vocab, dtype, rows)
    rng = np.random.default_rng(rows)
    mask = (rng.random(rows) < .8).astype(np.uint8)
    target[rng.random(rows) < .1] = -1
    live = (mask > 0) & (target >= 0)
    v[torch.from_numpy(~live).cuda()] = float("nan")
    g, h = (rng.normal(0, 1, rows).astype(np.float32).astype(np.float64) for _ in range(2))
    _, H, st = check_forward(edp_lib, ring, v, zd, target, live=live, mask=cuda(mask))
    run_grad(edp_lib, ring, v, target, st, H, g, h, 1.0, v, mask=cuda(mask))
    got = to_np(v.double())
    check_grad(zd[live], target[live], g[live], h[live], 1.0, got[live], dtype)
    assert not got[~live].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 5000, 40_000])
def test_special_values(edp_lib, dtype, vocab):
    """The type's lowest value and -infinity as masks, one allowed token, no
    allowed token, NaN and +infinity, a target that is excluded."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    low = torch.finfo(TYPES[dtype]).min
    store, v = view(8, vocab, dtype)
    v.normal_(0, 1)
    v[0, 1:] = low                      # one token has all the probability
    v[1, :] = low                       # uniform
    v[2, 1:] = -torch.inf
    v[3, :] = -torch.inf                # reported, written as 0
    v[4, vocab // 2] = float("nan")
    v[5, vocab - 1] = torch.inf
    v[6, 3] = -torch.inf                # the target itself
    v[7, :] = torch.finfo(TYPES[dtype]).max
    target = np.array([0, 5, 0, 0, 0, 0, 3, 9], np.int32)
    logp, H = (torch.full((8,), 7.0, device="cuda") for _ in range(2))
    st = torch.full((8, 2), 7.0, device="cuda")
    edp.edp_token_logprob(ring.ctx, v, cuda(target), logp, entropy=H, stats=st)
    status, msg = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID and "-infinity" in msg and "row 3" in msg
    lp, ent = to_np(logp), to_np(H)
    ln = np.log(vocab)
    assert abs(lp[0]) <= 1e-6 and abs(ent[0]) <= 1e-5
    assert abs(lp[1] + ln) <= 2e-5 and abs(ent[1] - ln) <= 2e-5
    assert abs(lp[2]) <= 1e-6 and abs(ent[2]) <= 1e-5
    assert lp[3] == 0 and ent[3] == 0 and not to_np(st)[3].any()
    assert np.isnan(lp[4:6]).all() and np.isnan(ent[4:6]).all()
    assert lp[6] == -np.inf and np.isfinite(ent[6])
    assert abs(lp[7] + ln) <= 2e-5 and abs(ent[7] - ln) <= 2e-5
    g = torch.ones(8, device="cuda")
    out = torch.full_like(v, 7.0)
    edp.edp_token_logprob_grad(ring.ctx, v, cuda(target), st, g, out, entropy=H, dentropy=g)
    edp.edp_sync(ring.ctx)
    d = to_np(out.double())
    assert np.isfinite(d[[0, 1, 2, 3, 6, 7]]).all() and not d[3].any()
    assert np.isnan(d[4]).all() and np.isnan(d[5]).all()
    assert np.all(np.abs(d[0]) <= 1e-5) and np.all(np.abs(d[2]) <= 1e-5)
    assert abs(d[1, 5] - (1 - 1 / vocab)) <= 5e-3 and abs(d[6, 3] - 1) <= 1e-6


def test_bad_target_is_reported(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    _, v, target, zd = make(4, 100, "f32", 0)
    target[2] = 100
    logp = torch.full((4,), 7.0, device="cuda")
    edp.edp_token_logprob(ring.ctx, v, cuda(target), logp)
    status, _ = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID and to_np(logp)[2] == 0 and to_np(logp)[3] != 0
    out = torch.full_like(v, 7.0)
    st = torch.ones(4, 2, device="cuda")
    edp.edp_token_logprob_grad(ring.ctx, v, cuda(target), st, logp, out)
    status, _ = edp.edp_sync_status(ring.ctx)
    assert status == edp.EDP_ERR_INVALID and not to_np(out)[2].any() and to_np(out)[3].any()


def test_gradient_against_differences(edp_lib):
    """The GPU's gradient of sum g logp + h entropy against central differences
    of the 64-bit loss (step 1e-5: an error of about 1e-9)."""
    ring = ctx_of(edp_lib)
    _, v, target, zd = make(2, 11, "f32", 8)
    g, h = np.array([.5, -2.0]), np.array([1.5, .25])
    _, H, st = check_forward(edp_lib, ring, v, zd, target, 0.5)
    out = torch.zeros_like(v)
    run_grad(edp_lib, ring, v, target, st, H, g, h, 0.5, out)

    def f(x):
        logp, ent, _, _ = L.token_logprob(x, target, .5)
        return g @ logp + h @ ent

    for i in np.ndindex(*zd.shape):
        a, b = zd.copy(), zd.copy()
        a[i] += 1e-5
        b[i] -= 1e-5
        assert abs(to_np(out)[i] - (f(a) - f(b)) / 2e-5) <= 2e-5


def test_rows_beyond_32_bits(edp_lib):
    """Elements beyond 2^31, bytes beyond 2^32: the last rows of a large array."""
    ring = ctx_of(edp_lib)
    rows, vocab = 16_500, 131_072
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    assert z.numel() > 2**31
    tail = torch.randn(3, vocab, device="cuda").to(torch.bfloat16)
    z[-3:] = tail
    target = np.full(rows, 17, np.int32)
    mask = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    mask[-3:] = 1
    mask[:2] = 1
    logp, H = torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda")
    st = torch.zeros(rows, 2, device="cuda")
    edp_lib.edp_token_logprob(ring.ctx, z, cuda(target), logp, mask=mask, entropy=H, stats=st)
    g = torch.ones(rows, device="cuda")
    edp_lib.edp_token_logprob_grad(ring.ctx, z, cuda(target), st, g, z, mask=mask)
    edp_lib.edp_sync(ring.ctx)
    zd = to_np(tail.double())
    ref = L.token_logprob(zd, target[-3:])
    assert np.all(np.abs(to_np(logp)[-3:] - ref[0]) <= 1e-5 + 1e-6 * np.abs(ref[0]))
    assert np.all(np.abs(to_np(logp)[:2] + np.log(vocab)) <= 3e-5) and not to_np(logp)[2:-3].any()
    check_grad(zd, target[-3:], np.ones(3), None, 1.0, to_np(z[-3:].double()), "bf16")
    assert int((z[2:-3] != 0).sum()) == 0 and int((z[:2] == 0).sum()) == 0


def test_streams_graph_and_repeatability(edp_lib):
    """The same bits on another stream, from a graph, and again."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    _, v, target, zd = make(37, 30_000, "bf16", 4)
    t, g = cuda(target), torch.randn(37, device="cuda")

    def go(stream=None):
        o = [torch.zeros(37, device="cuda") for _ in range(2)]
        st, d = torch.zeros(37, 2, device="cuda"), torch.zeros_like(v)
        torch.cuda.synchronize()
        edp.edp_token_logprob(ring.ctx, v, t, o[0], entropy=o[1], stats=st, stream=stream)
        edp.edp_token_logprob_grad(ring.ctx, v, t, st, g, d, entropy=o[1], dentropy=g,
                                   stream=stream)
        return [*o, st, d]

    a = go()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b = go(side)
    side.synchronize()
    outs = [torch.zeros_like(x) for x in a]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        edp.edp_token_logprob(ring.ctx, v, t, outs[0], entropy=outs[1], stats=outs[2])
        edp.edp_token_logprob_grad(ring.ctx, v, t, outs[2], g, outs[3], entropy=outs[1],
                                   dentropy=g)
    graph.replay()
    torch.cuda.synchronize()
    for x, y, w in zip(a, b, outs):
        assert torch.equal(x, y) and torch.equal(x, w)


def test_refusals(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    z = torch.zeros(4, 10, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    o, st = torch.zeros(4, device="cuda"), torch.zeros(4, 2, device="cuda")
    host = torch.zeros(4)

    def refused(f, *a, **k):
        with pytest.raises(edp.EdpError) as e:
            f(ring.ctx, *a, **k)
        assert e.value.status == edp.EDP_ERR_INVALID
        assert "edp_token_logprob" in str(e.value)

    for T in (0.0, -1.0, float("nan"), float("inf")):
        refused(edp.edp_token_logprob, z, t, o, temperature=T)
        refused(edp.edp_token_logprob_grad, z, t, st, o, z, temperature=T)
    refused(edp.edp_token_logprob, z, None, o)
    refused(edp.edp_token_logprob, z, t, None)
    refused(edp.edp_token_logprob, z, t, host)
    refused(edp.edp_token_logprob, z.cpu(), t, o)
    refused(edp.edp_token_logprob, z, t, o, mask=torch.zeros(4, dtype=torch.uint8))
    refused(edp.edp_token_logprob_grad, z, t, st, o, z, entropy=o)
    refused(edp.edp_token_logprob_grad, z, t, st, o, z, dentropy=o)
    refused(edp.edp_token_logprob_grad, z, t, None, o, z)
    refused(edp.edp_token_logprob_grad, z, t, st, o, None)
    wide = torch.zeros(4, 20, device="cuda")
    with pytest.raises(ValueError):
        edp.edp_token_logprob(ring.ctx, wide[:, ::2], t, o)
    with pytest.raises(TypeError):
        edp.edp_token_logprob(ring.ctx, z.double(), t, o)
    with pytest.raises(ValueError):
        edp.edp_token_logprob_grad(ring.ctx, z, t, st, o, wide)
    lib = edp.lib()
    args = (0, 4, 10, 10, t.data_ptr(), None, 1.0, o.data_ptr(), None, None, None)
    ok = lib.edp_token_logprob(ring.ctx, z.data_ptr(), *args)
    assert ok == edp.EDP_OK
    for i, bad in [(0, 3), (2, 0), (3, 9), (1, 1 << 31)]:
        a = list(args)
        a[i] = bad
        assert lib.edp_token_logprob(ring.ctx, z.data_ptr(), *a) == edp.EDP_ERR_INVALID
    assert lib.edp_token_logprob(ring.ctx, z.data_ptr() + 2, *args) == edp.EDP_ERR_INVALID
    assert lib.edp_token_logprob(None, z.data_ptr(), *args) == edp.EDP_ERR_INVALID
    # in place with another stride
    grad = (0, 4, 10, 10, t.data_ptr(), None, 1.0, st.data_ptr(), None, o.data_ptr(), None)
    assert lib.edp_token_logprob_grad(ring.ctx, wide.data_ptr(), *grad, wide.data_ptr(), 20,
                                      None) == edp.EDP_ERR_INVALID
    # no rows: nothing is done, nothing is looked at
    assert edp.edp_token_logprob(ring.ctx, z[:0], None, None) == edp.EDP_OK
    edp.edp_sync(ring.ctx)
