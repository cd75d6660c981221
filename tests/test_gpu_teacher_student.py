"""A teacher's lists and the student's step on them together, as a program uses them: the
arrays that edp_token_top writes go to edp_distill_loss as they are.  The oracle makes both
steps in 64 bits; the lists' fp32 numbers are the kernel's own, so that the second step's
bounds are those of the loss's tests."""
import gc

import numpy as np
import pytest
import torch

from gpu_util import to_np
from oracle import losses as L

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {k: torch.finfo(t).eps / 2 for k, t in TYPES.items()}
LEAST = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0**-24}


def ctx_of(edp):
    cfg = edp.make_config(64, (1, 16, 16), edp.EDP_XFORM_CHW_NORM_BF16)
    return edp.Ring(cfg, action=False, reward=False, done=False)


def near(got, want):
    """The lists' bounds; -infinity (no token) is only near itself."""
    with np.errstate(invalid="ignore"):
        return np.all((got == want) | (np.abs(got - want) <= 1e-5 + 1e-6 * np.abs(want)))


class Batch:
    """Logits of a teacher and of a student, tokens, sequences and a mask."""

    def __init__(self, rows, vocab, top, teacher, student, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.t = (3 * torch.randn(rows, vocab, generator=g, device="cuda")).to(TYPES[teacher])
        noise = torch.randn(rows, vocab, generator=g, device="cuda")
        self.s = (self.t.float() + noise).to(TYPES[student])
        self.mask = (torch.rand(rows, generator=g, device="cuda") < .8).to(torch.uint8)
        self.off = torch.tensor([0, rows // 4, rows // 4, rows - 2], device="cuda")
        self.ids = torch.full((rows, top), 7, dtype=torch.int32, device="cuda")
        self.lp = torch.full((rows, top), 7.0, device="cuda")
        self.rest, self.each = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
        self.loss = torch.full((1,), 7.0, device="cuda")
        self.dtype = student

    def teach(self, edp, ring, temperature=1.0):
        edp.edp_token_top(ring.ctx, self.t, self.ids, self.lp, mask=self.mask, rest=self.rest,
                          temperature=temperature)

    def learn(self, edp, ring, cfg, dlogits, with_rest=True):
        edp.edp_distill_loss(ring.ctx, cfg, self.s, self.ids, self.lp, self.loss,
                             rest=self.rest if with_rest else None, mask=self.mask,
                             off=self.off, n_seq=3, row_loss=self.each, dlogits=dlogits)

    def check(self, s0, d, kind, beta, reduce, with_rest):
        keep = to_np(self.mask) > 0
        ids, lp, rest = to_np(self.ids), to_np(self.lp).astype(float), to_np(self.rest)
        # the lists are the teacher's
        want = L.token_top(to_np(self.t.double())[keep], ids.shape[1])
        assert np.array_equal(ids[keep], want[0]) and (ids[~keep] == -1).all()
        assert near(lp[keep], want[1]) and near(rest[keep], want[2])
        # and the loss is of them
        loss, each, grad = L.distill(s0, ids, lp, rest.astype(float) if with_rest else None, keep,
                                     to_np(self.off), kind, beta, reduce)
        # |ln p|, |ln q| and their differences are below 40 here: 2 (1.2e-5 + 1.2e-5 40 +
        # 3e-6 80) < 1.5e-3 of a probability at the worst, of which the sum is 2
        tol = 1.5e-3
        assert abs(float(self.loss) - loss) <= tol
        assert np.all(np.abs(to_np(self.each) - each) <= tol)
        w = L.weights(keep, to_np(self.off), reduce)
        bound = tol * w[:, None] + UNIT[self.dtype] * np.abs(grad) + LEAST[self.dtype]
        assert np.all(np.abs(to_np(d.double()) - grad) <= bound)


@pytest.mark.parametrize("teacher,student", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("kind,beta,with_rest", [(L.FORWARD, 0.0, True), (L.FORWARD, 0.0, False),
                                                 (L.REVERSE, 0.0, True), (L.MIX, 0.6, True)])
@pytest.mark.parametrize("rows,vocab,top", [(9, 97, 100), (24, 4_001, 20), (60, 33_003, 64),
                                            (1_500, 301, 12), (1_200, 2_600, 40)])
def test_lists_to_loss(edp_lib, teacher, student, kind, beta, with_rest, rows, vocab, top):
    edp, ring = edp_lib, ctx_of(edp_lib)
    b = Batch(rows, vocab, top, teacher, student, rows + top)
    s0 = to_np(b.s.double())
    cfg = edp.make_distill_config(kind, edp.EDP_REDUCE_SEQ_MEAN, beta)
    b.teach(edp, ring)
    b.learn(edp, ring, cfg, b.s, with_rest)  # in the logits' place
    edp.edp_sync(ring.ctx)
    b.check(s0, b.s, kind, beta, L.SEQ_MEAN, with_rest)


def test_in_one_graph_beside_other_losses(edp_lib):
    """Teacher, student and a policy loss captured together and replayed with new logits, while
    another context of the device works on its own stream."""
    edp, ring, other = edp_lib, ctx_of(edp_lib), ctx_of(edp_lib)
    b, new = (Batch(40, 9_001, 16, "bf16", "bf16", s) for s in (1, 2))
    side = Batch(40, 9_001, 16, "bf16", "bf16", 3)
    d, d2 = torch.zeros_like(b.s), torch.zeros_like(b.s)
    cfg = edp.make_distill_config(edp.EDP_DISTILL_REVERSE, edp.EDP_REDUCE_SEQ_SUM)
    x, ploss = torch.randn(40, device="cuda"), torch.zeros(8, device="cuda")
    pc = edp.make_policy_config()

    def step():
        b.teach(edp, ring)
        b.learn(edp, ring, cfg, d)
        edp.edp_policy_loss(ring.ctx, pc, x, x, x, 40, ploss, mask=b.mask)

    s, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    gc.collect()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    b.t.copy_(new.t)
    b.s.copy_(new.s)
    b.mask.copy_(new.mask)
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s):
            g.replay()
        with torch.cuda.stream(s2):
            side.teach(edp, other)
            side.learn(edp, other, cfg, d2)
    torch.cuda.synchronize()
    edp.edp_sync(ring.ctx)
    edp.edp_sync(other.ctx)
    b.check(to_np(b.s.double()), d, L.REVERSE, 0.0, L.SEQ_SUM, True)
    side.check(to_np(side.s.double()), d2, L.REVERSE, 0.0, L.SEQ_SUM, True)


def test_a_student_at_its_teacher(edp_lib):
    """The same logits on both sides: no loss and no gradient beyond the numbers' rounding."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    b = Batch(12, 5_003, 50, "f32", "f32", 5)
    b.s = b.t.clone()
    d = torch.zeros_like(b.s)
    for kind, beta in ((edp.EDP_DISTILL_FORWARD, 0.0), (edp.EDP_DISTILL_REVERSE, 0.0),
                       (edp.EDP_DISTILL_MIX, .5)):
        b.teach(edp, ring)
        b.learn(edp, ring, edp.make_distill_config(kind, edp.EDP_REDUCE_SEQ_SUM, beta), d)
        edp.edp_sync(ring.ctx)
        # each logarithm to 1e-5 + 1e-6 of it (below 20), of classes that sum to 1, on both sides
        assert b.each.abs().max() <= 2 * (1e-5 + 2e-5) and d.abs().max() <= 2 * (1e-5 + 2e-5)


def test_sampled_token_among_the_list(edp_lib):
    """What an actor reports: the given token's log-probability is its entry's, bit for bit,
    and the same that edp_token_logprob gives to a last rounding."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    b = Batch(30, 20_003, 10, "bf16", "bf16", 6)
    b.mask.fill_(1)
    b.teach(edp, ring)
    target = b.ids[:, 3].contiguous()
    lp, H, st = (torch.zeros(30, *s, device="cuda") for s in ((), (), (2,)))
    lp2, H2, st2 = (torch.zeros(30, *s, device="cuda") for s in ((), (), (2,)))
    edp.edp_token_top(ring.ctx, b.t, b.ids, b.lp, target=target, logp=lp, entropy=H, stats=st)
    edp.edp_token_logprob(ring.ctx, b.t, target, lp2, entropy=H2, stats=st2)
    edp.edp_sync(ring.ctx)
    assert torch.equal(lp, b.lp[:, 3]) and torch.equal(st[:, 0], st2[:, 0])
    for x, y in ((lp, lp2), (H, H2)):
        assert torch.all((x - y).abs() <= 2 * (1e-5 + 1e-6 * y.abs()))
    assert torch.all((st[:, 1] - st2[:, 1]).abs() <= 2e-5 * st2[:, 1])
    # its stats serve the gradient, too
    g, d = torch.ones(30, device="cuda"), torch.zeros_like(b.t)
    edp.edp_token_logprob_grad(ring.ctx, b.t, target, st, g, d)
    edp.edp_sync(ring.ctx)
    want = L.token_logprob_grad(to_np(b.t.double()), to_np(target), np.ones(30))
    assert np.all(np.abs(to_np(d.double()) - want) <= UNIT["bf16"] * np.abs(want) + 4e-5)


@pytest.mark.parametrize("reduce", [L.TOKEN_MEAN, L.SEQ_MEAN])
def test_lists_right_before_the_loss(edp_lib, reduce):
    """Teacher after teacher without a pause: each loss is of the lists written just before it
    (the loss's kernels start while the ones before them end)."""
    edp, ring = edp_lib, ctx_of(edp_lib)
    batches = [Batch(2_000, 1_001, 16, "bf16", "bf16", s) for s in range(4)]
    cfg = edp.make_distill_config(edp.EDP_DISTILL_FORWARD, reduce)
    d = [torch.zeros_like(b.s) for b in batches]
    alone = []
    for b, g in zip(batches, d):
        b.teach(edp, ring)
        torch.cuda.synchronize()
        b.learn(edp, ring, cfg, g)
        torch.cuda.synchronize()
        alone.append((b.loss.clone(), b.each.clone(), g.clone()))
        b.ids.fill_(-1)
        b.lp.fill_(float("nan"))
        g.fill_(7.0)
    torch.cuda.synchronize()
    for _ in range(20):
        for b, g in zip(batches, d):
            b.teach(edp, ring)
            b.learn(edp, ring, cfg, g)
    edp.edp_sync(ring.ctx)
    for b, g, want in zip(batches, d, alone):
        for x, y in zip((b.loss, b.each, g), want):
            assert torch.equal(x, y)
