"""A context's first call on a stream that does not wait for the default one:
its sums start at 0 whatever its memory held, and whatever the default stream
still has to do."""
import numpy as np
import pytest
import torch

from gpu_util import cuda, to_np
from oracle import losses as L

pytestmark = pytest.mark.gpu


class Memory:
    """An allocator whose blocks are full of ones, and which leaves the default
    stream busy."""

    def __init__(self, edp):
        self.live, self.work = {}, torch.randn(4096, 4096, device="cuda")
        self.alloc = edp.ALLOC_FN(self._alloc)
        self.free = edp.FREE_FN(self._free)

    def _alloc(self, user, nbytes):
        t = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for _ in range(40):
            torch.mm(self.work, self.work)
        self.live[t.data_ptr()] = t
        return t.data_ptr()

    def _free(self, user, p):
        self.live.pop(p, None)

    def ring(self, edp, rows=64):
        cfg = edp.make_config(rows, (3, 16, 16), edp.EDP_XFORM_HWC_CHW_BF16)
        cfg.alloc, cfg.free = self.alloc, self.free
        return edp.Ring(cfg, action=False, reward=False, done=False)


@pytest.mark.parametrize("rows,E", [(50, 16), (5000, 64)])
def test_balance_loss(edp_lib, rows, E):
    edp, memory = edp_lib, Memory(edp_lib)
    ring = memory.ring(edp)
    rng = np.random.default_rng(rows)
    z = torch.randn(rows, E, device="cuda")
    sel = rng.integers(0, E, (rows, 2)).astype(np.int32)
    d_sel = cuda(sel)
    want, counts, prob, _ = L.balance(to_np(z.double()), sel, np.ones(rows), 1.0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):  # and what the first call leaves behind
        loss, p = torch.zeros(1, device="cuda"), torch.zeros(E, device="cuda")
        n = torch.zeros(E, dtype=torch.int64, device="cuda")
        torch.cuda.synchronize()
        edp.edp_balance_loss(ring.ctx, z, d_sel, 1.0, loss, n, prob=p, stream=side)
        side.synchronize()
        torch.cuda.synchronize()
        assert np.array_equal(to_np(n), counts)
        assert np.all(np.abs(to_np(p) - prob) <= 1e-5 * prob)
        assert abs(float(loss) - want) <= 1e-5 * want
    ring.close()
    assert not memory.live


def test_shuffle(edp_lib, orc):
    edp, memory = edp_lib, Memory(edp_lib)
    n = 20_000
    ring = memory.ring(edp, n)
    obs = torch.zeros((n, 768), dtype=torch.uint8, device="cuda")
    edp.edp_ingest(ring.ctx, obs, n)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for round_ in range(2):
        idx = torch.full((n,), -1, dtype=torch.int64, device="cuda")
        torch.cuda.synchronize()
        edp.edp_sample(ring.ctx, edp.EDP_SAMPLE_PERMUTE, n, 5, round_, idx, stream=side)
        edp.edp_sync(ring.ctx, side)
        assert np.array_equal(to_np(idx), orc.permutation(n, 5, round_))
    ring.close()
    assert not memory.live
