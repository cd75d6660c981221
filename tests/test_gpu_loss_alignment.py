"""Arrays off their type's alignment are refused before anything is launched."""
import pytest
import torch

from test_gpu_logprob import ctx_of

pytestmark = pytest.mark.gpu


def calls(edp):
    """(name, arguments, {argument's place: bytes to move it by})"""
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    z, x, st, loss = f(4, 8), [f(8) for _ in range(8)], f(4, 2), f(8)
    i32 = torch.zeros(32, dtype=torch.int32, device="cuda")
    off, pair = torch.tensor([0, 2, 4], device="cuda"), torch.tensor([[0, 1]], device="cuda")
    counts = torch.zeros(9, dtype=torch.int64, device="cuda")
    keep = (z, x, st, loss, i32, off, pair, counts)
    p = lambda t: t.data_ptr()  # noqa: E731
    a = [p(t) for t in x]
    pc, qc = edp.make_policy_config(), edp.make_preference_config(.1)
    logits = [p(z), edp.EDP_F32, 4, 8, 8, p(i32), None, 1.0]
    return keep, [
        ("edp_token_logprob", [*logits, a[0], a[1], p(st), None], {5: 2, 8: 2, 9: 1, 10: 2}),
        ("edp_token_logprob_grad", [*logits, p(st), a[0], a[1], a[2], p(z), 8, None],
         {5: 1, 8: 2, 9: 2, 10: 3, 11: 2}),
        ("edp_policy_loss", [pc, *a[:5], None, p(off), 2, 4, p(loss), a[5], a[6], None],
         {1: 2, 2: 2, 3: 1, 4: 2, 5: 2, 7: 4, 10: 2, 11: 2, 12: 1}),
        ("edp_policy_loss_logits", [pc, p(z), edp.EDP_F32, 4, 8, 8, p(i32), 1.0, a[0], a[1], a[2],
                                    None, p(off), 2, p(loss), a[3], a[4], p(z), 8, None],
         {6: 2, 8: 2, 9: 2, 10: 1, 12: 4, 14: 2, 15: 2, 16: 2}),
        ("edp_preference_loss", [qc, a[0], a[1], None, p(off), 2, 4, p(pair), 1, p(loss), a[2],
                                 a[3], a[4], None],
         {1: 2, 2: 2, 4: 4, 7: 4, 9: 2, 10: 1, 11: 2, 12: 2}),
        ("edp_balance_loss", [p(z), edp.EDP_F32, 4, 8, 8, p(i32), 2, None, .1, 1.0, p(loss),
                              p(counts), a[0], p(z), 8, None], {5: 2, 10: 2, 11: 4, 12: 2}),
    ]


def test_refused_and_then_taken(edp_lib):
    edp, ring = edp_lib, ctx_of(edp_lib)
    keep, todo = calls(edp)
    for name, args, moved in todo:
        fn = getattr(edp.lib(), name)
        for i, by in moved.items():
            bad = list(args)
            bad[i] += by
            assert fn(ring.ctx, *bad) == edp.EDP_ERR_INVALID, (name, i)
            assert b"aligned" in edp.lib().edp_last_error(ring.ctx), (name, i)
        assert fn(ring.ctx, *args) == edp.EDP_OK, name
        edp.edp_sync(ring.ctx)
