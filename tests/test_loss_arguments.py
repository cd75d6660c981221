"""The losses' Python calls take arrays of the types that the library reads, and
refuse others before anything is called: an int64 target would be read as pairs
of int32, an int32 offset beyond its end.  Targets, choices, masks, offsets, pairs
and counts have to be long enough and in order as well."""
import pytest
import torch

from paper_2609_24456_gb300 import build, edp

N, V = 6, 8


@pytest.fixture(autouse=True)
def library():
    build.build()


def calls():
    f = lambda *s: torch.zeros(s)  # noqa: E731
    target, mask = torch.zeros(N, dtype=torch.int32), torch.ones(N, dtype=torch.uint8)
    off, pair = torch.tensor([0, 2, N]), torch.tensor([[0, 1]])
    rows = dict(target=target, mask=mask, entropy=f(N))
    tokens = dict(logp=f(N), ref_logp=f(N), mask=mask, off=off, dlogp=f(N))
    pc, qc = edp.make_policy_config(), edp.make_preference_config(.1)
    return {
        edp.edp_token_logprob: dict(logits=f(N, V), logp=f(N), stats=f(N, 2), **rows),
        edp.edp_token_logprob_grad: dict(logits=f(N, V), dlogits=f(N, V), stats=f(N, 2),
                                         dlogp=f(N), dentropy=f(N), **rows),
        edp.edp_policy_loss: dict(cfg=pc, old_logp=f(N), adv=f(N), n_tokens=N, n_seq=2, loss=f(8),
                                  entropy=f(N), dentropy=f(N), **tokens),
        edp.edp_policy_loss_logits: dict(cfg=pc, logits=f(N, V), dlogits=f(N, V), old_logp=f(N),
                                         adv=f(N), ref_logp=f(N), logp=f(N), loss=f(8), off=off,
                                         n_seq=2, **rows),
        edp.edp_preference_loss: dict(cfg=qc, n_tokens=N, n_seq=2, pair=pair, n_pair=1, loss=f(4),
                                      seq_ratio=f(2), pair_loss=f(1), **tokens),
        edp.edp_balance_loss: dict(logits=f(N, V), sel=torch.zeros(N, 2, dtype=torch.int32),
                                   coef=1.0, loss=f(1), prob=f(V), mask=mask,
                                   counts=torch.zeros(V, dtype=torch.int64)),
    }


def arrays(args):
    return [k for k, v in args.items() if isinstance(v, torch.Tensor) and "logits" not in k]


@pytest.mark.parametrize("call", list(calls()), ids=lambda f: f.__name__)
def test_types_and_sizes(call):
    """The library itself refuses the null context, with its own status."""
    args = calls()[call]
    with pytest.raises(edp.EdpError) as e:
        call(None, stream=0, **args)
    assert "elements" not in str(e.value)
    for k in arrays(args):
        x = args[k]
        for t in (torch.float64, torch.int64, torch.int32, torch.bfloat16, torch.int16):
            if x.dtype == t or x.dtype == torch.uint8 and t == torch.bool:
                continue
            with pytest.raises(TypeError, match=call.__name__):
                call(None, stream=0, **dict(args, **{k: x.to(t)}))
        if x.dtype == torch.float32:
            continue
        for bad in (x.reshape(-1)[1:], torch.cat([x.reshape(-1)] * 2)[::2]):
            if k == "sel" or bad.is_contiguous() and bad.numel() == x.numel():
                continue
            with pytest.raises(edp.EdpError, match=call.__name__ + ".*elements") as e:
                call(None, stream=0, **dict(args, **{k: bad}))
            assert e.value.status == edp.EDP_ERR_INVALID
    if "sel" in args:
        with pytest.raises(edp.EdpError, match="elements"):
            call(None, stream=0, **dict(args, sel=args["sel"][1:]))
        with pytest.raises(ValueError):
            call(None, stream=0, **dict(args, sel=args["sel"].t()))


@pytest.mark.parametrize("call", list(calls()), ids=lambda f: f.__name__)
def test_other_types_with_the_same_bytes(call):
    """bool and int8 masks, unsigned offsets, plain addresses, no array."""
    args = calls()[call]
    same = dict(mask=[torch.bool, torch.int8], off=[torch.uint64])
    for k in arrays(args):
        for x in [args[k].to(t) for t in same.get(k, [])] + (
                [args[k].data_ptr(), None] if k != "sel" else []):
            with pytest.raises(edp.EdpError) as e:
                call(None, stream=0, **dict(args, **{k: x}))
            assert "elements" not in str(e.value)
