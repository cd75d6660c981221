"""The Python calls of the lists and of the distillation loss: arrays of one number per row are
checked for their length and order like all others, before anything is called."""
import pytest
import torch

from paper_2609_24456_gb300 import build, edp
from test_distill_arguments import K, N, V, calls


@pytest.fixture(autouse=True)
def library():
    build.build()


@pytest.mark.parametrize("call,names", [
    (edp.edp_token_top, ("logp", "entropy", "rest", "stats")),
    (edp.edp_distill_loss, ("rest", "loss", "row_loss"))], ids=lambda x: getattr(x, "__name__", ""))
def test_lengths_and_orders(call, names):
    args = calls()[call]
    assert (N, V, K) == (6, 8, 3)
    for k in names:
        x = args[k]
        strided = torch.zeros(x.shape + (2,))[..., 0] if k != "loss" else torch.zeros(0)
        for bad in (x[1:], strided):
            with pytest.raises(edp.EdpError, match=call.__name__ + ".*elements") as e:
                call(None, stream=0, **dict(args, **{k: bad}))
            assert e.value.status == edp.EDP_ERR_INVALID, k
        for good in (torch.cat([x, x]), None if k != "loss" else x, x.data_ptr()):
            with pytest.raises(edp.EdpError) as e:  # the null context, by the library itself
                call(None, stream=0, **dict(args, **{k: good}))
            assert "elements" not in str(e.value), k


def test_a_column_of_a_wider_array():
    """As a program may hold them: `rest` beside other numbers of its rows."""
    args = calls()[edp.edp_distill_loss]
    wide = torch.zeros(N, 4)
    with pytest.raises(edp.EdpError, match="strided"):
        edp.edp_distill_loss(None, stream=0, **dict(args, rest=wide[:, 0]))
    with pytest.raises(edp.EdpError) as e:
        edp.edp_distill_loss(None, stream=0, **dict(args, rest=wide[:, 0].contiguous()))
    assert "elements" not in str(e.value)
