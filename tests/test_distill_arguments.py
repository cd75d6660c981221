"""The Python calls of the lists and of the distillation loss take arrays of the types and
sizes that the library reads, and refuse others before anything is called; the
configuration's layout is the header's."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2609_24456_gb300 import build, edp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
N, V, K = 6, 8, 3


@pytest.fixture(autouse=True)
def library():
    build.build()


def calls():
    f = lambda *s: torch.zeros(s)  # noqa: E731
    ids = torch.zeros(N, K, dtype=torch.int32)
    mask, off = torch.ones(N, dtype=torch.uint8), torch.tensor([0, 2, N])
    return {
        edp.edp_token_top: dict(logits=f(N, V), ids=ids, top_logp=f(N, K), logp=f(N), rest=f(N),
                                target=torch.zeros(N, dtype=torch.int32), mask=mask,
                                entropy=f(N), stats=f(N, 2)),
        edp.edp_distill_loss: dict(cfg=edp.make_distill_config(), logits=f(N, V), ids=ids,
                                   value=f(N, K), loss=f(1), rest=f(N), mask=mask, off=off,
                                   n_seq=2, row_loss=f(N), dlogits=f(N, V)),
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
            if x.dtype == t:
                continue
            with pytest.raises(TypeError, match=call.__name__):
                call(None, stream=0, **dict(args, **{k: x.to(t)}))
        if k not in ("ids", "value", "top_logp", "target", "mask", "off"):
            continue
        short = x[1:] if k != "ids" else x.t().contiguous().t()
        for bad in (short, torch.cat([x, x], -1)[..., ::2] if x.dim() == 1 else x.t().reshape(
                K, N).t()):
            if bad.is_contiguous() and bad.numel() == x.numel():
                continue
            with pytest.raises(edp.EdpError, match=call.__name__ + ".*elements") as e:
                call(None, stream=0, **dict(args, **{k: bad}))
            assert e.value.status == edp.EDP_ERR_INVALID
    for bad in (args["ids"][1:], args["ids"][0], args["ids"].reshape(-1)):
        with pytest.raises(ValueError, match=call.__name__):
            call(None, stream=0, **dict(args, ids=bad))
    with pytest.raises(ValueError):
        call(None, stream=0, **dict(args, logits=torch.zeros(V, N).t()))
    if "dlogits" in args:
        for bad in (torch.zeros(N, V + 1), torch.zeros(N, V, dtype=torch.bfloat16)):
            with pytest.raises(ValueError, match="dlogits"):
                call(None, stream=0, **dict(args, dlogits=bad))


def test_configuration(tmp_path):
    c = edp.make_distill_config(edp.EDP_DISTILL_MIX, edp.EDP_REDUCE_SEQ_SUM, .25, 1.0, 3.0, 8.0)
    assert (c.kind, c.reduce, c.beta, c.teacher_temperature, c.norm, c.grad_scale) == \
        (2, 2, .25, 1.0, 3.0, 8.0)
    cls, name = edp.edp_distill_config, "edp_distill_config"
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"edp.h\"\n"
                   "int main(void) { printf(\"%%zu\\n\", sizeof(%s));\n" % name +
                   "".join("printf(\"%%zu\\n\", offsetof(%s, %s));\n" % (name, f)
                           for f, _ in cls._fields_) +
                   "printf(\"%d %d %d\\n\", EDP_DISTILL_FORWARD, EDP_DISTILL_REVERSE, "
                   "EDP_DISTILL_MIX); return 0; }")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    want = [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_] + [
        edp.EDP_DISTILL_FORWARD, edp.EDP_DISTILL_REVERSE, edp.EDP_DISTILL_MIX]
    assert [int(x) for x in got] == want
