"""symar_norm of more than sixteen rows a multiprocessor (of 148) that are at most 512 channels long, 1024 on no boundary: several rows a block, against the formula
in 64 bits.  Bounds: test_norm_gpu.py's (a thread adds up at most 32 elements here too)."""
import pytest
import torch

from paper_2607_16100_b200 import symar
from test_norm_gpu import BF16, F32, check, normal

pytestmark = pytest.mark.gpu
MANY = 16 * 148 + 1


@pytest.mark.parametrize("n", [1, 7, 8, 24, 56, 64, 72, 120, 128, 129, 136, 250, 256, 264, 300, 504, 512, 513, 520, 777, 1000, 1023, 1024])
@pytest.mark.parametrize("rows", [MANY, MANY + 7, 5003, 40001])
def test_sizes(n, rows):
    x, res, w, w2 = normal(rows, n, seed=n), normal(rows, n, seed=1, scale=3), normal(n, seed=2), normal(n, seed=3, dtype=F32)
    check(x, res, before=("rms", w, None, 1e-6, 0))
    check(x, res, after=("rms", w2, None, 1e-5, 1), before=("layer", w, normal(n, seed=4), 1e-5, 0), scale=0.5, residual_scale=1.25)


@pytest.mark.parametrize("xt", [BF16, F32])
@pytest.mark.parametrize("st", [BF16, F32])
@pytest.mark.parametrize("gate", [None, "channel", "row", "all", "one"])
@pytest.mark.parametrize("m,n", [(MANY, 64), (2900, 40), (3111, 128), (2501, 256), (2700, 248), (2403, 512), (2600, 130), (2400, 999)])
def test_types_gates_and_kinds(xt, st, gate, m, n):
    x, res = normal(m, n, seed=1, dtype=xt), normal(m, n, seed=2, dtype=st)
    g = {None: None, "channel": (n,), "row": (m, 1), "all": (m, n), "one": ()}[gate]
    g = normal(*g, seed=3, dtype=xt) if g is not None else None
    w, b = normal(n, seed=4, dtype=st), normal(n, seed=5, dtype=st)
    for act in ("none", "sigmoid", "tanh"):
        for after, before in ((None, "rms"), ("rms", None), ("layer", "rms"), ("rms", "layer"), (None, None)):
            check(x, res, after and (after, w, b, 1e-5, 0), before and (before, w, None, 1e-5, 1), g, act, 0.7, -1.5)
            check(x, None, after and (after, None, b, 1e-5, 0), before and (before, None, None, 1e-5, 0), g, act)


@pytest.mark.parametrize("n", [64, 128, 200, 512, 130, 1000])
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_heads_of_wider_rows(n, offset):
    """The first heads of a fused projection's result, also transposed; nothing beside the results is written."""
    for dtype in (BF16, F32):
        room = normal(700, 6, n + 16, seed=n, dtype=dtype)
        x = room[:, :4, offset:offset + n]
        out, old = torch.full_like(room, 7.0), torch.full_like(room, 7.0)
        w = normal(n, seed=2, dtype=dtype)
        check(x, None, before=("rms", w, None, 1e-6, 0), out=out[:, 1:5, offset:offset + n])
        res = room[:, 2:, offset:offset + n]
        check(x.transpose(0, 1), res.transpose(0, 1), after=("layer", w, None, 1e-6, 0), before=("rms", None, w, 1e-6, 0), gate=normal(4, 1, 1, seed=6, dtype=dtype),
              out=out[:, 1:5, offset:offset + n].transpose(0, 1), residual_out=old[:, 1:5, offset:offset + n].transpose(0, 1))
        for o in (out, old):
            assert (o[:, (0, 5)] == 7).all() and (o[..., :offset] == 7).all() and (o[..., offset + n:] == 7).all()


def test_results_may_be_the_operands():
    for m, n in ((MANY, 128), (9001, 64), (2500, 512), (2500, 130), (2400, 1000)):
        x, res, w = normal(m, n, seed=1), normal(m, n, seed=2, dtype=F32), normal(n, seed=3)
        y, r = symar.norm(x, res, before=symar.Norm("rms", w))
        a, b = x.clone(), res.clone()
        symar.norm(a, b, before=symar.Norm("rms", w), out=a, residual_out=b)
        assert torch.equal(a, y) and torch.equal(b, r)
