"""How much of a probability enters the second product where rows are few: sixteen bits, in two parts of eight.

Bound.  x = probability times its group's scale.  Its upper eight bits enter as they are; what they leave, below 2^-7 of x, is rounded to eight
bits (2^-8 of it): 2^-15 of x in all.  Beside that: the scale is used with the zero point's bits in it (15 of 2^-23 at most, below 2^-19); scores
are off by e (the sums of the first product truncate, D additions of 2^-23, and as much again for scaling and 2^x), the sums over n tokens
truncate (2^-23 each), and the result is rounded to bf16 once (2^-8).  The scale of the scores is 2^-10 here, so that e is small beside
2^-15, and values have both signs, so that many results are small beside their terms: there the parts show."""
import numpy as np
import pytest
import torch

from paper_2607_16100_b200 import symar
from test_kv_gpu import Setup, normal

SCALE = 2.0 ** -10


def bound(terms, out, e, n):
    """terms: sum of p |v|."""
    return terms * (2.0 ** -15 + 2.0 ** -19 + 2.5 * e + n * 2.0 ** -23) * 1.01 + 2.0 ** -8 * np.abs(out) + 1e-37


def upper(x):
    return (x.astype(np.float32).view(np.uint32) & 0xffff0000).view(np.float32)


def rounded(x):
    b = x.astype(np.float32).view(np.uint32)
    return ((b + 0x7fff + (b >> 16 & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


PARTS = {"two parts": lambda x: upper(x).astype(np.float64) + rounded(x - upper(x)), "the upper bits alone": upper, "one part, rounded": rounded}


@pytest.mark.parametrize("n", [17, 130, 700])
@pytest.mark.parametrize("how", PARTS)
def test_the_bound_tells_two_parts_from_one(how, n):
    """The product in numpy, on values of the kind that the GPU test takes."""
    rng = np.random.default_rng(n)
    dim, rows = 64, 8
    lo, hi = -rng.uniform(1.5, 3.5, n), rng.uniform(1.5, 3.5, n)
    s = ((hi - lo) / 15).astype(np.float32)
    z = np.rint(-lo / s)
    codes = rng.integers(0, 16, (n, dim)) - z[:, None]
    p = np.exp(SCALE * 8 * rng.standard_normal((rows, n)))
    p /= p.sum(1, keepdims=True)
    want = p @ (codes * s[:, None].astype(np.float64))
    x = (p.astype(np.float32) * s).astype(np.float32)
    got = rounded(PARTS[how](x).astype(np.float64) @ codes).astype(np.float64)
    tol = bound(p @ np.abs(codes * s[:, None]), want, 0.0, n)
    beyond = (np.abs(got - want) > tol).sum()
    assert beyond == 0 if how == "two parts" else beyond > 0            # (one element beyond its bound fails the test below)


@pytest.mark.gpu
@pytest.mark.parametrize("seqs,hq,hkv,dim,page", [
    ([(1, 17), (1, 130), (1, 700)], 8, 1, 128, 16), ([(1, 17), (1, 130), (1, 700)], 10, 1, 128, 64), ([(1, 300), (1, 16)], 16, 8, 64, 32),
    ([(1, 90)], 32, 2, 64, 16), ([(1, 200), (1, 33)], 4, 1, 256, 32), ([(1, 200)], 16, 1, 256, 16), ([(5, 70), (1, 257)], 8, 2, 128, 32),
    ([(1, 9000)], 8, 1, 128, 64),
])
def test_few_rows(seqs, hq, hkv, dim, page):
    c = symar.KVContext.on_torch()
    s = Setup(seqs, hkv, dim, page, seed=2)
    filled = s.fill(c, seed=11)
    q = normal(s.tokens, hq, dim, seed=5)
    got = c.attention(s.cache, s.batch, q, scale=SCALE).double().cpu().numpy()
    share = hq // hkv
    for row, (b, pos) in enumerate(s.place):
        k, v = (t[:pos + 1] for t in filled[b])
        for h in range(hq):
            kk, vv, qq = k[:, h // share], v[:, h // share], q[row, h].double()
            p = torch.softmax(kk @ qq * SCALE, 0)
            e = 2 * dim * 2.0 ** -23 * SCALE * (kk.abs() @ qq.abs()).max().item() + 1e-6
            want = (p @ vv).cpu().numpy()
            tol = bound((p @ vv.abs()).cpu().numpy(), want, e, pos + 1)
            err = np.abs(got[row, h] - want)
            assert (err <= tol).all(), (row, h, (err / tol).max())
    c.destroy()
