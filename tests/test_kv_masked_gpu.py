"""What a row must not see does not reach it: tokens of the same sequence after it, and tokens before its window, whatever is stored
for them.  And windows of any size."""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar
from test_kv_gpu import Setup, kv, normal      # noqa: F401  (kv is a fixture)

pytestmark = pytest.mark.gpu

CASES = [
    # seqs (new, total), q_heads, kv_heads, dim, page, window, sequence and position of the odd token
    ([(9, 40), (1, 30)], 8, 2, 128, 16, 0, 0, 35),           # few rows: one of the new tokens
    ([(9, 40), (1, 30)], 8, 2, 128, 16, 5, 0, 28),           # before some rows' window, inside others'
    ([(1, 70)], 8, 2, 64, 16, 20, 0, 49),                    # just outside one row's window, in a chunk that it reads
    ([(1, 70)], 8, 2, 64, 16, 20, 0, 50),                    # just inside
    ([(40, 90)], 5, 1, 256, 32, 0, 0, 60),
    ([(33, 33)], 32, 2, 128, 64, 7, 0, 20),
    ([(300, 700), (150, 150)], 32, 8, 128, 16, 0, 0, 555),   # many rows
    ([(300, 700), (150, 150)], 32, 8, 128, 16, 64, 0, 640),
    ([(1500, 1500)], 8, 8, 64, 16, 100, 0, 777),
    ([(700, 700)], 16, 8, 128, 64, 0, 0, 699),               # the last token: all other rows are before it
    ([(700, 700)], 16, 8, 128, 64, 1, 0, 300),               # seen by itself alone
]


@pytest.mark.parametrize("odd", [math.nan, math.inf])
@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("seqs,hq,hkv,dim,page,window,b,pos", CASES)
def test_hidden_tokens_may_hold_anything(kv, seqs, hq, hkv, dim, page, window, b, pos, side, odd):      # noqa: F811
    s = Setup(seqs, hkv, dim, page, seed=2, single=False)
    s.fill(kv, seed=11)
    q = normal(s.tokens, hq, dim, seed=5)
    clean = kv.attention(s.cache, s.batch, q, window=window)
    # the last channel of head 0 of one token: its group of 64 channels reads back as NaN
    k, v = kv.read(s.cache, s.whole().batch, s.whole().tokens, dtype=torch.float32)
    row = sum(t for _, t in seqs[:b]) + pos
    kk, vv = k[row:row + 1].clone(), v[row:row + 1].clone()
    (kk if side == "k" else vv)[0, 0, -1] = odd
    one = symar.KVBatch(torch.tensor([pos + 1], dtype=torch.int32, device="cuda"), s.table[b:b + 1].contiguous())
    kv.append(s.cache, one, kk, vv)
    got = kv.attention(s.cache, s.batch, q, window=window)
    share = hq // hkv
    sees = torch.tensor([c == b and pos <= p and (not window or pos > p - window) for c, p in s.place], device="cuda")
    assert sees.any() or window == 20
    # (what the token's own other group holds was stored anew from its read-back values: the same but for rounding)
    other = torch.isfinite(clean)
    hit = torch.zeros_like(other)
    hit[:, :share, slice(None) if side == "k" else slice(dim - 64, dim)] = True
    hit &= sees[:, None, None]
    assert torch.isnan(got[hit]).all()
    assert torch.isfinite(got[~hit]).all()
    assert torch.equal(got[~sees], clean[~sees])


@pytest.mark.parametrize("seqs,hq,hkv,dim,page", [([(9, 3), (1, 30)], 8, 2, 128, 16), ([(20, 9)], 1, 1, 128, 16), ([(40, 20)], 5, 1, 256, 32),
                                                   ([(900, 400), (300, 1)], 16, 8, 128, 16), ([(1500, 700)], 8, 8, 64, 16)])
def test_a_window_of_any_size(kv, seqs, hq, hkv, dim, page):      # noqa: F811
    """More new tokens than tokens, so that positions are negative; a window no smaller than the sequence hides nothing."""
    s = Setup(seqs, hkv, dim, page, seed=4, single=False)
    s.fill(kv, seed=13)
    q = normal(s.tokens, hq, dim, seed=6)
    want = kv.attention(s.cache, s.batch, q)
    for window in (max(t for _, t in seqs), 100000, 2 ** 31 - 1):
        assert torch.equal(kv.attention(s.cache, s.batch, q, window=window), want), window
