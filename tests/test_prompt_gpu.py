"""Attention of many query rows at a time (prompts and pieces of them) over the 4-bit cache, against 64 bits.  The setting, the poisoned
pages and the bound are those of test_kv_gpu.py; here sequences have hundreds of rows, so the reference works on whole heads."""
import pytest
import torch

from paper_2607_16100_b200 import symar
from test_kv_gpu import Setup, kv, normal      # noqa: F401  (kv is a fixture)

pytestmark = pytest.mark.gpu


def reference(s, filled, q, scale, window):
    share = q.shape[1] // s.heads
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    first = 0
    for (new, total), (k, v) in zip(s.seqs, filled):
        rows = slice(first, first + new)
        first += new
        if not new or not total:
            continue
        at = torch.arange(total - new, total, device="cuda")[:, None]
        token = torch.arange(total, device="cuda")[None]
        hidden = (token > at) | (token <= at - (window or total))
        for h in range(q.shape[1]):
            kk, vv, qq = k[:, h // share], v[:, h // share], q[rows, h].double()
            logits = (qq @ kk.T * scale).masked_fill(hidden, -torch.inf)
            p = torch.nan_to_num(torch.softmax(logits, -1))                  # rows that see nothing: zeros
            big = (qq.abs() @ kk.abs().T * scale).masked_fill(hidden, 0.0).amax(-1, keepdim=True)
            e = 2 * q.shape[2] * 2.0 ** -23 * big + 1e-6
            out[rows, h] = p @ vv
            tol[rows, h] = (p @ vv.abs()) * (2.5 * e + 2.0 ** -8 + total * 2.0 ** -23) + 2.0 ** -8 * out[rows, h].abs()
    return out, tol * 1.01 + 1e-37


CASES = [
    # seqs (new, total), q_heads, kv_heads, dim, page, window
    ([(700, 700)], 16, 8, 128, 64, 0),                       # two heads to a share: 64 tokens a block
    ([(300, 700), (150, 150)], 32, 8, 128, 16, 0),
    ([(257, 1000), (1, 77), (0, 5), (400, 401)], 40, 8, 128, 32, 0),     # shares of five; one row, none, and blocks that end in rows of padding
    ([(1500, 1500)], 8, 8, 64, 16, 0),
    ([(600, 2111), (333, 333)], 8, 8, 64, 128, 100),         # a window shorter than a block's tokens
    ([(512, 3000)], 24, 8, 128, 256, 1000),
    ([(2000, 2000)], 8, 8, 128, 64, 1),
    ([(900, 400), (300, 1)], 16, 8, 128, 16, 0),             # more new tokens than tokens: the first rows see nothing
    ([(1200, 2111), (700, 700)], 8, 8, 64, 128, 100),        # a window shorter than a block's tokens, and many blocks
    ([(16, 16 + 37 * i) for i in range(12)], 64, 8, 128, 16, 0),         # blocks that are half full, of unequal lengths
    ([(40, 333), (1, 900), (150, 150), (64, 2000)], 64, 8, 128, 32, 77), # the same beside one token, under a window
]


@pytest.mark.parametrize("seqs,hq,hkv,dim,page,window", CASES)
def test_prompts(kv, seqs, hq, hkv, dim, page, window):      # noqa: F811
    s = Setup(seqs, hkv, dim, page, seed=2)
    filled = s.fill(kv, seed=11)
    q = normal(s.tokens, hq, dim, seed=5)
    got = kv.attention(s.cache, s.batch, q, window=window)
    want, tol = reference(s, filled, q, dim ** -0.5, window)
    assert torch.isfinite(got).all()
    err = (got.double() - want).abs()
    assert (err <= tol).all(), (err / tol).max().item()
    for row, (_, pos) in enumerate(s.place):
        if pos < 0:
            assert (got[row] == 0).all()
    for _ in range(3):
        assert torch.equal(got, kv.attention(s.cache, s.batch, q, window=window))
    assert kv.status()[0] == symar.OK


@pytest.mark.parametrize("scale", [0.03, 5.0])
def test_prompts_with_flat_and_sharp_softmax(kv, scale):     # noqa: F811
    """Scores that rise along the tokens, so that the running maximum moves again and again."""
    s = Setup([(640, 900)], 8, 128, 32, seed=3)
    w = s.whole()
    ramp = torch.linspace(0.1, 4.0, w.tokens, device="cuda")[:, None, None]
    k, v = (normal(w.tokens, 8, 128, seed=i, dtype=torch.float32) for i in (1, 2))
    kv.append(s.cache, w.batch, k.abs() * ramp, v)
    k, v = kv.read(s.cache, w.batch, w.tokens, dtype=torch.float32)
    q = normal(s.tokens, 16, 128, seed=6).abs()
    got = kv.attention(s.cache, s.batch, q, scale=scale)
    want, tol = reference(s, [(k.double(), v.double())], q, scale, 0)
    assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("new", [600, 1300])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_prompts_take_any_strides(kv, offset, new):          # noqa: F811
    s = Setup([(new, new + 100)], 8, 128, 16, seed=5)
    s.fill(kv, seed=51)
    q = normal(s.tokens, 16, 128, seed=6)
    want = kv.attention(s.cache, s.batch, q)
    room = torch.zeros(s.tokens, 16 * 128 + 8 + offset, device="cuda", dtype=torch.bfloat16)
    qs = room[:, offset:offset + 2048].unflatten(1, (16, 128))
    qs.copy_(q)
    o = torch.full((16, s.tokens, 136 + offset), 7.0, device="cuda", dtype=torch.bfloat16)
    out = o[:, :, offset:offset + 128].transpose(0, 1)
    kv.attention(s.cache, s.batch, qs, out=out)
    assert torch.equal(out, want)
    assert (o[:, :, :offset] == 7.0).all() and (o[:, :, offset + 128:] == 7.0).all()


@pytest.mark.parametrize("total", [600, 1300])
def test_prompt_and_single_tokens_agree(kv, total):          # noqa: F811
    """The same rows by the two kernels: within twice the bound of the same value."""
    s = Setup([(total, total)], 8, 128, 16, seed=6)
    filled = s.fill(kv, seed=61)
    q = normal(total, 16, 128, seed=7)
    whole = kv.attention(s.cache, s.batch, q).double()
    _, tol = reference(s, filled, q, 128 ** -0.5, 0)
    for t in (0, 1, 63, 64, 65, 300, total - 1):
        batch = symar.KVBatch(torch.tensor([t + 1], dtype=torch.int32, device="cuda"), s.table)
        one = kv.attention(s.cache, batch, q[t:t + 1]).double()
        assert ((whole[t] - one[0]).abs() <= 2 * tol[t]).all()


@pytest.mark.parametrize("total", [600, 1300])
def test_a_page_that_is_not_there(kv, total):                # noqa: F811
    c = symar.KVContext.on_torch()
    s = Setup([(total, total)], 8, 128, 16, seed=7)
    filled = s.fill(kv, seed=71)
    q = normal(total, 16, 128, seed=1)
    table = s.table.clone()
    table[0, 3] = -1
    got = c.attention(s.cache, symar.KVBatch(s.lengths, table, s.start), q)
    code, seq, position = c.status()
    assert code == symar.ERR_INVAL and seq == 0 and position == 48
    # its tokens are not seen: rows before them are as ever, rows after them are the softmax over the others
    want, tol = reference(s, filled, q, 128 ** -0.5, 0)
    assert ((got[:48].double() - want[:48]).abs() <= tol[:48]).all()
    k, v = filled[0]
    keep = torch.cat([torch.arange(48), torch.arange(64, total)]).cuda()
    for t in (64, 100, total - 1):
        kk, vv = (x[keep[keep <= t]] for x in (k, v))
        for h in (0, 7, 15):
            p = torch.softmax(kk[:, h // 2] @ q[t, h].double() * 128 ** -0.5, 0)
            assert ((got[t, h].double() - p @ vv[:, h // 2]).abs() <= 2 * tol[t, h] + 2.0 ** -8 * (p @ vv[:, h // 2].abs())).all()
    c.destroy()
