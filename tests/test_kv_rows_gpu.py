"""Which rows of q, k and v belong to which token of which sequence: rows before token_start[0], behind token_start[seqs] (the padding of
a call of a fixed size), and a token_start that goes beyond the call's rows.  A row of no sequence: append stores nothing and copies its
q, read and attention give zeros."""
import pytest
import torch

from paper_2607_16100_b200 import symar
from test_kv_gpu import Setup, kv, normal      # noqa: F401  (kv is a fixture)
from test_prompt_gpu import reference

pytestmark = pytest.mark.gpu

# few rows, and enough for the prompt kernel
SIZES = [([(3, 40), (0, 9), (5, 30)], 4, 2, 64, 16), ([(2, 17), (1, 1)], 8, 2, 128, 32), ([(6, 300)], 4, 1, 256, 64),
         ([(300, 400), (150, 150), (0, 7)], 32, 8, 128, 16), ([(1500, 1500)], 8, 8, 64, 16)]


def moved(s, front, behind):
    """The batch of `s` with its rows from `front` on, and that many rows in all."""
    return symar.KVBatch(s.lengths, s.table, s.start + front), front + s.tokens + behind


def starts(s):
    s.start = torch.tensor([0] + [n for n, _ in s.seqs], dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    s.batch = symar.KVBatch(s.lengths, s.table, s.start)


def padded(x, front, behind, fill):
    y = torch.full((front + x.shape[0] + behind, *x.shape[1:]), fill, dtype=x.dtype, device=x.device)
    y[front:front + x.shape[0]] = x
    return y


@pytest.mark.parametrize("front,behind", [(2, 0), (0, 3), (5, 300)])
@pytest.mark.parametrize("seqs,hq,hkv,dim,page", SIZES)
def test_append_and_read_leave_rows_of_no_sequence_alone(kv, seqs, hq, hkv, dim, page, front, behind):      # noqa: F811
    s, t = (Setup(seqs, hkv, dim, page, seed=1, single=False) for _ in range(2))
    for x in (s, t):
        starts(x)
        x.fill(kv, seed=3)                       # what earlier calls have stored
    q, k, v = (normal(s.tokens, h, dim, seed=i) for i, h in enumerate((hq, hkv, hkv)))
    for rot, interleaved in ((dim, False), (6, True), (0, False)):        # queries in pairs of eights, one by one, not turned
        table = symar.rope_table(2000, rot) if rot else None
        want = kv.append(s.cache, s.batch, k, v, q=q, rotations=table, interleaved=interleaved)
        batch, rows = moved(t, front, behind)
        pq, pk, pv = (padded(x, front, behind, 3.0) for x in (q, k, v))
        got = kv.append(t.cache, batch, pk, pv, q=pq, rotations=table, interleaved=interleaved)
        assert torch.equal(t.cache.pages, s.cache.pages)
        assert torch.equal(got, padded(want, front, behind, 3.0))
        for a, b in zip(kv.read(t.cache, batch, rows), kv.read(s.cache, s.batch, s.tokens)):
            assert torch.equal(a, padded(b, front, behind, 0.0))
    assert kv.status()[0] == symar.OK


@pytest.mark.parametrize("front,behind", [(2, 0), (0, 3), (5, 300)])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("seqs,hq,hkv,dim,page", SIZES)
def test_attention_of_rows_of_no_sequence_is_zero(kv, seqs, hq, hkv, dim, page, front, behind, offset):      # noqa: F811
    s = Setup(seqs, hkv, dim, page, seed=2, single=False)
    starts(s)
    filled = s.fill(kv, seed=5)
    q = normal(s.tokens, hq, dim, seed=6)
    want, tol = reference(s, filled, q, dim ** -0.5, 0)
    batch, rows = moved(s, front, behind)
    room = torch.full((rows, hq * dim + 8 + offset), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[:, offset:offset + hq * dim].unflatten(1, (hq, dim))
    kv.attention(s.cache, batch, padded(q, front, behind, 3.0), out=out)
    assert ((out[front:front + s.tokens].double() - want).abs() <= tol).all()
    assert (out[:front] == 0).all() and (out[front + s.tokens:] == 0).all()
    assert (room[:, :offset] == 7.0).all() and (room[:, offset + hq * dim:] == 7.0).all()


def test_a_batch_of_empty_sequences_gives_zeros(kv):      # noqa: F811
    s = Setup([(0, 5), (0, 0)], 2, 128, 16, single=False)
    q = normal(9, 8, 128, seed=1)
    out = torch.full_like(q, 7.0)
    kv.attention(s.cache, s.batch, q, out=out)
    assert (out == 0).all()


@pytest.mark.parametrize("seqs,hq,hkv,dim,page", SIZES)
def test_rows_that_a_call_does_not_have(kv, seqs, hq, hkv, dim, page):      # noqa: F811
    """token_start may go beyond the call's rows: the rows that are there have the positions that token_start gives them."""
    s, t = (Setup(seqs, hkv, dim, page, seed=3, single=False) for _ in range(2))
    for x in (s, t):
        starts(x)
        x.fill(kv, seed=7)
    q, k, v = (normal(s.tokens, h, dim, seed=i) for i, h in enumerate((hq, hkv, hkv)))
    keep = max(1, s.tokens - 2)
    table = symar.rope_table(2000, dim)
    a = kv.append(s.cache, s.batch, k, v, q=q, rotations=table)
    b = kv.append(t.cache, t.batch, k[:keep], v[:keep], q=q[:keep], rotations=table)
    assert torch.equal(b, a[:keep])
    x = t.whole()
    k, v = (y.double().split([n for _, n in seqs]) for y in kv.read(t.cache, x.batch, x.tokens, dtype=torch.float32))
    want, tol = reference(t, list(zip(k, v)), a, dim ** -0.5, 0)
    assert ((kv.attention(t.cache, t.batch, b).double() - want[:keep]).abs() <= tol[:keep]).all()
