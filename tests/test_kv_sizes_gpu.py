"""Attention over the range of sizes that the header promises.  A power of two in q and its inverse in the keys leaves the scores as they
are, one in the values comes out again: the results have to be the same bits."""
import pytest
import torch

from paper_2607_16100_b200 import symar
from test_kv_gpu import Setup, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs,hq,hkv,dim", [([(1, 300), (1, 17)], 8, 1, 128), ([(1, 300)], 10, 1, 64), ([(3, 300)], 4, 1, 256),
                                             ([(700, 700)], 16, 8, 128), ([(700, 700)], 16, 8, 64)])
def test_powers_of_two_change_nothing(seqs, hq, hkv, dim):
    c = symar.KVContext.on_torch()
    want = None
    for of_q, of_v in ((0, 0), (1, 0), (30, 0), (59, 0), (-30, 0), (-57, 0), (0, 97), (0, -100), (59, 97), (-57, -100)):
        s = Setup(seqs, hkv, dim, 16, seed=2)
        w = s.whole()
        # normal numbers of these counts are below 8 in size
        k, v = (normal(w.tokens, hkv, dim, seed=i, dtype=torch.float32) for i in (1, 2))
        c.append(s.cache, w.batch, k * 2.0 ** -of_q, v * 2.0 ** of_v)
        q = (normal(s.tokens, hq, dim, seed=5).double() * 2.0 ** of_q).bfloat16()
        got = c.attention(s.cache, s.batch, q).double() * 2.0 ** -of_v
        want = got if want is None else want
        assert torch.equal(got, want), (of_q, of_v)
    assert torch.isfinite(want).all() and c.status()[0] == symar.OK
    c.destroy()
