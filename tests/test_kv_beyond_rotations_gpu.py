"""A token whose position lies beyond the table of rotations cannot be turned: its entry is stored as NaN, so that whoever attends to it
sees it (and not what the page held before), and the context's status says where it was."""
import pytest
import torch

from paper_2607_16100_b200 import symar
from test_kv_gpu import DT, Setup, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (6, True), (20, False)])
def test_a_token_beyond_the_table(dtype, rot, interleaved):
    c = symar.KVContext.on_torch()
    s = Setup([(4, 40), (1, 20)], 2, 64, 16, seed=1)
    s.fill(c, seed=3)                                    # another request's tokens
    q, k, v = (normal(s.tokens, h, 64, seed=i, dtype=DT[dtype]) for i, h in enumerate((4, 2, 2)))
    qo = c.append(s.cache, s.batch, k, v, q=q, rotations=symar.rope_table(38, rot), interleaved=interleaved)
    code, seq, position = c.status()
    assert code == symar.ERR_INVAL and seq == 0 and position in (38, 39)
    c.reset()
    rk, rv = c.read(s.cache, s.batch, s.tokens, dtype=torch.float32)
    there = torch.tensor([p < 38 for _, p in s.place], device="cuda")
    assert torch.isfinite(rk[there]).all() and torch.isfinite(rv[there]).all()
    assert torch.isnan(rk[~there]).all() and torch.isnan(rv[~there]).all()
    assert torch.equal(qo[~there], q[~there])            # its query goes along as it is
    out = c.attention(s.cache, s.batch, qo.bfloat16())
    assert torch.isfinite(out[there]).all() and torch.isnan(out[~there]).all()
    assert c.status()[0] == symar.OK
    c.destroy()
