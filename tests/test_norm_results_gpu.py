"""symar.norm with one tensor for both results: refused, and nothing of it written."""
import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu


def test_one_tensor_for_both_results():
    x, res = (torch.randn(6, 64, device="cuda").bfloat16() for _ in range(2))
    norm = symar.Norm("rms")
    for one in (x, res, torch.zeros_like(x)):
        kept = one.clone()
        with pytest.raises(symar.SymarError):
            symar.norm(x, res, before=norm, out=one, residual_out=one)
        assert torch.equal(one, kept)
    want = symar.norm(x, res, before=norm)
    a, b = x.clone(), res.clone()
    symar.norm(a, b, before=norm, out=b, residual_out=a)            # each in the other's place
    assert torch.equal(b, want[0]) and torch.equal(a, want[1])
