"""symar_norm at the library's boundary with weights beside a norm that is none: they change nothing."""
import ctypes

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n", [(5, 512), (700, 1024), (3000, 128), (40, 130), (3000, 130)])
@pytest.mark.parametrize("none", ["after", "before"])
def test_weights_of_a_norm_that_is_none(m, n, none):
    g = torch.Generator("cuda").manual_seed(n)
    x, res = (torch.randn(m, n, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(n, generator=g, device="cuda").bfloat16()
    wrong = torch.full((n,), float("nan"), device="cuda")
    norm = symar.Norm("rms", w, eps=1e-5)
    want = symar.norm(x, res, **{"after" if none == "before" else "before": norm})
    out, old = torch.empty_like(x), torch.empty_like(x)
    sides = {"after": symar.NormSide(weight=w.data_ptr(), eps=1e-5, kind=1, dtype=symar.BF16), "before": symar.NormSide(weight=w.data_ptr(), eps=1e-5, kind=1, dtype=symar.BF16)}
    sides[none] = symar.NormSide(weight=wrong.data_ptr(), bias=wrong.data_ptr(), eps=1e-5, kind=0, dtype=symar.F32, plus_one=1)
    a = symar.NormArgs(x=x.data_ptr(), x_ld=n, residual=res.data_ptr(), residual_ld=n, residual_out=old.data_ptr(), residual_out_ld=n,
                       out=None if none == "before" else out.data_ptr(), out_ld=n, scale=1.0, residual_scale=1.0, groups=1, m=m, n=n, dtype=symar.BF16,
                       stream_dtype=symar.BF16, **sides)
    assert symar.load().symar_norm(ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == symar.OK
    torch.cuda.synchronize()
    assert torch.equal(old, want[1]) and (none == "before" or torch.equal(out, want[0]))
