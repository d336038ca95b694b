"""symar_experts where the first expert's rows begin behind row 0: what stands before them is nobody's, as what stands behind the last expert's."""
import pytest
import torch

from paper_2607_16100_b200 import symar
from test_experts_gpu import BF16, F32, whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts,n", [([3, 0, 2], 40), ([50, 60, 0], 40), ([900, 700], 4000)])
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("first", [1, 37])
def test_rows_before_the_first_expert(counts, n, out, by_row, first):
    used = sum(counts)
    rows, tokens, k = first + used + 2, 64, 72
    g = torch.Generator().manual_seed(used)
    row_token = torch.full((rows,), -1)
    row_token[first:first + used] = torch.randint(0, tokens, (used,), generator=g)
    start = torch.tensor([0, *counts]).cumsum(0) + first
    one = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    r = symar.Routes(one, one.float(), start.to(torch.int32).cuda(), row_token.to(torch.int32).cuda(), one)
    r.tokens = tokens
    x, w = whole(rows if by_row else tokens, k, seed=1), whole(len(counts), n, k, seed=2)
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    got = symar.experts(x, w, r, by_row=by_row, out=torch.full((rows, n), 7.0, dtype=out, device="cuda"), status=status)
    assert status.item() == symar.OK
    assert (got[:first] == 7).all() and (got[first + used:] == 7).all()
    for e in range(len(counts)):
        lo, hi = int(start[e]), int(start[e + 1])
        xe = x[lo:hi] if by_row else x[r.row_token[lo:hi].long()]
        assert torch.equal(got[lo:hi], (xe.double() @ w[e].double().T).float().to(out)), e
