"""symar_experts with many rows an expert: tiles of 256 rows by pairs of multiprocessors, rows by token put in order first, against the formula in 64 bits.  Bounds:
test_experts_gpu.py's.  That a case is one of them shows in the workspace that its rows by token ask for."""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar
from test_experts_gpu import ACTS, BF16, check, lists, normal, whole

pytestmark = pytest.mark.gpu


def in_pairs(r, w, gated, ranks=1):
    n, k = w.shape[-2] // (2 if gated else 1), w.shape[-1]
    k_room = (k + 7) // 8 * 8
    a = symar.ExpertsArgs(x_ld=k_room, x_group=k_room, row_token=1 << 20, groups=ranks, experts=r.experts, rows=r.rows, x_rows=r.tokens, n=n, k=k, out_dtype=symar.BF16,
                          gated=1 if gated else 0)
    import ctypes
    return symar.load().symar_experts_workspace(ctypes.byref(a)) > 0


COUNTS = [[257, 0, 256, 1, 700, 255, 512, 90], [600, 0, 0, 1400], [1, 2, 3, 1900, 0, 0, 127, 129, 33, 64], [5000]]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "_".join(map(str, c)))
@pytest.mark.parametrize("n,k", [(2600, 72), (2563, 136), (2600, 1000), (2688, 520)])
@pytest.mark.parametrize("by_row", [False, True])
def test_whole_numbers_are_exact(counts, n, k, by_row):
    """Several turns of the ring, a part of a slice at the end, an odd number of 128 channels, rows on no boundary."""
    n = n * 3 if len(counts) == 4 else n
    r = lists(counts, 90, seed=n, spare=3)
    x, w = whole(r.rows if by_row else 90, k, seed=1), whole(len(counts), n, k, seed=2)
    assert in_pairs(r, w, False)
    got = symar.experts(x, w, r, by_row=by_row, out=torch.full((r.rows, n), 7.0, dtype=BF16, device="cuda"))
    start = r.expert_start.tolist()
    for e in range(len(counts)):
        rows = slice(start[e], start[e + 1])
        xe = x[rows] if by_row else x[r.row_token[rows].long()]
        assert torch.equal(got[rows], (xe.double() @ w[e].double().T).float().to(BF16)), e
    assert (got[start[-1]:] == 7).all()


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "_".join(map(str, c)))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("act", list(ACTS))
def test_real_numbers(counts, gated, by_row, act):
    n, k, e = (3 if len(counts) == 4 else 1) * (1300 if gated else 2600), 328, len(counts)
    r = lists(counts, 300, seed=3, spare=1)
    x, w = normal(r.rows if by_row else 300, k, seed=1), normal(e, n * (1 + gated), k, seed=2, scale=k ** -0.5)
    assert in_pairs(r, w, gated)
    check(x, w, r, normal(e, n * (1 + gated), seed=3), act, gated, by_row)


@pytest.mark.parametrize("n", [1281, 1340, 1343, 1344, 1345, 1408, 1409])
@pytest.mark.parametrize("k", [8, 56, 64, 120, 264, 3000])
@pytest.mark.parametrize("gated", [False, True])
def test_sizes(n, k, gated):
    n = n if gated else 2 * n
    counts = [300, 0, 530, 220, 255, 700]
    r = lists(counts, 100, seed=n, spare=2)
    w = normal(6, n * (1 + gated), k, seed=2, scale=k ** -0.5)
    assert in_pairs(r, w, gated)
    check(normal(100, k, seed=1), w, r, None, "silu", gated)


@pytest.mark.parametrize("ranks", [2, 5])
@pytest.mark.parametrize("shared", ["none", "x", "w"])
@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_ranks(ranks, shared, by_row, gated):
    r = lists([400, 290, 1, 0, 900], 130, spare=2)
    n, k = 1100 if gated else 2200, 264
    x = normal(*(() if shared == "x" else (ranks,)), r.rows if by_row else 130, k, seed=1)
    w = normal(*(() if shared == "w" else (ranks,)), 5, n * (1 + gated), k, seed=2, scale=k ** -0.5)
    bias = normal(ranks, 5, n * (1 + gated), seed=3)
    assert in_pairs(r, w, gated, ranks)
    check(x, w, r, bias if shared != "w" else bias[0], "gelu", gated, by_row)


@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_strides(by_row, gated):
    """Operands and results inside larger tensors, ranks side by side in a row; nothing beside the result is written."""
    r = lists([900, 700, 0, 333], 240, spare=2)
    rows, n, k = r.rows if by_row else 240, 1300, 100
    wide = n * (1 + gated)
    x = normal(rows, 3, 120, seed=1)[:, 1:, 8:8 + k].transpose(0, 1)
    w = normal(2, 4, wide + 5, 128, seed=2, scale=k ** -0.5)[:, :, 2:wide + 2, :k]
    assert in_pairs(r, w, gated, 2)
    for offset in (0, 1, 4):
        room = torch.full((r.rows, 2, n + 8), 7.0, dtype=BF16, device="cuda")
        check(x, w, r, by_row=by_row, gated=gated, act="silu", out=room[..., offset:offset + n].transpose(0, 1))
        assert (room[..., :offset] == 7).all() and (room[..., offset + n:] == 7).all()


def test_more_tiles_than_pairs_and_the_same_bits_again():
    """Many tiles a pair, several rounds of both accumulators; another call, and a replay of a captured one, give the same bits."""
    r = lists([1000, 1, 0, 3000, 517, 2000], 1500, spare=2)
    x, w, bias = normal(1500, 712, seed=1), normal(6, 2 * 1536, 712, seed=2, scale=712 ** -0.5), normal(6, 2 * 1536, seed=3)
    assert in_pairs(r, w, True)
    first = check(x, w, r, bias, "silu", True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(first)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            symar.experts(x, w, r, bias=bias, act="silu", gated=True, out=out)
    used = int(r.expert_start[-1])
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:used], first[:used])


def test_values_that_are_not_finite_stay_in_their_row_and_wrong_tokens_are_reported():
    r = lists([900, 1100], 40, seed=5)
    x, w = whole(40, 128, seed=1), whole(2, 3000, 128, seed=2)
    w = torch.where(w == 0, torch.ones_like(w), w)
    assert in_pairs(r, w, False)
    y = x.clone()
    y[3, 5], y[4, 7] = math.nan, math.inf
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    got = symar.experts(y, w, r, status=status)
    assert status.item() == symar.OK
    token = r.row_token.long()
    fine = (token != 3) & (token != 4)
    want = torch.cat([x[token[:900]].double() @ w[0].double().T, x[token[900:]].double() @ w[1].double().T]).float().to(BF16)
    assert torch.equal(got[fine], want[fine]) and torch.isnan(got[token == 3]).all() and torch.isinf(got[token == 4]).all()
    r.row_token[5], r.row_token[1999] = 40, -2
    got = symar.experts(x, w, r, status=status)
    assert status.item() == symar.ERR_INVAL
    fine = torch.ones(2000, dtype=torch.bool, device="cuda")
    fine[[5, 1999]] = False
    assert torch.equal(got[fine], want[fine])


def test_lists_that_are_wrong():
    r = lists([800, 600, 700], 64, seed=1)
    x, w = whole(64, 64, seed=1), whole(3, 4000, 64, seed=2)
    assert in_pairs(r, w, False)
    r.expert_start.copy_(torch.tensor([-7, 900, 200, 100000]))
    got = symar.experts(x, w, r)
    xe = x[r.row_token.long()].double()
    assert torch.equal(got, torch.cat([xe[:900] @ w[0].double().T, xe[900:] @ w[2].double().T]).float().to(BF16))
