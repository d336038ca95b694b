"""symar_experts against the formula in 64 bits.

Whole numbers: every product and sum is exact in binary32 in whatever order, so a result without an activation is the exact value
rounded once.  Real numbers: with S = sum |x w| (+ |bias|), sums are off by d = k 2^-23 S (bf16 results: one chain of truncating additions) or
(min(k, 128) 2^-23 + ceil(k / 128) 2^-24) S (float32), 8 x 2^-24 of S for bias and the activation's own roundings; |act'| < 1.13.  A gated result is
off by 1.13 d_gate |up| + |act| d_up + 1.13 d_gate d_up.  It is rounded once: 2^-8 (bf16) or 2^-24."""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
ACTS = {
    "none": lambda y: y,
    "relu": lambda y: y.clamp(min=0),
    "gelu": lambda y: 0.5 * y * torch.erfc(-y / math.sqrt(2)),
    "gelu_tanh": lambda y: 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))),
    "silu": lambda y: y * torch.sigmoid(y),
}


def normal(*shape, seed, scale=1.0, dtype=BF16):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def whole(*shape, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device="cuda").to(BF16)


def lists(counts, tokens, seed=0, spare=0):
    """Routes of given rows per expert; the rows' tokens are drawn, the last `spare` rows are nobody's."""
    rows = sum(counts) + spare
    g = torch.Generator().manual_seed(seed)
    row_token = torch.cat([torch.randint(0, tokens, (sum(counts),), generator=g), torch.full((spare,), -1)]).to(torch.int32).cuda()
    start = torch.tensor([0, *counts]).cumsum(0).to(torch.int32).cuda()
    one = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    r = symar.Routes(one, one.float(), start, row_token, one)
    r.tokens = tokens                      # (rows of any tokens, not a choice of each)
    return r


def reference(x, w, r, bias, act, gated, by_row):
    groups = x.shape[0] if x.dim() == 3 else (w.shape[0] if w.dim() == 4 else 1)
    n = w.shape[-2] // (2 if gated else 1)
    k = x.shape[-1]
    want, d = torch.zeros(groups, r.rows, n, dtype=torch.float64, device="cuda"), torch.zeros(groups, r.rows, n, dtype=torch.float64, device="cuda")
    start = r.expert_start.tolist()
    for g in range(groups):
        xg, wg = (x[g] if x.dim() == 3 else x).double(), w[g] if w.dim() == 4 else w
        for e in range(r.experts):
            lo, hi = start[e], start[e + 1]
            if lo == hi:
                continue
            xe = xg[lo:hi] if by_row else xg[r.row_token[lo:hi].long()]
            we = wg[e].double()
            b = 0.0 if bias is None else (bias[g, e] if bias.dim() == 3 else bias[e]).double()
            y, s = xe @ we.T + b, xe.abs() @ we.abs().T + abs(b)
            err = lambda out: {BF16: k * 2.0 ** -23, F32: min(k, 128) * 2.0 ** -23 + math.ceil(k / 128) * 2.0 ** -24}[out] + 8 * 2.0 ** -24      # noqa: E731
            want[g, lo:hi], d[g, lo:hi] = (ACTS[act](y), s) if not gated else (ACTS[act](y[:, :n]) * y[:, n:], 0.0)
            if gated:
                # (float32's chain is the shorter one; bf16's bound holds for both)
                f = err(BF16)
                d[g, lo:hi] = (1.13 * f * s[:, :n] * (y[:, n:].abs() + f * s[:, n:]) + ACTS[act](y[:, :n]).abs() * f * s[:, n:])
            else:
                d[g, lo:hi] = 1.13 * err(F32 if out_of.dtype == F32 else BF16) * s
    return want, d


class out_of:
    dtype = BF16


def check(x, w, r, bias=None, act="none", gated=False, by_row=False, out_dtype=BF16, **kw):
    out_of.dtype = out_dtype
    want, d = reference(x, w, r, bias, act, gated, by_row)
    out = kw.pop("out", None)
    if out is None:
        shape = want.shape if x.dim() == 3 or w.dim() == 4 else want.shape[1:]
        out = torch.full(shape, 7.0, dtype=out_dtype, device="cuda")
    got = symar.experts(x, w, r, bias=bias, act=act, gated=gated, by_row=by_row, out=out, **kw)
    assert got is out
    used = int(r.expert_start[-1])
    view = got.view(want.shape) if got.is_contiguous() else got
    if view.dim() == 2:
        view = view[None]
    assert (view[:, used:] == 7).all()
    half = 2.0 ** -8 if out_dtype == BF16 else 2.0 ** -24
    tol = (half + 8 * 2.0 ** -24) * want.abs() + d * (1 + half) + 1e-37
    err = (view[:, :used].double() - want[:, :used]).abs()
    assert torch.isfinite(view[:, :used]).all() and (err <= tol[:, :used]).all(), (err / tol[:, :used]).max().item()
    return got


COUNTS = [[1], [0, 3, 0], [1, 0, 2, 5, 1, 0, 0, 9], [16, 17, 31, 32, 33], [64, 65, 63, 1], [130, 0, 127, 128], [257, 255, 256, 300, 16], [1000]]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "_".join(map(str, c)))
@pytest.mark.parametrize("n,k", [(1, 8), (64, 64), (130, 72), (256, 520), (1003, 136)])
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("by_row", [False, True])
def test_whole_numbers_are_exact(counts, n, k, out, by_row):
    r = lists(counts, 50, seed=n, spare=3)
    x, w = whole(r.rows if by_row else 50, k, seed=1), whole(len(counts), n, k, seed=2)
    got = symar.experts(x, w, r, by_row=by_row, out=torch.full((r.rows, n), 7.0, dtype=out, device="cuda"))
    start = r.expert_start.tolist()
    for e in range(len(counts)):
        rows = slice(start[e], start[e + 1])
        xe = x[rows] if by_row else x[r.row_token[rows].long()]
        assert torch.equal(got[rows], (xe.double() @ w[e].double().T).float().to(out)), e
    assert (got[start[-1]:] == 7).all()


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "_".join(map(str, c)))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("act", list(ACTS))
def test_real_numbers(counts, gated, out, act):
    r = lists(counts, 40, seed=3, spare=1)
    n, k, e = 200, 328, len(counts)
    x, w = normal(40, k, seed=1), normal(e, n * (1 + gated), k, seed=2, scale=k ** -0.5)
    check(x, w, r, normal(e, n * (1 + gated), seed=3), act, gated, out_dtype=out)


@pytest.mark.parametrize("n", [1, 3, 60, 63, 64, 65, 128, 129, 516, 1031])
@pytest.mark.parametrize("k", [8, 56, 64, 120, 2048])
@pytest.mark.parametrize("gated", [False, True])
def test_sizes(n, k, gated):
    r = lists([5, 40, 0, 1], 20, spare=2)
    for out in (BF16, F32):
        check(normal(20, k, seed=1), normal(4, n * (1 + gated), k, seed=2, scale=k ** -0.5), r, None, "silu", gated, out_dtype=out)


@pytest.mark.parametrize("ranks", [2, 5])
@pytest.mark.parametrize("shared", ["none", "x", "w"])
@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_ranks(ranks, shared, by_row, gated):
    for counts in ([3, 0, 2], [200, 90, 1]):
        r = lists(counts, 30, spare=2)
        n, k = 136, 264
        x = normal(*(() if shared == "x" else (ranks,)), r.rows if by_row else 30, k, seed=1)
        w = normal(*(() if shared == "w" else (ranks,)), 3, n * (1 + gated), k, seed=2, scale=k ** -0.5)
        bias = normal(ranks, 3, n * (1 + gated), seed=3)
        for out in (BF16, F32):
            check(x, w, r, bias if shared != "w" else bias[0], "gelu", gated, by_row, out)


@pytest.mark.parametrize("by_row", [False, True])
def test_strides(by_row):
    """Operands and results inside larger tensors, ranks side by side in a row; nothing beside the result is written."""
    r = lists([9, 70, 0, 33], 24, spare=2)
    rows, n, k = r.rows if by_row else 24, 100, 192
    x = normal(rows, 3, k + 16, seed=1)[:, 1:, 8:8 + k].transpose(0, 1)
    w = normal(2, 4, n + 5, k + 8, seed=2, scale=k ** -0.5)[:, :, 2:n + 2, :k]
    for offset in (0, 1, 4):
        for out in (BF16, F32):
            room = torch.full((r.rows, 2, n + 8), 7.0, dtype=out, device="cuda")
            got = room[..., offset:offset + n].transpose(0, 1)
            check(x, w, r, by_row=by_row, out_dtype=out, out=got)
            assert (room[..., :offset] == 7).all() and (room[..., offset + n:] == 7).all()
    many = normal(5, 1, k, seed=4)                                   # one token of every rank
    one = lists([1, 2, 0, 1], 1)
    check(many, normal(4, n, k, seed=2, scale=k ** -0.5), one)


def test_rows_on_no_boundary_are_refused():
    r = lists([3, 2], 8)
    x, w = normal(8, 136, seed=1), normal(2, 16, 136, seed=2)
    for bad in ((x[:, 1:129], w[..., :128]), (x[:, :128], w[..., 1:129]), (normal(8, 132, seed=1)[:, :128], w[..., :128]), (x[:, :100], normal(2, 16, 100, seed=1)),
                (normal(1, 136, seed=1).expand(8, 136), w), (x, w[:1].expand(2, 16, 136))):
        with pytest.raises(symar.SymarError) as e:
            symar.experts(*bad, r)
        assert e.value.code == symar.ERR_UNSUPPORTED
    check(x[:, :100], w[..., :100], r)                               # odd k in rows on boundaries


def test_lists_that_are_wrong():
    """Starts that fall or leave the rows are brought into order; tokens outside x are reported, other rows right."""
    x, w = whole(10, 64, seed=1), whole(3, 40, 64, seed=2)
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    r = lists([4, 5, 3], 10)
    r.expert_start.copy_(torch.tensor([-7, 4, 2, 100]))
    out = torch.full((12, 40), 7.0, device="cuda", dtype=BF16)
    symar.experts(x, w, r, out=out, status=status)
    xe = x[r.row_token.long()].double()
    want = torch.cat([xe[:4] @ w[0].double().T, xe[4:] @ w[2].double().T])
    assert torch.equal(out, want.to(BF16)) and status.item() == symar.OK
    r = lists([4, 5, 3], 10)
    r.row_token[5], r.row_token[9] = 10, -2
    symar.experts(x, w, r, out=out, status=status)
    assert status.item() == symar.ERR_INVAL
    fine = [i for i in range(12) if i not in (5, 9)]
    e = torch.tensor([0] * 4 + [1] * 5 + [2] * 3)
    want = torch.stack([w[e[i]].double() @ x[r.row_token[i]].double() for i in fine])
    assert torch.equal(out[fine], want.to(BF16))
    symar.experts(x, w, lists([4, 5, 3], 10), out=out, status=status)
    assert status.item() == symar.OK


def test_values_that_are_not_finite_stay_in_their_row():
    r = lists([20, 30], 12, seed=5)
    x, w = whole(12, 128, seed=1), whole(2, 72, 128, seed=2)
    w = torch.where(w == 0, torch.ones_like(w), w)
    x[3, 5], x[4, 7] = math.nan, math.inf
    got = symar.experts(x, w, r, out_dtype=F32)
    e = torch.tensor([0] * 20 + [1] * 30, device="cuda")
    want = torch.einsum("rk,rnk->rn", x[r.row_token.long()].double(), w[e].double())
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[fine].double(), want[fine])


def test_nothing_to_sum_and_nothing_to_do():
    r = lists([3, 0, 2], 4, spare=1)
    x, w, b = torch.empty(4, 0, device="cuda", dtype=BF16), torch.empty(3, 20, 0, device="cuda", dtype=BF16), normal(3, 20, seed=1)
    out = torch.full((6, 20), 7.0, device="cuda", dtype=BF16)
    symar.experts(x, w, r, bias=b, act="relu", out=out)
    assert torch.equal(out[:5], b.clamp(min=0)[[0, 0, 0, 2, 2]]) and (out[5] == 7).all()
    none = symar.route(torch.empty(0, 3, device="cuda"), 2)
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    assert symar.experts(torch.empty(0, 64, device="cuda", dtype=BF16), normal(3, 8, 64, seed=1), none, status=status).shape == (0, 8)
    assert status.item() == symar.OK
    idle = symar.route(torch.full((5, 3), -math.inf, device="cuda"), 2)
    out = torch.full((10, 8), 7.0, device="cuda", dtype=BF16)
    symar.experts(normal(5, 64, seed=2), normal(3, 8, 64, seed=1), idle, out=out)
    assert (out == 7).all()


def test_a_graph_replays_other_lists():
    """The lists are read on the device: a captured call goes by what they hold when it is replayed."""
    x, w, w2 = normal(96, 256, seed=1), normal(16, 2 * 128, 256, seed=2, scale=1 / 16), normal(16, 256, 128, seed=3, scale=1 / 11)
    logits = normal(96, 16, seed=4, dtype=F32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            r = symar.route(logits, 3)
            h = symar.experts(x, w, r, act="silu", gated=True)
            y = symar.combine(symar.experts(h, w2, r, by_row=True), r)
    for seed in (5, 6, 7):
        logits.copy_(normal(96, 16, seed=seed, dtype=F32) + (30 if seed == 6 else 0) * (torch.arange(16, device="cuda") < 3))
        graph.replay()
        torch.cuda.synchronize()
        a = symar.route(logits, 3)
        b = symar.experts(x, w, a, act="silu", gated=True)
        assert torch.equal(a.row_token, r.row_token) and torch.equal(h, b)
        assert torch.equal(symar.combine(symar.experts(b, w2, a, by_row=True), a), y)
        check(x, w, a, None, "silu", True)


def test_refusals():
    r = lists([3, 2], 8)
    x, w, b = normal(8, 64, seed=1), normal(2, 16, 64, seed=2), normal(2, 16, seed=3)
    for kw in (dict(bias=b[:, :8]), dict(bias=b.float()), dict(act="tanh"), dict(by_row=True), dict(out=torch.empty(4, 16, device="cuda", dtype=BF16)),
               dict(out=torch.empty(5, 16, device="cuda", dtype=BF16), out_dtype=F32), dict(out_dtype=torch.float16), dict(gated=True, bias=b[0]),
               dict(status=b), dict(out=torch.empty(1, 16, device="cuda", dtype=BF16).expand(5, 16))):
        with pytest.raises(symar.SymarError):
            symar.experts(x, w, r, **kw)
    for a, c in ((x.float(), w), (x[:7], w), (x, w[:1]), (x, w[..., :32]), (x.cpu(), w), (x, w.cpu()), (x[None, None], w), (x, w[0]), (x[None], w[None].expand(2, 2, 16, 64)),
                 (x.T.contiguous().T, w)):
        with pytest.raises(symar.SymarError):
            symar.experts(a, c, r)
    with pytest.raises(symar.SymarError):
        symar.experts(x, w[:, :15], r, gated=True)                   # rows of gate and up: not an even number


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("counts,n,k", [([1], 64, 4096), ([3], 200, 1000), ([1, 0, 2], 129, 2048), ([5, 64, 1, 0, 9], 24, 1536), ([70, 3], 100, 4104),
                                        ([1, 2, 9, 1, 17, 0, 33, 64, 1, 5], 1280, 8192)], ids=lambda c: str(c).replace(" ", ""))
def test_few_tiles_share_multiprocessors(counts, n, k, by_row, out, gated):
    """Products of few tiles over a long k, which blocks divide; the last one has several tiles for each group of blocks."""
    if gated and n == 1280:
        n = 640
    r = lists(counts, 30, spare=2)
    x = whole(r.rows if by_row else 30, k, seed=1)
    w = whole(len(counts), n * (1 + gated), k, seed=2)
    if not gated:
        got = symar.experts(x, w, r, by_row=by_row, out_dtype=out)
        start = r.expert_start.tolist()
        for e in range(len(counts)):
            rows = slice(start[e], start[e + 1])
            xe = x[rows] if by_row else x[r.row_token[rows].long()]
            assert torch.equal(got[rows], (xe.double() @ w[e].double().T).float().to(out)), e
    x, w = normal(*x.shape, seed=3), normal(*w.shape, seed=4, scale=k ** -0.5)
    first = check(x, w, r, normal(len(counts), n * (1 + gated), seed=5), "silu", gated, by_row, out)
    again = check(x, w, r, normal(len(counts), n * (1 + gated), seed=5), "silu", gated, by_row, out)
    assert torch.equal(first, again)


@pytest.mark.parametrize("experts", [31, 32, 33, 127, 128, 129, 500, 1024])
@pytest.mark.parametrize("most", [3, 130])
def test_numbers_of_experts(experts, most):
    """Experts with and without rows at every place of the counting."""
    g = torch.Generator().manual_seed(experts)
    counts = (torch.randint(0, most, (experts,), generator=g) * (torch.rand(experts, generator=g) < 0.6)).tolist()
    counts[-1] = 2
    r = lists(counts, 60, seed=1, spare=2)
    x, w = whole(60, 64, seed=1), whole(experts, 24, 64, seed=2)
    for out in (BF16, F32):
        got = symar.experts(x, w, r, out=torch.full((r.rows, 24), 7.0, dtype=out, device="cuda"))
        e = torch.repeat_interleave(torch.arange(experts), torch.tensor(counts)).cuda()
        used = len(e)
        want = torch.einsum("rk,rnk->rn", x[r.row_token[:used].long()].double(), w[e].double())
        assert torch.equal(got[:used], want.float().to(out)) and (got[used:] == 7).all()
