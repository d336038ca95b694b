"""Norm, router, experts and combine as a program calls them: on streams given by handle, from several threads, in graphs that fork and join, with results
that are views."""
import threading

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(*shape, seed, scale=1.0, dtype=BF16):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


class Layer:
    """One expert layer's calls, with many rows (pairs, rows put in order first) or few."""

    def __init__(self, tokens, seed=0, hidden=256, experts=8, top_k=2):
        self.top_k = top_k
        self.x, self.res, self.w = normal(tokens, hidden, seed=seed), normal(tokens, hidden, seed=seed + 1, dtype=F32), normal(hidden, seed=9)
        self.router = normal(experts, hidden, seed=3, scale=1 / 16)
        self.w_in, self.w_out = normal(experts, 2 * 640, hidden, seed=4, scale=1 / 16), normal(experts, hidden, 640, seed=5, scale=1 / 25)
        self.norm = symar.Norm("rms", self.w, eps=1e-5)

    def __call__(self, x=None, res=None, stream=None):
        x, res = self.x if x is None else x, self.res if res is None else res
        y, r = symar.norm(x, res, after=self.norm, before=self.norm, stream=stream)
        logits = symar.linear(y, self.router, out_dtype=F32, stream=stream)
        routes = symar.route(logits, self.top_k, stream=stream)
        h = symar.experts(y, self.w_in, routes, gated=True, act="silu", stream=stream)
        h = symar.experts(h, self.w_out, routes, by_row=True, stream=stream)
        return symar.combine(h, routes, residual=y, stream=stream), r


@pytest.mark.parametrize("tokens", [3, 100, 3000])
def test_on_a_stream_given_by_handle(tokens):
    """Everything behind a long wait on that stream, with operands that are made there, and nothing of it kept by the caller but the results."""
    layer = Layer(tokens)
    want = layer()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
            x, res = layer.x * 1, layer.res * 1
        got = layer(x, res, stream=side.cuda_stream)
        junk = [torch.full((tokens, 4096), 7.0, device="cuda") for _ in range(4)]      # (memory of the current stream's pool is another)
        side.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        del junk


def test_from_several_threads():
    layers = [Layer(t, seed=t) for t in (5, 700, 64, 2500)]
    want = [layer() for layer in layers]
    torch.cuda.synchronize()
    wrong = []

    def work(layer, want):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(30):
                got = layer()
                stream.synchronize()
                if not (torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])):
                    wrong.append(layer)
    threads = [threading.Thread(target=work, args=a) for a in zip(layers, want)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong


def test_two_branches_of_a_graph_and_a_graph_beside_it():
    """Two layers side by side in one graph and the same ones in another: no workspace is shared."""
    a, b = Layer(2500), Layer(900, seed=7)
    want = a(), b()
    main, side, graphs, outs = torch.cuda.Stream(), torch.cuda.Stream(), [], []
    main.wait_stream(torch.cuda.current_stream())
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(main), torch.cuda.graph(graph, stream=main):
            side.wait_stream(main)
            with torch.cuda.stream(side):
                left = a()
            right = b()
            main.wait_stream(side)
        graphs.append(graph), outs.append((left, right))
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(main):
            graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for got in outs:
            for g, w in zip(got, want):
                assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


def test_lists_of_a_program_of_its_own():
    """Routes from tensors that a program made; a token may name an expert twice."""
    x, w = normal(6, 64, seed=1), normal(3, 40, 64, seed=2)
    choice = torch.tensor([[0, 0], [2, 0], [1, 2], [2, 2], [1, 1], [0, 1]], dtype=torch.int32, device="cuda")
    order = torch.sort(choice.flatten(), stable=True).indices
    start = torch.tensor([0, 4, 8, 12], dtype=torch.int32, device="cuda")
    row = torch.empty(12, dtype=torch.int32, device="cuda")
    row[order] = torch.arange(12, dtype=torch.int32, device="cuda")
    weights = torch.rand(6, 2, device="cuda")
    r = symar.Routes(choice, weights, start, (order // 2).to(torch.int32), row.view(6, 2))
    assert r.choice is choice and r.experts == 3 and r.rows == 12
    got = symar.combine(symar.experts(x, w, r, out_dtype=F32), r)
    def summed(x, w):
        return sum(weights[:, j, None].double() * torch.einsum("tk,tnk->tn", x, w[choice[:, j].long()]) for j in range(2))
    # 64 truncating additions of 2^-23, one more sum, two weights and their sum, of the terms' sizes; the result's half step
    size = summed(x.double().abs(), w.double().abs())
    tol = (64 * 2.0 ** -23 + 8 * 2.0 ** -24) * size
    assert ((got.double() - summed(x.double(), w.double())).abs() <= tol).all()


def test_results_into_the_heap():
    heap = symar.SymHeap.on_torch(4, 1 << 16)
    r = symar.route(normal(20, 8, seed=1, dtype=F32), 2)
    y = normal(4, r.rows, 64, seed=2)
    out = heap.view(0, (20, 64), BF16)
    assert symar.combine(y, r, out=out) is out
    assert torch.equal(out, symar.combine(y, r))
    x, res = normal(20, 64, seed=3), normal(20, 64, seed=4)
    n = symar.Norm("rms")
    into = heap.view(8192, (20, 64), BF16)
    symar.norm(x.expand(4, 20, 64), res.expand(4, 20, 64), before=n, out=into, residual_out=torch.empty(4, 20, 64, dtype=BF16, device="cuda"))
    want, _ = symar.norm(x, res, before=n)
    assert all(torch.equal(into[q], want) for q in range(4))
