"""The operators on streams: behind work of other streams, behind copies and fills, captured with forks and joins.  Whole-number operands,
whose products are exact in any order, and results of an uncaptured call, which have to come out again bit for bit."""
import ctypes

import pytest
import torch

from paper_2607_16100_b200 import symar
from test_kv_gpu import Setup, kv, normal      # noqa: F401  (kv is a fixture)

pytestmark = pytest.mark.gpu


def whole(*shape, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device="cuda").to(torch.bfloat16)


def test_a_chain_of_products_sees_every_result():
    """Each product reads what the one before it wrote, two hundred of them without a pause."""
    n = 256
    perm = torch.randperm(n, generator=torch.Generator().manual_seed(1))
    w = torch.eye(n)[perm].to(torch.bfloat16).cuda()          # y[:, i] = x[:, perm[i]]
    x = whole(5, n, seed=2)
    a, b = x.clone(), torch.empty_like(x)
    want = x.cpu()
    for _ in range(200):
        symar.linear(a, w, out=b)
        a, b = b, a
        want = want[:, perm]
    assert torch.equal(a.cpu(), want)


def test_behind_fills_and_copies():
    """The operand is overwritten by a fill and a copy on the same stream right before and right after each call."""
    x, w = whole(64, 512, seed=3), whole(256, 512, seed=4)
    y = (x.float() @ w.float().T).to(torch.bfloat16)
    out, buf = torch.empty(64, 256, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    outs = []
    for _ in range(50):
        buf.fill_(7)
        buf.copy_(x)
        outs.append(symar.linear(buf, w))
        buf.fill_(9)
        out.zero_()
        symar.linear(x, w, out=out)
        outs.append(out.clone())
    assert all(torch.equal(o, y) for o in outs)


def test_captured_with_a_fork_a_join_and_a_status_word(kv):  # noqa: F811
    c = symar.KVContext.on_torch()
    s = Setup([(3, 40), (1, 200), (2, 17)], 2, 128, 16, seed=9)
    s.fill(kv, seed=91)
    q = normal(s.tokens, 8, 128, seed=3)
    want = kv.attention(s.cache, s.batch, q).clone()
    x, w = whole(7, 128, seed=5), whole(96, 128, seed=6)
    y = (x.float() @ w.float().T).to(torch.bfloat16)
    word = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    staged, out, prod = torch.empty_like(q), torch.empty_like(q), torch.empty_like(y)
    args = symar.LinearArgs(x=x.data_ptr(), x_ld=128, x_group=0, w=w.data_ptr(), w_ld=128, w_group=0, out=prod.data_ptr(), out_ld=96,
                            out_group=0, m=7, n=96, k=128, groups=1, act=0, root=-1, out_dtype=symar.BF16, status=word.data_ptr())
    lib = symar.load()
    main, side, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    main.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(main), torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        with torch.cuda.stream(side):
            assert lib.symar_linear(ctypes.byref(args), ctypes.c_void_p(side.cuda_stream)) == symar.OK
        staged.copy_(q)
        main.wait_stream(side)
        c.attention(s.cache, s.batch, staged, out=out)
        kv.attention(s.cache, s.batch, out, out=staged)       # one more behind it, of its result
    for _ in range(3):
        out.zero_(), prod.zero_(), word.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(prod, y) and word.item() == symar.OK
        assert torch.equal(staged, kv.attention(s.cache, s.batch, want))
    assert c.status()[0] == symar.OK
