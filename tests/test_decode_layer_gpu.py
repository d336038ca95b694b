"""The operators together, as the example runs them: products, append, attention, the ranks' projections into the symmetric heap and the
AllReduce, against the same chain in 64 bits."""
import importlib.util
from pathlib import Path

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu

PATH = Path(symar.__file__).parent / "examples" / "decode_layer.py"
spec = importlib.util.spec_from_file_location("decode_layer", PATH)
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def chain64(block, x, before, lengths, start):
    """The block in 64 bits.  `before`: every sequence's cached (keys, values) before the call; the new ones are taken from the cache as
    it holds them, so that quantisation, tested elsewhere, is no part of the comparison."""
    tokens, dim, share = x.shape[0], block.dim, block.q_heads // block.kv_heads
    qkv = (x.double() @ block.w_qkv.double().T).unflatten(1, (-1, dim))
    q = qkv[:, :block.q_heads]
    half = dim // 2
    out = torch.zeros(tokens, block.q_heads, dim, dtype=torch.float64, device="cuda")
    for b, total in enumerate(lengths):
        k, v = before[b]
        for row in range(start[b], start[b + 1]):
            pos = total - (start[b + 1] - row)
            c, s = block.rotations[pos, :, 0].double(), block.rotations[pos, :, 1].double()
            turned = torch.cat([q[row, :, :half] * c - q[row, :, half:] * s, q[row, :, half:] * c + q[row, :, :half] * s], -1)
            for h in range(block.q_heads):
                p = torch.softmax(k[:pos + 1, h // share] @ turned[h] * dim ** -0.5, 0)
                out[row, h] = p @ v[:pos + 1, h // share]
    of_ranks = out.view(tokens, block.ranks, -1).transpose(0, 1)
    return torch.bmm(of_ranks, block.w_out.double().transpose(1, 2)).sum(0) + x.double()


def held(block, lengths):
    """Keys and values of every sequence as the cache holds them."""
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    start = torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    k, v = block.context.read(block.cache, symar.KVBatch(n, block.page_table, start), sum(lengths), dtype=torch.float32)
    return list(zip(k.double().split(lengths), v.double().split(lengths)))


@pytest.mark.parametrize("ranks,hidden,hq,hkv,dim", [(8, 512, 16, 8, 64), (4, 256, 8, 2, 128), (2, 384, 10, 2, 64)])
def test_prompt_then_tokens(ranks, hidden, hq, hkv, dim):
    new = [37, 5, 64]
    block = example.AttentionBlock(ranks, hidden, hq, hkv, dim, seqs=3, tokens=sum(new), positions=100, page_size=16)
    gen = torch.Generator(device="cuda").manual_seed(3)
    lengths = [0, 0, 0]
    for counts in (new, [1, 1, 1], [1, 1, 1]):
        lengths = [a + b for a, b in zip(lengths, counts)]
        start = [0]
        for c in counts:
            start.append(start[-1] + c)
        x = torch.randn(start[-1], hidden, generator=gen, device="cuda").to(torch.bfloat16)
        one = all(c == 1 for c in counts)
        y = block(x, torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                  None if one else torch.tensor(start, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        block.check()
        for r in range(1, ranks):
            assert torch.equal(y[r], y[0])
        want = chain64(block, x, held(block, lengths), lengths, start)
        # roundings to bf16 along the way, 2^-8 of a value at most each: q, its rotation, probabilities, attention's output, partial
        # sums, the sum; in the 2-norm they stay below six times that
        assert (y[0].double() - want).norm() <= 6 * 2.0 ** -8 * want.norm()


def test_example_runs(capsys):
    example.main()
    assert "us per step" in capsys.readouterr().out
