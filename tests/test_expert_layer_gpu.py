"""The operators of a mixture of experts together, as examples/expert_layer.py runs them, against the layer in 64 bits.

Bound of the result in the 2-norm, of the block's own norm: every rounding to bf16 is off by 2^-8 of its tensor; the products' and sums' binary32 is far
below.  A random product takes a rounding of its operand to at most three times that of its result (1 + sqrt(k / n) and alike, for the sizes here), the gated
activation counts its two factors.  x as it enters: none; silu(gate) up: 1, 3 behind the way down; the rows: 1; the sums of a token's
rows: 1; the AllReduce of eight ranks' sums: 1; the norm of that: 2 (a factor's error beside the vector's).  Together below 16 x 2^-8 of the block's result, and a rounding of what is
stored."""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar
from paper_2607_16100_b200.examples import decode_layer, expert_layer

pytestmark = pytest.mark.gpu


def in_64_bits(block, x, stream, idle):
    r, n = block.routes, x.shape[0]
    x = x.double()
    logits = x @ block.w_router.double().T
    score = torch.sigmoid(logits)
    out = torch.zeros_like(x)
    for t in range(n):
        if idle is not None and idle[t]:
            assert (r.choice[t] == -1).all()
            continue
        chosen = r.choice[t].long()
        # the router's own choice may differ from 64 bits' where logits are next to each other: by no more than their bound
        least, rest = score[t, chosen].min(), score[t].clone()
        rest[chosen] = -1
        assert rest.max() <= least + 1e-4
        weights = score[t, chosen] / score[t, chosen].sum()
        for w, e in zip(weights, chosen):
            for g in range(block.ranks):
                h = block.w_in[g, e].double() @ x[t]
                gate, up = h.chunk(2)
                out[t] += w * (block.w_out[g, e].double() @ (gate * torch.sigmoid(gate) * up))
    def rms(v, norm):
        return v / (v.square().mean(-1, keepdim=True) + 1e-5).sqrt() * norm.weight.double()
    a = rms(out, block.after)
    new = stream.double() + a
    return rms(new, block.before), new, a


def near(got, want, size):
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    err = (got.double() - want).norm(dim=-1)
    assert (err <= 16 * 2.0 ** -8 * size + half * want.norm(dim=-1)).all(), (err / size).max().item()


@pytest.mark.parametrize("tokens,dtype", [(1, torch.bfloat16), (5, torch.float32), (40, torch.bfloat16)])
def test_the_block_against_64_bits(tokens, dtype):
    block = expert_layer.ExpertBlock(8, 512, 16, 4, 768, tokens=48)
    g = torch.Generator("cuda").manual_seed(tokens)
    stream = torch.randn(tokens, 512, generator=g, device="cuda").to(dtype)
    idle = torch.zeros(tokens, 1, dtype=torch.bool, device="cuda")
    if tokens > 4:
        idle[3] = True
    x, _ = symar.norm(stream.bfloat16(), before=block.before)
    y, new = block(x, stream, idle)
    block.check()
    want, want_new, a = in_64_bits(block, x, stream, idle)
    near(new, want_new, a.norm(dim=-1))
    # the last norm divides what it is off by the stream's size
    near(y, want, a.norm(dim=-1) / want_new.square().mean(-1).sqrt() * 1.5)
    for q in range(block.ranks):
        assert torch.equal(block.summed[q, :tokens], block.summed[0, :tokens])


def test_a_captured_layer_follows_its_tokens():
    """Attention and experts of a layer in one graph: replays with other tokens, some of them idle, give what calls give."""
    hidden, seqs = 512, 6
    attention = decode_layer.AttentionBlock(8, hidden, 8, 8, 64, seqs=seqs, tokens=seqs, positions=64, page_size=16)
    other = decode_layer.AttentionBlock(8, hidden, 8, 8, 64, seqs=seqs, tokens=seqs, positions=64, page_size=16)
    experts = expert_layer.ExpertBlock(8, hidden, 16, 2, 512, tokens=seqs)
    g = torch.Generator("cuda").manual_seed(1)

    def layer(block, x, lengths, idle):
        h = block(x, lengths)[0]
        y, _ = symar.norm(h, before=experts.before)
        return experts(y, h, idle)

    x, lengths = torch.zeros(seqs, hidden, device="cuda", dtype=torch.bfloat16), torch.zeros(seqs, dtype=torch.int32, device="cuda")
    idle = torch.zeros(seqs, 1, dtype=torch.bool, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y, new = layer(attention, x, lengths, idle)
    for step in range(4):
        x.copy_(torch.randn(seqs, hidden, generator=g, device="cuda"))
        lengths.copy_(torch.tensor([step + 1] * 4 + [0, step // 2]))
        idle.copy_((lengths == 0)[:, None])
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), new.clone()
        want = layer(other, x, lengths, idle)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.isfinite(got[0]).all()
    attention.check(), other.check(), experts.check()


def test_the_example_runs(capsys):
    expert_layer.main()
    assert capsys.readouterr().out.count("us per step") == 4


def test_no_choice_of_a_finite_router_is_lost():
    """Every token's weights sum to one, every row stands in its expert's range."""
    x = torch.randn(3000, 96, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    r = symar.route(x, 6)
    assert ((r.weights.sum(-1) - 1).abs() < 8 * 2.0 ** -24).all() and int(r.expert_start[-1]) == 18000
    start, row = r.expert_start.long(), r.token_row.long()
    assert ((row >= start[r.choice.long()]) & (row < start[r.choice.long() + 1])).all()
    assert torch.equal(row.flatten().sort().values, torch.arange(18000, device="cuda"))
    assert torch.equal(r.row_token[row].long(), torch.arange(3000, device="cuda")[:, None].expand(3000, 6))
    assert math.isfinite(float(r.weights.sum()))
