"""The feed-forward half of a tensor-parallel decoder layer with a mixture of experts, on P emulated ranks, around its AllReduce.

One step for a batch of tokens, some of which may be idle slots:

1. ``symar.linear``     the router's logits, on every rank the same;
2. ``symar.route``      every token's experts, and the lists that sort tokens by expert;
3. ``symar.experts``    gate and up of every rank's share of the experts' channels, the tokens gathered, silu(gate) * up;
4. ``symar.experts``    the way down, on the rows as they stand: each rank's partial sums;
5. ``symar.combine``    a token's rows summed with their weights, straight into the rank's segment of the symmetric heap;
6. ``SymHeap.allreduce`` the sum of the partial sums, on every rank;
7. ``symar.norm``       that normed and added to the residual stream, and the sum normed for the next block: one pass.

Run it:  python -m paper_2607_16100_b200.examples.expert_layer
"""
from __future__ import annotations

import math

import torch

from paper_2607_16100_b200 import symar


class ExpertBlock:
    def __init__(self, ranks: int, hidden: int, experts: int, top_k: int, channels: int, *, tokens: int, seed: int = 0, device="cuda"):
        if channels % ranks:
            raise ValueError("every rank has the same share of an expert's channels")
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape, fan):
            return (torch.randn(*shape, generator=g, device=device) * fan ** -0.5).to(torch.bfloat16)

        self.ranks, self.hidden, self.top_k = ranks, hidden, top_k
        share = channels // ranks
        self.w_router = weight(experts, hidden, fan=hidden)
        self.w_in = weight(ranks, experts, 2 * share, hidden, fan=hidden)       # the gate's channels, then up's
        self.w_out = weight(ranks, experts, hidden, share, fan=channels)
        self.bias = torch.zeros(experts, device=device)                        # what balances the experts: takes part in the choice only
        self.after, self.before = (symar.Norm("rms", 1 + weight(hidden, fan=100), eps=1e-5) for _ in range(2))
        self.heap = symar.SymHeap.on_torch(ranks, 2 * -(-tokens * hidden * 2 // symar.ALIGN) * symar.ALIGN, device)
        self.out_offset = self.heap.bytes_per_rank // 2
        self.partial = self.heap.view(0, (tokens, hidden), torch.bfloat16)
        self.summed = self.heap.view(self.out_offset, (tokens, hidden), torch.bfloat16)
        self.word = torch.zeros(3, dtype=torch.int32, device=device)

    def __call__(self, x, stream, idle=None):
        """x [tokens, hidden] bf16, the normed stream; stream [tokens, hidden], the residual stream (bf16 or float32); idle [tokens, 1] bool: slots
        without a token.  Returns (the next block's x, the stream with this block's result)."""
        tokens = x.shape[0]
        logits = symar.linear(x, self.w_router, out_dtype=torch.float32)
        if idle is not None:
            logits.masked_fill_(idle, -math.inf)
        self.routes = symar.route(logits, self.top_k, score="sigmoid", bias=self.bias)
        rows = symar.experts(x, self.w_in, self.routes, gated=True, act="silu", status=self.word[:1])
        rows = symar.experts(rows, self.w_out, self.routes, by_row=True, status=self.word[1:2])
        symar.combine(rows, self.routes, out=self.partial[:, :tokens])
        self.heap.allreduce(0, self.out_offset, tokens * self.hidden, symar.BF16, symar.AUTO, torch.cuda.current_stream().cuda_stream)
        return symar.norm(self.summed[0, :tokens], stream, after=self.after, before=self.before, status=self.word[2:])

    def check(self) -> None:
        """Raises if a call recorded an error on the device (synchronises)."""
        for code, *where in (self.heap.status(), *((c,) for c in self.word.tolist())):
            if code != symar.OK:
                raise symar.SymarError(code, f"on the device, at {where}")


def main() -> None:
    # hidden size 8192 over eight ranks, 64 experts of 2048 channels, four a token
    block = ExpertBlock(8, 8192, 64, 4, 2048, tokens=64)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for tokens in (1, 4, 16, 64):
        stream = torch.randn(tokens, 8192, generator=gen, device="cuda")
        x, _ = symar.norm(stream.bfloat16(), before=block.before)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                y, new = block(x, stream)
                x.copy_(y), stream.copy_(new)
        torch.cuda.synchronize()
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(3):
            graph.replay()
        start.record()
        for _ in range(32):
            graph.replay()
        stop.record()
        torch.cuda.synchronize()
        block.check()
        used = int(block.routes.choice.unique().numel())
        print(f"{tokens} tokens, {used} experts: {start.elapsed_time(stop) / 32 * 1e3:.1f} us per step of the block")


if __name__ == "__main__":
    main()
