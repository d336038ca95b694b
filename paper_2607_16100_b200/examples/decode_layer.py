"""The attention half of a tensor-parallel decoder layer on P emulated ranks, ending in its AllReduce.

One step for a batch of sequences, each with one new token (or, with ``token_start``, with a piece of a prompt):

1. ``symar.linear``      queries, keys and values of all ranks' heads (each rank's columns side by side in one matrix);
2. ``KVContext.append``  rotation, and the new keys and values into the 4-bit paged cache;
3. ``KVContext.attention`` over the cache;
4. ``symar.linear``      the ranks' output projections, one launch, every rank's partial sums written straight into its
                         segment of the symmetric heap; rank 0 carries the residual;
5. ``SymHeap.allreduce`` the sum of the partial sums, on every rank.

(The norms of a layer are left out.)  Run it:  python -m paper_2607_16100_b200.examples.decode_layer
"""
from __future__ import annotations

import torch

from paper_2607_16100_b200 import symar


class AttentionBlock:
    def __init__(self, ranks: int, hidden: int, q_heads: int, kv_heads: int, head_dim: int, *, seqs: int, tokens: int,
                 positions: int, page_size: int = 64, seed: int = 0, device="cuda"):
        if q_heads % ranks:
            raise ValueError("every rank has the same number of query heads")
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape, fan):
            return (torch.randn(*shape, generator=g, device=device) * fan ** -0.5).to(torch.bfloat16)

        self.ranks, self.hidden, self.q_heads, self.kv_heads, self.dim = ranks, hidden, q_heads, kv_heads, head_dim
        self.w_qkv = weight((q_heads + 2 * kv_heads) * head_dim, hidden, fan=hidden)
        mine = q_heads // ranks * head_dim
        self.w_out = weight(ranks, hidden, mine, fan=q_heads * head_dim)
        self.rotations = symar.rope_table(positions, head_dim, base=500000.0, device=device)
        # a page table that gives every sequence room for `positions` tokens
        columns = -(-positions // page_size)
        self.cache = symar.PagedKV.zeros(seqs * columns, kv_heads, head_dim, page_size, device)
        self.page_table = torch.arange(seqs * columns, dtype=torch.int32, device=device).view(seqs, columns)
        self.context = symar.KVContext()
        self.heap = symar.SymHeap.on_torch(ranks, 2 * -(-tokens * hidden * 2 // symar.ALIGN) * symar.ALIGN, device)
        self.out_offset = self.heap.bytes_per_rank // 2
        self.partial = self.heap.view(0, (tokens, hidden), torch.bfloat16)
        self.summed = self.heap.view(self.out_offset, (tokens, hidden), torch.bfloat16)

    def __call__(self, x, lengths, token_start=None):
        """x [tokens, hidden] bf16 and the sequences' lengths with the new tokens; returns [ranks, tokens, hidden]: every rank's result
        (a view of the heap, good until the next call)."""
        tokens, dim = x.shape[0], self.dim
        batch = symar.KVBatch(lengths, self.page_table, token_start)
        qkv = symar.linear(x, self.w_qkv).unflatten(1, (-1, dim))
        q, k, v = qkv.split([self.q_heads, self.kv_heads, self.kv_heads], 1)
        q = self.context.append(self.cache, batch, k, v, q=q, rotations=self.rotations)
        heads = self.context.attention(self.cache, batch, q)
        # each rank's heads of every token: [ranks, tokens, heads of a rank x dim], as strides
        of_ranks = heads.view(tokens, self.ranks, -1).transpose(0, 1)
        symar.linear(of_ranks, self.w_out, residual=x, root=0, out=self.partial[:, :tokens])
        stream = torch.cuda.current_stream().cuda_stream
        self.heap.allreduce(0, self.out_offset, tokens * self.hidden, symar.BF16, symar.AUTO, stream)
        return self.summed[:, :tokens]

    def check(self) -> None:
        """Raises if a call recorded an error on the device (synchronises)."""
        for code, *where in (self.heap.status(), self.context.status()):
            if code != symar.OK:
                raise symar.SymarError(code, f"on the device, at {where}")


def main() -> None:
    # hidden size 8192 over eight ranks, batch 4: the message of one AllReduce is 4 x 16 KiB per rank
    seqs, cached = 4, 4096
    block = AttentionBlock(8, 8192, 64, 8, 128, seqs=seqs, tokens=seqs * 64, positions=cached + 64)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for begin in range(0, cached, 64):              # prompts, 64 tokens of every sequence at a time
        x = torch.randn(seqs * 64, 8192, generator=gen, device="cuda").to(torch.bfloat16)
        lengths = torch.full((seqs,), begin + 64, dtype=torch.int32, device="cuda")
        block(x, lengths, torch.arange(0, seqs * 64 + 1, 64, dtype=torch.int32, device="cuda"))
    x = torch.randn(seqs, 8192, generator=gen, device="cuda").to(torch.bfloat16)
    lengths = torch.full((seqs,), cached, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):   # one token of every sequence
            lengths += 1
            y = block(x, lengths)
            x.copy_(y[0])
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
    print(f"{seqs} sequences, {int(lengths[0])} tokens each: {start.elapsed_time(stop) / 32 * 1e3:.1f} us per step of the block")


if __name__ == "__main__":
    main()
