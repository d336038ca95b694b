"""The Python calls of the operators on a GPU: streams, memory and status words that they take or make by themselves."""
import os
import subprocess
import sys
from pathlib import Path

import pytest
import torch

from paper_2607_16100_b200 import symar
from test_kv_gpu import Setup, normal

pytestmark = pytest.mark.gpu


def test_reset_is_one_of_the_streams_calls():
    """Captured between a call that records an offence and one that does not, on a side stream, with no stream named anywhere."""
    c = symar.KVContext.on_torch()
    s = Setup([(1, 40), (1, 20)], 1, 128, 16, seed=7)
    s.fill(c, seed=71)
    q = normal(2, 8, 128, seed=1)
    want = c.attention(s.cache, s.batch, q)
    table = s.table.clone()
    table[1, 1] = -1
    bad = symar.KVBatch(s.lengths, table)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(q)
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        c.attention(s.cache, bad, q, out=out)
        c.reset()
        c.attention(s.cache, s.batch, q, out=out)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        assert c.status()[0] == symar.OK
        assert torch.equal(out, want)
    c.attention(s.cache, bad, q)
    assert c.status()[0] == symar.ERR_INVAL
    c.destroy()


def test_a_context_given_back_during_a_capture():
    """Its memory stays as it is until something may wait; the capture goes on."""
    c, other = symar.KVContext.on_torch(), symar.KVContext.on_torch()
    s = Setup([(1, 40)], 1, 128, 16, seed=7)
    s.fill(c, seed=71)
    q = normal(1, 8, 128, seed=1)
    want = c.attention(s.cache, s.batch, q)
    out, graph, side = torch.empty_like(q), torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        other.destroy()
        c.attention(s.cache, s.batch, q, out=out)
    assert len(symar._late) == 1
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    c.destroy()
    assert not symar._late


def stream_of(t):
    """The stream whose pool a tensor's memory is of."""
    at = t.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


def test_results_are_of_the_stream_that_is_named():
    c = symar.KVContext.on_torch()
    s = Setup([(1, 40), (1, 20)], 2, 128, 16, seed=7)
    s.fill(c, seed=71)
    q, k = normal(2, 8, 128, seed=1), normal(2, 2, 128, seed=2)
    x, w = normal(4, 128, seed=3), normal(64, 128, seed=4)
    side = torch.cuda.Stream()
    want = symar.linear(x, w), *c.read(s.cache, s.batch, 2), c.attention(s.cache, s.batch, q), symar.rope_table(9, 64)
    torch.cuda.synchronize()
    for handle, home in ((side.cuda_stream, side), (0, torch.cuda.default_stream())):
        with torch.cuda.stream(torch.cuda.default_stream() if handle else side):         # the other one is current
            got = (symar.linear(x, w, stream=handle), *c.read(s.cache, s.batch, 2, stream=handle),
                   c.attention(s.cache, s.batch, q, stream=handle), symar.rope_table(9, 64, stream=handle))
            turned = c.append(s.cache, s.batch, k, k, q=q, stream=handle)
        torch.cuda.synchronize()
        for t in (*got, turned):
            assert stream_of(t) == home.cuda_stream
        assert all(torch.equal(a, b) for a, b in zip(got[:1] + got[4:], want[:1] + want[4:]))
    assert c.status()[0] == symar.OK
    c.destroy()


def test_a_product_reports_to_the_status_word_it_is_given():
    x, w = normal(4, 128, seed=3), normal(64, 128, seed=4)
    want = symar.linear(x, w)
    words = torch.full((3,), 77, dtype=torch.int32, device="cuda")
    assert torch.equal(symar.linear(x, w, status=words[1]), want)
    assert words.tolist() == [77, symar.OK, 77]
    for a, b in ((x[:0], w), (x, w[:0]), (x[:, :0], w[:, :0])):          # nothing to do is done: a word of an earlier call does not stay
        words.fill_(77)
        symar.linear(a, b, status=words[1])
        assert words.tolist() == [77, symar.OK, 77]
    for bad in (words, words[:0], words[:1].long(), words[:1].cpu(), words[:1].float()):
        with pytest.raises(symar.SymarError):
            symar.linear(x, w, status=bad)


def test_threads_each_with_a_stream_and_a_context():
    """Products need no context; cache calls of two threads share a cache and a batch, and have a context each.  In a process of its own, so
    that the first call that the library sees comes from all threads at once."""
    program = """
import sys, threading
import torch
from paper_2607_16100_b200 import symar
from test_kv_gpu import Setup, normal
n = 6
fill = symar.KVContext.on_torch()
s = Setup([(1, 400), (1, 20), (1, 77)], 2, 128, 16, seed=7)
q, x, w = normal(3, 8, 128, seed=1), normal(33, 328, seed=3), normal(64, 328, seed=4)
s.fill(fill, seed=71)
own = [(torch.cuda.Stream(), symar.KVContext.on_torch()) for _ in range(n)]
torch.cuda.synchronize()
got, gate = [None] * n, threading.Barrier(n)
def work(i):
    stream, c = own[i]
    with torch.cuda.stream(stream):
        gate.wait()
        for _ in range(50):
            got[i] = symar.linear(x, w), c.attention(s.cache, s.batch, q)
        stream.synchronize()
threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
[t.start() for t in threads]
[t.join() for t in threads]
assert all(torch.equal(a, b) for g in got for a, b in zip(g, got[0]))
want = x.double() @ w.double().T
assert ((got[0][0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 328 * 2.0 ** -23 * (x.double().abs() @ w.double().abs().T)).all()
assert torch.equal(got[0][1], fill.attention(s.cache, s.batch, q))
assert all(c.status()[0] == symar.OK for _, c in own)
print("threads agree")
"""
    run = subprocess.run([sys.executable, "-c", program], cwd=Path(__file__).parent, capture_output=True, text=True, timeout=300,
                         env={**os.environ, "PYTHONPATH": str(Path(__file__).parent.parent)})
    assert run.returncode == 0 and "threads agree" in run.stdout, run.stderr[-2000:]
