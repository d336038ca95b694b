"""The status word of symar.norm: cleared by every call, whatever kernel it takes, and refused where it is no word."""
import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n", [(1, 8192), (700, 1024), (601, 9000), (5000, 128), (5000, 130), (30, 2049), (0, 64), (4, 0)])
def test_every_call_clears_it(m, n):
    x = torch.randn(m, n, device="cuda").bfloat16()
    norm = symar.Norm("rms")
    word = torch.full((3,), 9, dtype=torch.int32, device="cuda")
    want = symar.norm(x, x, before=norm)
    got = symar.norm(x, x, before=norm, status=word[1:2])
    assert word.tolist() == [9, symar.OK, 9] and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y, _ = symar.norm(x, x, before=norm, status=word[1:2])
    for _ in range(2):
        word.fill_(9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert word.tolist() == [9, symar.OK, 9] and torch.equal(y, want[0])


def test_refusals():
    x = torch.randn(4, 64, device="cuda")
    word = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (word, word[:1].float(), word[:1].cpu(), word[:0]):
        with pytest.raises(symar.SymarError):
            symar.norm(x, before=symar.Norm(), status=bad)
