"""The warps of symar_experts that hand out results read tensor memory and meet at barriers as whole warps: every wait of theirs is one for all lanes, and lanes come
together before a barrier.  (By the source: nothing that a test could run on a device shows it.)"""
from paper_2607_16100_b200 import build

TEXT = (build.CSRC / "symar_experts.cu").read_text()


def part(text, begin, end):
    at = text.index(begin)
    return text[at:text.index(end, at)]


def test_waits_are_of_whole_warps():
    kernels = TEXT[TEXT.index("experts_kernel(const"):]
    for results in (part(kernels, "// ---- results ----", "done:"), part(kernels, "// ---- results: this block's", "done:")):
        waits = [w for w in ("bar_wait(", "pair_wait(", "warp_wait(", "pair_warp_wait(") if w in results]
        assert waits
        single = results.replace("pair_warp_wait(", "").replace("warp_wait(", "")
        assert "pair_wait(" not in single and "bar_wait(" not in single
    wait = part(TEXT, "bool pair_warp_wait(", "\n}\n")
    assert "__all_sync(0xffffffffu, pair_try(" in wait and "__any_sync(0xffffffffu, *failed" in wait


def test_lanes_come_together_before_a_barrier():
    """Behind a loop in which halves of a warp may have different numbers of tokens."""
    loops = TEXT.split("(a.gated ? lane >> 4 : 0); i < ")[1:]
    assert len(loops) == 2
    for loop in loops:
        assert loop.index("__syncwarp();") < loop.index("results_sync();")


def test_nothing_is_sent_or_expected_once_a_wait_gave_up():
    """A barrier whose phase never ended takes no other arrival, and other blocks' memory no more parts."""
    results = part(TEXT[TEXT.index("experts_kernel(const"):], "// ---- results ----", "done:")
    assert results.count("bar_expect(") == 1 and results.count("if (tid == 128 && whole) bar_expect(parts_here") == 1
    assert results.count("far_store(") == 1 and "if (token >= t.count || !whole) break;" in results
    loop = results[:results.rindex("pair_warp_wait(")]               # (behind the last tile nothing follows)
    assert loop.count("pair_warp_wait(") == loop.count("whole &= pair_warp_wait(") == 2
