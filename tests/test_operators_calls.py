"""The Python calls of the operators, without a GPU: which stream, device and memory they name to the library.  A stand-in for the library
takes their arguments; tensors are torch's CPU ones, whose device index is -1."""
import contextlib
import types

import pytest
import torch

from paper_2607_16100_b200 import symar


class Library:
    """Every function returns OK and notes its name and arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def fn(*args):
            self.calls.append((name, args))
            return symar.OK
        return fn


@pytest.fixture()
def lib(monkeypatch):
    symar._torch()
    lib = Library()
    monkeypatch.setattr(symar, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(symar, "_device", lambda: -1)
    monkeypatch.setattr(symar, "_lib", lib)
    return lib


@contextlib.contextmanager
def noted(log, index):
    log.append(index)
    yield


def context(lib, index=-1, keepalive=None):
    c = object.__new__(symar.KVContext)
    c._lib, c._h, c._keepalive, c.index = lib, 77, keepalive, index
    return c


def test_reset_and_status_follow_the_current_stream_and_the_contexts_device(lib, monkeypatch):
    entered = []
    monkeypatch.setattr(torch.cuda, "device", lambda index: noted(entered, index))
    c = context(lib, index=3)
    c.reset()
    assert lib.calls == [("symar_kv_reset", (77, 1003))] and entered == [3]
    c.reset(5)
    assert lib.calls[-1] == ("symar_kv_reset", (77, 5)) and entered == [3, 3]
    assert c.status() == (0, 0, 0)
    assert lib.calls[-1][0] == "symar_kv_status" and entered == [3, 3, 3]
    c._h = None


def test_torchs_memory_is_kept_until_no_kernel_uses_it(lib, monkeypatch):
    """The allocator knows nothing of the streams that the context's calls ran on."""
    capturing, log = [False], []

    class Memory:
        def __del__(self):
            log.append("freed")

    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    monkeypatch.setattr(torch.cuda, "synchronize", lambda index: log.append(("waited", index)))
    context(lib, 2, Memory()).destroy()
    assert lib.calls == [("symar_kv_destroy", (77,))] and log == [("waited", 2), "freed"]
    log.clear()
    capturing[0] = True                                          # where nothing may wait: by the next that may
    context(lib, 2, Memory()).destroy()
    assert log == []
    capturing[0] = False
    context(lib, 2, None).destroy()                              # (memory of the library's own: cudaFree waits)
    assert log == []
    context(lib, 1, Memory()).destroy()
    assert log == [("waited", 1), ("waited", 2), "freed", "freed"]


def setting(index=-1):
    """A cache of two heads and a batch of three tokens, as the calls see them."""
    cache = object.__new__(symar.PagedKV)
    cache.pages, cache.head_dim, cache.page_size, cache.kv_heads = torch.empty(4, 2, 2304, dtype=torch.uint8), 128, 16, 2
    cache.index, cache.args = index, symar.KVCacheArgs(0, 4, 2, 128, 16)
    cache.ref = cache.args
    batch = object.__new__(symar.KVBatch)
    batch.index, batch._fields, batch._last = index, (0, None, 0, 4, 3), (None, None)
    return cache, batch, torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 4, 128, dtype=torch.bfloat16)


def test_results_come_from_the_memory_of_the_stream_that_is_named(lib, monkeypatch):
    entered = []
    monkeypatch.setattr(torch.cuda, "stream", lambda s: noted(entered, s))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: (handle, device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda index: (0, index))
    cache, batch, k, q = setting()
    c = context(lib)
    for stream, want in ((None, []), (999, []), (5, [(5, -1)]), (0, [(0, -1)])):          # 999: the current one
        for call, results in ((lambda: c.append(cache, batch, k, k, q=q, stream=stream), 1),
                              (lambda: c.read(cache, batch, 3, stream=stream), 2),
                              (lambda: c.attention(cache, batch, q, stream=stream), 1)):
            entered.clear()
            call()
            assert entered == want * results
            assert lib.calls[-1][1][-1] == (999 if stream is None else stream)
        entered.clear()
        c.append(cache, batch, k, k, q=q, q_out=q, stream=stream)
        c.attention(cache, batch, q, out=q, stream=stream)
        assert entered == []
    c._h = None


def test_a_batch_may_be_shared_by_threads(lib):
    """What one call hands to the library stays as it was while another is made with more rows."""
    cache, batch, _, _ = setting()
    c = context(lib)
    for tokens in (3, 7, 7, 0, 3):
        c.read(cache, batch, tokens)
    handed = [args[2] for name, args in lib.calls]
    assert [h._obj.tokens for h in handed] == [3, 7, 7, 0, 3]
    assert all(h._obj.seqs == 3 and h._obj.table_ld == 4 for h in handed)
    assert handed[1] is handed[2]                                # (a loop's calls make it once)
    c._h = None


@pytest.mark.parametrize("of_context,of_cache,of_batch", [(0, -1, -1), (-1, 0, -1), (-1, -1, 0), (1, 1, 0), (0, 1, 1)])
def test_context_cache_and_batch_are_of_one_device(lib, of_context, of_cache, of_batch):
    cache, batch, k, q = setting()
    c = context(lib, of_context)
    cache.index, batch.index = of_cache, of_batch
    for call in (lambda: c.append(cache, batch, k, k, q=q), lambda: c.read(cache, batch, 3), lambda: c.attention(cache, batch, q)):
        with pytest.raises(symar.SymarError, match="device"):
            call()
    assert lib.calls == []
    c._h = None


def test_tensors_of_other_dimensions_are_refused(lib):
    cache, batch, k, q = setting()
    c = context(lib)
    for call in (lambda t: c.append(cache, batch, t, k), lambda t: c.append(cache, batch, k, t), lambda t: c.append(cache, batch, k, k, q=t),
                 lambda t: c.append(cache, batch, k, k, q=q, q_out=t), lambda t: c.attention(cache, batch, t),
                 lambda t: c.attention(cache, batch, q, out=t)):
        for t in (q[0, 0, 0], q[0, 0], q[0], q[None]):
            with pytest.raises(symar.SymarError):
                call(t)
    assert lib.calls == []
    c._h = None


def test_a_table_of_rotations_is_on_a_gpu(lib):
    """(Its address goes to a kernel.)"""
    for device in ("cpu", torch.device("cpu"), "meta"):
        for stream in (None, 5):
            with pytest.raises(symar.SymarError, match="table"):
                symar.rope_table(4, 64, device=device, stream=stream)
    assert lib.calls == []
