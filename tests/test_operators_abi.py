"""Operators around a decoder layer's AllReduces: what the library refuses, which it does on the host, so none of this
needs a GPU (no call gets as far as a launch)."""
import ctypes

import pytest

from paper_2607_16100_b200 import build, symar

SOME = 1 << 20          # an aligned address that is never touched


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    return symar.load()


def linear_args(**change):
    f = dict(x=SOME, x_ld=64, x_group=0, w=SOME, w_ld=64, w_group=0, bias=None, bias_group=0, residual=None, residual_ld=0,
             residual_group=0, out=SOME, out_ld=32, out_group=0, groups=1, m=4, n=32, k=64, out_dtype=symar.BF16, act=0,
             root=-1)
    f.update(change)
    return ctypes.byref(symar.LinearArgs(**f))


@pytest.mark.parametrize("change", [
    dict(x=None), dict(w=None), dict(out=None), dict(m=-1), dict(n=-1), dict(k=-1), dict(groups=-1), dict(act=5), dict(act=-1),
    dict(out_dtype=2), dict(root=1), dict(root=-2), dict(x=SOME + 1), dict(w=SOME + 1), dict(bias=SOME + 1), dict(out=SOME + 1),
    dict(out=SOME + 2, out_dtype=symar.F32), dict(residual=SOME + 1), dict(groups=2, out_group=0), dict(out_ld=31), dict(x_ld=-64), dict(w_ld=-64),
    dict(x_group=-1), dict(w_group=-1), dict(bias_group=-1), dict(residual_ld=-1), dict(residual_group=-1), dict(out_group=-1),
], ids=lambda c: ",".join(f"{k}={v}" for k, v in c.items()))
def test_linear_refuses(lib, change):
    assert lib.symar_linear(linear_args(**change), None) == symar.ERR_INVAL


def test_linear_without_work_needs_no_pointers(lib):
    assert lib.symar_linear(None, None) == symar.ERR_INVAL
    for empty in ("m", "n", "groups"):
        assert lib.symar_linear(linear_args(**{empty: 0, "x": None, "w": None, "out": None}), None) == symar.OK


def test_page_bytes(lib):
    for heads in (1, 3, 8):
        for dim in (64, 128, 256):
            for page in (16, 32, 64, 128, 256):
                # codes: half a byte a channel; one word per 64 channels; keys and values
                assert lib.symar_kv_page_bytes(heads, dim, page) == heads * page * 2 * (dim // 2 + 4 * (dim // 64))
    for bad in ((0, 128, 64), (1, 96, 64), (1, 128, 48), (1, 128, 8), (1, 128, 512), (-1, 128, 64), (1, 0, 64), (1, 512, 64)):
        assert lib.symar_kv_page_bytes(*bad) == 0


def fake_context(lib):
    """The checks come before the first use of the context, so any address stands for one."""
    return ctypes.c_void_p(ctypes.addressof(fake_context.room))


fake_context.room = ctypes.create_string_buffer(4096)


def call(lib, which, cache=None, batch=None, args=None, kv=True):
    c = dict(pages=SOME, num_pages=4, kv_heads=2, head_dim=128, page_size=16)
    b = dict(lengths=SOME, token_start=None, page_table=SOME, table_ld=4, seqs=3, tokens=3)
    row = dict(zip(("", "_ld", "_head"), (SOME, 512, 128)))
    a = {"append": {**{n + s: v for n in ("q", "q_out", "k", "v") for s, v in row.items()},
                    "rotations": SOME, "rotation_rows": 64, "rot_dim": 128, "interleaved": 0, "q_heads": 4, "dtype": 1},
         "read": {**{n + s: v for n in ("k", "v") for s, v in row.items()}, "dtype": 1},
         "attention": {**{n + s: v for n in ("q", "out") for s, v in row.items()}, "scale": 0.0, "q_heads": 4, "window": 0,
                       "dtype": 1}}[which]
    kind = {"append": symar.KVAppendArgs, "read": symar.KVReadArgs, "attention": symar.KVAttentionArgs}[which]
    c.update(cache or {}), b.update(batch or {}), a.update(args or {})
    return getattr(lib, "symar_kv_" + which)(fake_context(lib) if kv else None, ctypes.byref(symar.KVCacheArgs(**c)),
                                             ctypes.byref(symar.KVBatchArgs(**b)), ctypes.byref(kind(**a)), None)


@pytest.mark.parametrize("which", ["append", "read", "attention"])
def test_cache_calls_refuse(lib, which):
    assert call(lib, which, kv=False) == symar.ERR_INVAL
    for bad in (dict(pages=None), dict(pages=SOME + 8), dict(num_pages=0)):
        assert call(lib, which, cache=bad) == symar.ERR_INVAL, bad
    for bad in (dict(head_dim=96), dict(page_size=24), dict(kv_heads=0)):
        assert call(lib, which, cache=bad) == symar.ERR_UNSUPPORTED, bad
    for bad in (dict(lengths=None), dict(page_table=None), dict(seqs=-1), dict(tokens=-1), dict(tokens=4), dict(table_ld=-1),
                dict(lengths=SOME + 2), dict(token_start=SOME + 1), dict(seqs=0)):
        assert call(lib, which, batch=bad) == symar.ERR_INVAL, bad
    assert call(lib, which, batch=dict(seqs=symar.KV_MAX_SEQS + 1, tokens=symar.KV_MAX_SEQS + 1)) == symar.ERR_UNSUPPORTED
    assert call(lib, which, args=dict(dtype=2)) == symar.ERR_INVAL
    assert call(lib, which, batch=dict(seqs=0, tokens=0, lengths=None, page_table=None)) == symar.OK


def test_append_refuses(lib):
    for bad in (dict(k=None), dict(v=None), dict(q_out=None), dict(rot_dim=127), dict(rot_dim=130), dict(rot_dim=0),
                dict(interleaved=2), dict(q_heads=-1), dict(rotations=SOME + 4), dict(rotation_rows=-1), dict(k=SOME + 1),
                dict(dtype=0, v=SOME + 2)):
        assert call(lib, "append", args=bad) == symar.ERR_INVAL, bad


def test_attention_refuses(lib):
    for bad in (dict(q=None), dict(out=None), dict(q_heads=3), dict(q_heads=0), dict(window=-1), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(q=SOME + 1)):
        assert call(lib, "attention", args=bad) == symar.ERR_INVAL, bad
    assert call(lib, "attention", args=dict(dtype=symar.F32)) == symar.ERR_UNSUPPORTED


@pytest.mark.parametrize("which,reads,writes", [("append", "q k v", "q_out"), ("read", "", "k v"), ("attention", "q", "out")])
def test_strides_refused(lib, which, reads, writes):
    for name in reads.split() + writes.split():
        for bad in ({name + "_ld": -512}, {name + "_head": -128}):
            assert call(lib, which, args=bad) == symar.ERR_INVAL, bad
    for name in writes.split():                              # rows that would be written over one another
        for bad in ({name + "_ld": 0}, {name + "_ld": 127}, {name + "_head": 0}, {name + "_head": 120}):
            assert call(lib, which, args=bad) == symar.ERR_INVAL, bad


def test_rope_table_refuses(lib):
    def rc(rows=16, table=SOME, **change):
        f = dict(base=1e4, factor=2.0, original=64.0, low=1.0, high=4.0, magnitude=1.0, kind=0, rot_dim=64)
        f.update(change)
        return lib.symar_rope_table(table, rows, ctypes.byref(symar.RopeScaling(**f)), None)
    for bad in (dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=258), dict(base=0.0), dict(kind=4), dict(kind=-1), dict(rows=-1),
                dict(table=None), dict(table=SOME + 4), dict(kind=1, factor=0.0), dict(kind=3, original=0.0),
                dict(kind=3, high=1.0), dict(kind=2, rot_dim=2)):
        assert rc(**bad) == symar.ERR_INVAL, bad
    assert lib.symar_rope_table(SOME, 4, None, None) == symar.ERR_INVAL
    assert rc(rows=0, table=None) == symar.OK


def test_context_refuses(lib):
    h = ctypes.c_void_p()
    need = lib.symar_kv_required_bytes()
    assert need > 0
    assert lib.symar_kv_create(None) == symar.ERR_INVAL
    assert lib.symar_kv_create_on(ctypes.byref(h), None, need) == symar.ERR_INVAL
    assert lib.symar_kv_create_on(ctypes.byref(h), SOME + 16, need) == symar.ERR_INVAL
    assert lib.symar_kv_create_on(ctypes.byref(h), SOME, need - 1) == symar.ERR_NOMEM
    assert lib.symar_kv_destroy(None) == symar.ERR_INVAL
    assert lib.symar_kv_reset(None, None) == symar.ERR_INVAL
    assert lib.symar_kv_status(None, None, None, None) == symar.ERR_INVAL
    assert not h
