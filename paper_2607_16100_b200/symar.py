"""ctypes binding of libsymar.so: argument marshalling only.

Function names and argument order follow ``include/symar.h``.  Every step of
the collective runs in the library's CUDA kernels; if the library is missing
or fails to load this module raises -- there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import (POINTER, byref, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_uint,
                    c_void_p)
from pathlib import Path

_PKG = Path(__file__).resolve().parent
# SYMAR_LIB selects another build of the same library (the system-scope or the bounds-checking
# flavour of paper_2607_16100_b200/build.py); by default the regular one.
LIB_PATH = Path(os.environ["SYMAR_LIB"]) if os.environ.get("SYMAR_LIB") else _PKG / "libsymar.so"

F32, BF16 = 0, 1
AUTO, ONESHOT, TWOSHOT, LL, SENTINEL, TWOSHOT_LL, TWOSHOT_SENTINEL, TWOSHOT_ATOMIC = 0, 1, 2, 3, 4, 5, 6, 7
ALGO_NAMES = {AUTO: "auto", ONESHOT: "oneshot", TWOSHOT: "twoshot", LL: "ll", SENTINEL: "sentinel",
              TWOSHOT_LL: "twoshot_ll", TWOSHOT_SENTINEL: "twoshot_sentinel", TWOSHOT_ATOMIC: "twoshot_atomic"}
DTYPE_NAMES = {F32: "f32", BF16: "bf16"}
DTYPE_SIZE = {F32: 4, BF16: 2}

OK, ERR_INVAL, ERR_NOMEM, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED = 0, -1, -2, -3, -4, -5
_ERR_NAMES = {
    ERR_INVAL: "SYMAR_ERR_INVAL", ERR_NOMEM: "SYMAR_ERR_NOMEM", ERR_CUDA: "SYMAR_ERR_CUDA",
    ERR_TIMEOUT: "SYMAR_ERR_TIMEOUT", ERR_UNSUPPORTED: "SYMAR_ERR_UNSUPPORTED",
}

MAX_RANKS, MAX_CTAS, LL_SLOTS, LL_SLOT_VECS, ALIGN = 8, 160, 64, 1024, 8192
VARIANT_CLUSTER = 0x40000000      # SYMAR_VARIANT_CLUSTER: the ranks of a slot launched as one thread-block cluster

# every symbol include/symar.h declares: (name, restype, argtypes)
SIGNATURES = [
    ("symheap_required_bytes", c_size_t, [c_int, c_size_t]),
    ("symheap_create", c_int, [POINTER(c_void_p), c_int, c_size_t]),
    ("symheap_create_on", c_int, [POINTER(c_void_p), c_int, c_size_t, c_void_p, c_size_t]),
    ("symheap_destroy", c_int, [c_void_p]),
    ("symheap_info", c_int, [c_void_p, c_void_p]),
    ("symheap_rank_ptr", c_void_p, [c_void_p, c_int, c_size_t]),
    ("symheap_reset", c_int, [c_void_p, c_void_p]),
    ("symheap_status", c_int, [c_void_p, POINTER(c_int), POINTER(c_int), POINTER(c_int), POINTER(c_int)]),
    ("allreduce", c_int, [c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_int, c_void_p]),
    ("allreduce_host", c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_int,
                               c_void_p]),
    ("symar_reduce_scatter", c_int, [c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_void_p]),
    ("symar_all_gather", c_int, [c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_void_p]),
    ("symar_broadcast", c_int, [c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_int, c_void_p]),
    ("symar_reduce", c_int, [c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_int, c_void_p]),
    ("allreduce_autotune", c_int, [c_void_p, c_int]),
    ("allreduce_autotune_size", c_int, [c_void_p, c_int, c_size_t]),
    ("allreduce_autotune_stream", c_int, [c_void_p, c_int, c_size_t, c_int]),
    ("symar_last_choice", c_int, [c_void_p, POINTER(c_int), POINTER(c_int), POINTER(c_int)]),
    ("symar_last_kernel", c_int, [c_void_p, POINTER(c_uint), POINTER(c_size_t)]),
    ("symar_query_choice", c_int, [c_void_p, c_size_t, c_int, POINTER(c_int), POINTER(c_int), POINTER(c_int)]),
    ("symar_tuned_entry", c_int, [c_void_p, c_int, c_int, c_int, POINTER(c_int), POINTER(c_int),
                                  POINTER(c_double)]),
    ("symar_table_save", c_int, [c_void_p, c_char_p]),
    ("symar_table_load", c_int, [c_void_p, c_char_p]),
    ("symar_set_launch", c_int, [c_void_p, c_int, c_int, c_int]),
    ("symar_set_variant", c_int, [c_void_p, c_int, c_uint]),
    ("symar_set_pdl", c_int, [c_void_p, c_int]),
    ("symar_set_placement", c_int, [c_void_p, c_int]),
    ("symar_placement", c_int, [c_void_p, POINTER(c_int), POINTER(c_int), POINTER(ctypes.c_ulonglong)]),
    ("symar_set_scratch_limit", c_int, [c_void_p, c_size_t]),
    ("symar_set_spin_limit_us", c_int, [c_void_p, c_uint]),
    ("symar_debug_inject", c_int, [c_void_p, c_int, c_uint, c_uint]),
    ("allreduce_static", c_int, [c_void_p, c_void_p, c_size_t, c_int, c_size_t, c_int, c_void_p, c_void_p]),
    ("symar_last_cuda_error", c_char_p, []),
    ("symar_probe_empty", c_int, [c_int, c_int, c_int, c_void_p]),
    ("symar_probe_empty_pdl", c_int, [c_int, c_int, c_int, c_void_p]),
    ("symar_probe_empty_cluster", c_int, [c_int, c_int, c_int, c_void_p]),
    ("symar_probe_fence", c_int, [c_int, POINTER(c_double)]),
    ("symar_probe_pingpong", c_int, [c_int, POINTER(c_double)]),
    ("symar_probe_pingpong_pair", c_int, [c_int, c_int, POINTER(c_double), POINTER(c_int)]),
    ("symar_debug_span", c_int, [c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_int, c_void_p, POINTER(c_double)]),
    ("symar_debug_phases", c_int, [c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_int, c_void_p, POINTER(c_double),
                                   POINTER(c_int)]),
    ("symar_check_selftest", c_int, [c_void_p, c_void_p]),
    ("symar_probe_barrier", c_int, [c_int, c_int, c_int, POINTER(c_double)]),
    ("symar_llbuffer_bytes", c_size_t, [c_int, c_size_t, c_size_t, c_int, c_int]),
    ("symar_llbuffer_init_sentinel", c_int, [c_void_p, c_size_t, c_void_p]),
    ("symar_linear", c_int, [c_void_p, c_void_p]),
    ("symar_kv_required_bytes", c_size_t, []),
    ("symar_kv_create", c_int, [POINTER(c_void_p)]),
    ("symar_kv_create_on", c_int, [POINTER(c_void_p), c_void_p, c_size_t]),
    ("symar_kv_destroy", c_int, [c_void_p]),
    ("symar_kv_reset", c_int, [c_void_p, c_void_p]),
    ("symar_kv_status", c_int, [c_void_p, POINTER(c_int), POINTER(c_int), POINTER(c_int)]),
    ("symar_kv_page_bytes", c_size_t, [c_int, c_int, c_int]),
    ("symar_rope_table", c_int, [c_void_p, c_int64, c_void_p, c_void_p]),
    ("symar_kv_append", c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    ("symar_kv_read", c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    ("symar_kv_attention", c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    ("symar_probe_pingpong_blocks", c_int, [c_int, c_int, c_int, c_int, POINTER(c_double), POINTER(c_int)]),
]


class SymarError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        detail = ""
        if code == ERR_CUDA and _lib is not None:
            detail = ": " + (_lib.symar_last_cuda_error() or b"").decode()
        super().__init__(f"{where} -> {_ERR_NAMES.get(code, code)}{detail}")


class HeapInfo(ctypes.Structure):
    _fields_ = [
        ("P", c_int), ("bytes_per_rank", c_size_t), ("user_bytes", c_size_t),
        ("ll_scratch_bytes", c_size_t), ("sentinel_scratch_bytes", c_size_t), ("atomic_scratch_bytes", c_size_t),
        ("flag_bytes", c_size_t),
        ("stride", c_size_t),
        ("total_bytes", c_size_t), ("base", c_void_p),
    ]


_lib = None


def load() -> ctypes.CDLL:
    """dlopen the library and declare every signature.  Raises if it is absent."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise ImportError(
                f"{LIB_PATH} not found: build it with `python -m paper_2607_16100_b200.build` "
                "(there is no non-CUDA path)")
        lib = ctypes.CDLL(str(LIB_PATH))
        for name, res, args in SIGNATURES:
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _ck(rc: int, where: str) -> None:
    if rc != OK:
        raise SymarError(rc, where)


def required_bytes(P: int, bytes_per_rank: int) -> int:
    return int(load().symheap_required_bytes(P, bytes_per_rank))


class SymHeap:
    """Owner of one ``symheap_t``.  ``device_mem`` (an int address) + ``device_bytes``
    place the heap in caller memory (``symheap_create_on``); otherwise the library
    allocates (``symheap_create``)."""

    def __init__(self, P: int, bytes_per_rank: int, device_mem: int | None = None,
                 device_bytes: int = 0, keepalive=None):
        self._lib = load()
        self._h = c_void_p()
        self._keepalive = keepalive
        if device_mem is None:
            _ck(self._lib.symheap_create(byref(self._h), P, bytes_per_rank), "symheap_create")
        else:
            _ck(self._lib.symheap_create_on(byref(self._h), P, bytes_per_rank, device_mem, device_bytes),
                "symheap_create_on")
        self.P = P
        self.bytes_per_rank = bytes_per_rank
        i = self.info()
        self.base = int(i.base)
        self.stride = int(i.stride)

    @classmethod
    def on_torch(cls, P: int, bytes_per_rank: int, device="cuda:0") -> "SymHeap":
        """Heap in a torch uint8 tensor (PyTorch provides the device memory)."""
        import torch
        n = required_bytes(P, bytes_per_rank)
        buf = torch.empty(n + ALIGN, dtype=torch.uint8, device=device)
        addr = (buf.data_ptr() + ALIGN - 1) // ALIGN * ALIGN
        with torch.cuda.device(buf.device):
            return cls(P, bytes_per_rank, addr, n, keepalive=buf)

    # -- lifetime --
    def destroy(self) -> None:
        if self._h:
            self._lib.symheap_destroy(self._h)
            self._h = c_void_p()
            self._keepalive = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # -- layout --
    def info(self) -> HeapInfo:
        i = HeapInfo()
        _ck(self._lib.symheap_info(self._h, byref(i)), "symheap_info")
        return i

    def rank_ptr(self, rank: int, offset: int = 0) -> int:
        p = self._lib.symheap_rank_ptr(self._h, rank, offset)
        if not p:
            raise SymarError(ERR_INVAL, "symheap_rank_ptr")
        return int(p)

    def reset(self, stream: int = 0) -> None:
        _ck(self._lib.symheap_reset(self._h, stream), "symheap_reset")

    def status(self):
        code, rank, peer, cta = c_int(), c_int(), c_int(), c_int()
        _ck(self._lib.symheap_status(self._h, byref(code), byref(rank), byref(peer), byref(cta)),
            "symheap_status")
        return code.value, rank.value, peer.value, cta.value

    # -- the collective --
    def allreduce_rc(self, in_off: int, out_off: int, count: int, dtype: int, algo: int = AUTO,
                     stream: int = 0) -> int:
        """Raw status code; offsets are turned into rank-0 symmetric addresses."""
        base = self.base
        return int(self._lib.allreduce(self._h, base + in_off, base + out_off, count, dtype, algo, stream))

    def allreduce(self, in_off: int, out_off: int, count: int, dtype: int, algo: int = AUTO,
                  stream: int = 0) -> None:
        _ck(self.allreduce_rc(in_off, out_off, count, dtype, algo, stream), "allreduce")

    def allreduce_ptr(self, in_ptr: int, out_ptr: int, count: int, dtype: int, algo: int = AUTO,
                      stream: int = 0) -> None:
        _ck(self._lib.allreduce(self._h, in_ptr, out_ptr, count, dtype, algo, stream), "allreduce")

    def allreduce_host(self, host_in: int, host_out: int, in_off: int, out_off: int, count: int,
                       dtype: int, algo: int = AUTO, stream: int = 0) -> None:
        base = self.base
        _ck(self._lib.allreduce_host(self._h, host_in, host_out, base + in_off, base + out_off, count,
                                     dtype, algo, stream), "allreduce_host")

    # -- sibling collectives (raw status codes; offsets become rank-0 symmetric addresses) --
    def reduce_scatter(self, in_off, out_off, recv_count, dtype, stream=0) -> int:
        return int(self._lib.symar_reduce_scatter(self._h, self.base + in_off, self.base + out_off, recv_count,
                                                  dtype, stream))

    def all_gather(self, in_off, out_off, send_count, dtype, stream=0) -> int:
        return int(self._lib.symar_all_gather(self._h, self.base + in_off, self.base + out_off, send_count,
                                              dtype, stream))

    def broadcast(self, in_off, out_off, count, dtype, root, stream=0) -> int:
        return int(self._lib.symar_broadcast(self._h, self.base + in_off, self.base + out_off, count, dtype,
                                             root, stream))

    def reduce(self, in_off, out_off, count, dtype, root, stream=0) -> int:
        return int(self._lib.symar_reduce(self._h, self.base + in_off, self.base + out_off, count, dtype, root,
                                          stream))

    # -- data movement helpers for heaps that live in a torch tensor --
    def _bytes_view(self, rank: int, offset: int, nbytes: int):
        if self._keepalive is None:
            raise RuntimeError("heap does not live in a torch tensor (use SymHeap.on_torch)")
        if not (0 <= rank < self.P) or offset < 0 or offset + nbytes > self.bytes_per_rank:
            raise SymarError(ERR_INVAL, "rank/offset/size outside the user region")
        start = self.base + rank * self.stride + offset - self._keepalive.data_ptr()
        return self._keepalive[start:start + nbytes]

    def view(self, offset: int, shape, dtype):
        """torch tensor [P, *shape] of every rank's user region from byte ``offset`` on (no copy)."""
        size = dtype.itemsize
        n = 1
        for d in shape:
            n *= d
        self._bytes_view(0, offset, n * size)                   # range check
        if offset % size:
            raise SymarError(ERR_INVAL, "SymHeap.view: offset")
        start = self.base + offset - self._keepalive.data_ptr()
        flat = self._keepalive[start:start + (self.P - 1) * self.stride + n * size].view(dtype)
        inner = [1] * len(shape)
        for i in range(len(shape) - 2, -1, -1):
            inner[i] = inner[i + 1] * shape[i + 1]
        return flat.as_strided((self.P, *shape), (self.stride // size, *inner))

    def write_rank(self, rank: int, offset: int, array) -> None:
        """Copy a host numpy array into rank ``rank``'s user region at ``offset``."""
        import numpy as np
        import torch
        a = np.ascontiguousarray(array)
        src = torch.from_numpy(a.view(np.uint8).reshape(-1))
        self._bytes_view(rank, offset, a.nbytes).copy_(src, non_blocking=False)

    def read_rank(self, rank: int, offset: int, count: int, np_dtype):
        """Copy ``count`` elements of ``np_dtype`` from rank ``rank``'s user region to the host."""
        import numpy as np
        n = count * np.dtype(np_dtype).itemsize
        return self._bytes_view(rank, offset, n).cpu().numpy().view(np_dtype).copy()

    def fill_user(self, byte: int) -> None:
        """Fill every rank's user region with one byte value (poison before a test)."""
        for q in range(self.P):
            self._bytes_view(q, 0, self.bytes_per_rank).fill_(byte)

    # -- selector --
    def autotune(self, dtype: int) -> None:
        _ck(self._lib.allreduce_autotune(self._h, dtype), "allreduce_autotune")

    def autotune_size(self, dtype: int, count: int) -> None:
        _ck(self._lib.allreduce_autotune_size(self._h, dtype, count), "allreduce_autotune_size")

    def autotune_stream(self, dtype: int, count: int, calls: int) -> None:
        _ck(self._lib.allreduce_autotune_stream(self._h, dtype, count, calls), "allreduce_autotune_stream")

    def last_choice(self):
        a, c, t = c_int(), c_int(), c_int()
        _ck(self._lib.symar_last_choice(self._h, byref(a), byref(c), byref(t)), "symar_last_choice")
        return a.value, c.value, t.value

    def last_kernel(self):
        v, sm = c_uint(), c_size_t()
        _ck(self._lib.symar_last_kernel(self._h, byref(v), byref(sm)), "symar_last_kernel")
        return v.value, sm.value

    def query_choice(self, count: int, dtype: int, algo: int = AUTO):
        a, c, t = c_int(algo), c_int(), c_int()
        _ck(self._lib.symar_query_choice(self._h, count, dtype, byref(a), byref(c), byref(t)),
            "symar_query_choice")
        return a.value, c.value, t.value

    def tuned_entry(self, dtype: int, log2_bytes: int, algo: int):
        c, t, us = c_int(), c_int(), c_double()
        rc = self._lib.symar_tuned_entry(self._h, dtype, log2_bytes, algo, byref(c), byref(t), byref(us))
        if rc != OK:
            return None
        return c.value, t.value, us.value

    def table_save(self, path: str) -> None:
        _ck(self._lib.symar_table_save(self._h, str(path).encode()), "symar_table_save")

    def table_load(self, path: str) -> None:
        _ck(self._lib.symar_table_load(self._h, str(path).encode()), "symar_table_load")

    def set_launch(self, algo: int, ctas_per_rank: int, threads: int) -> None:
        _ck(self._lib.symar_set_launch(self._h, algo, ctas_per_rank, threads), "symar_set_launch")

    def set_variant(self, algo: int, variant: int) -> None:
        _ck(self._lib.symar_set_variant(self._h, algo, variant), "symar_set_variant")

    def set_pdl(self, enabled: bool) -> None:
        _ck(self._lib.symar_set_pdl(self._h, 1 if enabled else 0), "symar_set_pdl")

    def set_placement(self, enabled: bool) -> None:
        _ck(self._lib.symar_set_placement(self._h, 1 if enabled else 0), "symar_set_placement")

    def placement(self):
        """(measured cleanly?, SMs on the second L2 half, home bits)"""
        m, n, hb = c_int(), c_int(), ctypes.c_ulonglong()
        _ck(self._lib.symar_placement(self._h, byref(m), byref(n), byref(hb)), "symar_placement")
        return bool(m.value), n.value, hb.value

    def set_scratch_limit(self, payload_bytes_per_iteration: int) -> None:
        _ck(self._lib.symar_set_scratch_limit(self._h, payload_bytes_per_iteration), "symar_set_scratch_limit")

    def set_spin_limit_us(self, us: int) -> None:
        _ck(self._lib.symar_set_spin_limit_us(self._h, us), "symar_set_spin_limit_us")

    def debug_span(self, in_off: int, out_off: int, count: int, dtype: int, algo: int = AUTO, stream: int = 0) -> float:
        """In-kernel span in ns (first CTA in -> last CTA out) of one synchronous call."""
        v = c_double()
        _ck(self._lib.symar_debug_span(self._h, self.rank_ptr(0, in_off), self.rank_ptr(0, out_off), count, dtype,
                                       algo, stream, byref(v)), "symar_debug_span")
        return v.value

    def debug_phases(self, in_off: int, out_off: int, count: int, dtype: int, algo: int = AUTO, stream: int = 0):
        """Per phase k = 0..7 of one synchronous call: (earliest, mean, latest) ns since the first CTA's
        start, and how many CTAs stamped it; phases the kernel does not have are left out."""
        ns = (c_double * 24)()
        n = (c_int * 8)()
        _ck(self._lib.symar_debug_phases(self._h, self.rank_ptr(0, in_off), self.rank_ptr(0, out_off), count, dtype,
                                         algo, stream, ns, n), "symar_debug_phases")
        return {k: {"first": ns[3 * k], "mean": ns[3 * k + 1], "last": ns[3 * k + 2], "ctas": n[k]}
                for k in range(8) if n[k] > 0}

    def check_selftest(self, stream: int = 0) -> int:
        """Raw status of the bounds-checking build's self-test (ERR_UNSUPPORTED in the regular build)."""
        return int(self._lib.symar_check_selftest(self._h, stream))

    def debug_inject(self, mute_rank: int = -1, delay_seed: int = 0, delay_max_ns: int = 0) -> None:
        _ck(self._lib.symar_debug_inject(self._h, mute_rank, delay_seed, delay_max_ns), "symar_debug_inject")


STATIC_MAX_BYTES = 32768


def allreduce_static(in_ptr: int, out_ptr: int, rank_pitch_bytes: int, P: int, count: int, dtype: int,
                     status_ptr: int = 0, stream: int = 0) -> int:
    """AllReduce on plain device buffers with library-internal static scratch; the
    library allocates nothing.  Returns the raw status code."""
    return int(load().allreduce_static(in_ptr, out_ptr, rank_pitch_bytes, P, count, dtype,
                                       status_ptr or None, stream))


# -- operators between the AllReduces of a decoder layer --
#
# These take torch tensors (device memory, strides, dtypes and the current stream); everything is computed in the
# library's kernels.  Innermost axes must be contiguous; all other strides are free.
#
# ``stream``: a handle (an int), torch's current stream unless given.  A result that a call makes then comes from that stream's memory, as
# if torch had made it there; tensors of other streams that it reads or writes are to be ready for it, and kept until it is
# done with them (Tensor.record_stream), as with torch's own calls.

ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
ROPE_KINDS = {"plain": 0, "linear": 1, "base": 2, "by_parts": 3}
KV_GROUP, KV_MAX_SEQS = 64, 4096


class LinearArgs(ctypes.Structure):
    _fields_ = [
        ("x", c_void_p), ("x_ld", c_int64), ("x_group", c_int64),
        ("w", c_void_p), ("w_ld", c_int64), ("w_group", c_int64),
        ("bias", c_void_p), ("bias_group", c_int64),
        ("residual", c_void_p), ("residual_ld", c_int64), ("residual_group", c_int64),
        ("out", c_void_p), ("out_ld", c_int64), ("out_group", c_int64),
        ("groups", c_int32), ("m", c_int32), ("n", c_int32), ("k", c_int32),
        ("out_dtype", c_int32), ("act", c_int32), ("root", c_int32), ("status", c_void_p),
    ]


class KVCacheArgs(ctypes.Structure):
    _fields_ = [("pages", c_void_p), ("num_pages", c_int64), ("kv_heads", c_int32), ("head_dim", c_int32),
                ("page_size", c_int32)]


class KVBatchArgs(ctypes.Structure):
    _fields_ = [("lengths", c_void_p), ("token_start", c_void_p), ("page_table", c_void_p), ("table_ld", c_int64),
                ("seqs", c_int32), ("tokens", c_int32)]


class RopeScaling(ctypes.Structure):
    _fields_ = [("base", c_double), ("factor", c_double), ("original", c_double), ("low", c_double), ("high", c_double),
                ("magnitude", c_double), ("kind", c_int32), ("rot_dim", c_int32)]


class KVAppendArgs(ctypes.Structure):
    _fields_ = [
        ("q", c_void_p), ("q_ld", c_int64), ("q_head", c_int64),
        ("q_out", c_void_p), ("q_out_ld", c_int64), ("q_out_head", c_int64),
        ("k", c_void_p), ("k_ld", c_int64), ("k_head", c_int64),
        ("v", c_void_p), ("v_ld", c_int64), ("v_head", c_int64),
        ("rotations", c_void_p), ("rotation_rows", c_int64),
        ("rot_dim", c_int32), ("interleaved", c_int32), ("q_heads", c_int32), ("dtype", c_int32),
    ]


class KVReadArgs(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("k_ld", c_int64), ("k_head", c_int64),
                ("v", c_void_p), ("v_ld", c_int64), ("v_head", c_int64), ("dtype", c_int32)]


class KVAttentionArgs(ctypes.Structure):
    _fields_ = [("q", c_void_p), ("q_ld", c_int64), ("q_head", c_int64),
                ("out", c_void_p), ("out_ld", c_int64), ("out_head", c_int64),
                ("scale", c_float), ("q_heads", c_int32), ("window", c_int32), ("dtype", c_int32)]


_T = None               # torch, once a call needed it
_raw_stream = None      # device index -> handle of torch's current stream
_device = None          # -> index of the current device
_CODES = {}             # torch dtype -> symar_dtype_t
_late = []              # (device index, memory) of contexts that were given back during a capture


def _torch():
    global _T, _raw_stream, _device
    if _T is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
        _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _CODES.update({torch.float32: F32, torch.bfloat16: BF16})
        _T = torch
    return _T


def _dtype_code(dtype, where: str) -> int:
    code = _CODES.get(dtype)
    if code is None:
        raise SymarError(ERR_UNSUPPORTED, f"{where}: dtype {dtype}")
    return code


def _bad(where: str, what: str):
    raise SymarError(ERR_INVAL, f"{where}: {what}")


def _call(fn, where, index: int, stream, *args) -> None:
    """fn(*args, stream) with CUDA device ``index`` current; stream None = torch's current one."""
    if stream is None:
        stream = _raw_stream(index)
    if index == _device():
        rc = fn(*args, stream)
    else:
        with _T.cuda.device(index):
            rc = fn(*args, stream)
    if rc != OK:
        raise SymarError(rc, where)


def _new(like, shape, dtype, index: int, stream):
    """An uninitialised result beside ``like`` where a stream is named, of that stream's pool: nothing that is still queued on
    torch's current stream uses its memory."""
    if stream is None or stream == _raw_stream(index):
        return like.new_empty(shape, dtype=dtype)
    with _T.cuda.stream(_T.cuda.ExternalStream(stream, device=index) if stream else _T.cuda.default_stream(index)):
        return like.new_empty(shape, dtype=dtype)


def linear(x, w, *, bias=None, residual=None, out=None, act: str = "none", root: int = -1, out_dtype=None, status=None,
           stream=None):
    """``act(x @ w.T + bias) + residual`` (``symar_linear``).

    x [m, k] or [groups, m, k] and w [n, k] or [groups, n, k] bfloat16; bias [n] or [groups, n]; residual and the
    result [m, n] or [groups, m, n] of ``out_dtype`` (bfloat16 unless said or given by ``out``).  Operands of two
    dimensions (or expanded ones) are shared by all groups.  ``root``: the one group that adds bias and residual,
    -1 = every group.  ``status``: an int32 CUDA tensor of one element that the call sets, on its stream, to OK or, where a wait
    inside the kernel gave up and the result is incomplete, to ERR_TIMEOUT; without it nothing says so."""
    torch = _T or _torch()
    where = "symar_linear"
    bf16 = torch.bfloat16
    if x.dtype is not bf16 or w.dtype is not bf16 or (bias is not None and bias.dtype is not bf16):
        raise SymarError(ERR_UNSUPPORTED, f"{where}: operands are bfloat16")
    index = x.get_device()
    xsh, wsh, xs, ws = x.shape, w.shape, x.stride(), w.stride()
    xd, wd = len(xsh), len(wsh)
    act_code = ACTS.get(act)
    if index < 0 or xd not in (2, 3) or wd not in (2, 3) or act_code is None:
        _bad(where, "x, w are CUDA tensors of two or three dimensions, act is one of " + ", ".join(ACTS))
    m, k, n = xsh[-2], xsh[-1], wsh[-2]
    if xd == 3 or wd == 3:
        groups = xsh[0] if xd == 3 else wsh[0]
        shape = (groups, m, n)
    else:
        groups, shape = 1, (m, n)
    if out is None:
        out = x.new_empty(shape, dtype=out_dtype or bf16) if stream is None else _new(x, shape, out_dtype or bf16, index, stream)
        os = out.stride()
    else:
        os = out.stride()
        if (out_dtype is not None and out.dtype is not out_dtype) or out.shape != shape or (n > 1 and os[-1] != 1) or \
                out.get_device() != index:
            _bad(where, f"out of shape {tuple(out.shape)}, {out.dtype}")
    if wsh[-1] != k or (wd == 3 and wsh[0] != groups) or w.get_device() != index:
        _bad(where, f"shapes of x {tuple(xsh)} and w {tuple(wsh)}, or not on one device")
    if k > 1 and (xs[-1] != 1 or ws[-1] != 1):
        _bad(where, "the innermost axis is contiguous")
    bp = bg = rp = rl = rg = 0
    if bias is not None:
        if bias.shape not in ((n,), (groups, n)) or (n > 1 and bias.stride(-1) != 1) or bias.get_device() != index:
            _bad(where, f"bias of shape {tuple(bias.shape)}")
        bp, bg = bias.data_ptr(), bias.stride(0) if bias.dim() == 2 else 0
    if residual is not None:
        rs = residual.stride()
        if residual.shape not in (shape, (m, n)) or residual.dtype is not out.dtype or (n > 1 and rs[-1] != 1) or \
                residual.get_device() != index:
            _bad(where, f"residual of shape {tuple(residual.shape)}, {residual.dtype}")
        rp, rl, rg = residual.data_ptr(), rs[-2], rs[0] if len(rs) == 3 else 0
    sp = 0
    if status is not None:
        if status.dtype is not torch.int32 or status.numel() != 1 or status.get_device() != index:
            _bad(where, f"status is one int32 on x's device, not {tuple(status.shape)} {status.dtype} on {status.device}")
        sp = status.data_ptr()
    args = LinearArgs(x.data_ptr(), xs[-2], xs[0] if xd == 3 else 0, w.data_ptr(), ws[-2], ws[0] if wd == 3 else 0, bp, bg, rp, rl,
                      rg, out.data_ptr(), os[-2], os[0] if len(os) == 3 else 0, groups, m, n, k,
                      _dtype_code(out.dtype, where), act_code, root, sp)
    _call((_lib or load()).symar_linear, where, index, stream, byref(args))
    return out


def rope_table(rows: int, rot_dim: int, *, base: float = 10000.0, kind: str = "plain", factor: float = 1.0,
               original: float = 0.0, low: float = 1.0, high: float = 32.0, magnitude: float = 1.0, device="cuda",
               stream=None):
    """[rows, rot_dim/2, 2] float32 (cos, sin) of every position and pair (``symar_rope_table``)."""
    torch = _torch()
    if kind not in ROPE_KINDS or rows < 0:
        _bad("symar_rope_table", f"rows {rows}, kind {kind!r}")
    at = torch.device(device)
    if at.type != "cuda":
        _bad("symar_rope_table", f"a table on {at}")
    index = _device() if at.index is None else at.index
    table = _new(torch.empty(0, dtype=torch.float32, device=at), (rows, rot_dim // 2, 2), torch.float32, index, stream)
    how = RopeScaling(base, factor, original, low, high, magnitude, ROPE_KINDS[kind], rot_dim)
    _call(load().symar_rope_table, "symar_rope_table", index, stream, table.data_ptr(), rows, byref(how))
    return table


class PagedKV:
    """A pool of 4-bit key/value pages in a torch uint8 tensor [pages, kv_heads, bytes of one head's page]."""

    def __init__(self, pages, head_dim: int, page_size: int):
        torch = _T or _torch()
        shape, index = pages.shape, pages.get_device()
        each = page_size * head_dim + 8 * page_size * (head_dim // KV_GROUP)
        if head_dim not in (64, 128, 256) or page_size not in (16, 32, 64, 128, 256):
            raise SymarError(ERR_UNSUPPORTED, f"PagedKV: head_dim {head_dim}, page_size {page_size}")
        if pages.dtype is not torch.uint8 or len(shape) != 3 or shape[2] != each or not pages.is_contiguous() or \
                index < 0:
            _bad("PagedKV", f"pages are a contiguous CUDA uint8 tensor [pages, kv_heads, {each}]")
        self.pages, self.head_dim, self.page_size, self.kv_heads, self.index = pages, head_dim, page_size, shape[1], index
        self.args = KVCacheArgs(pages.data_ptr(), shape[0], shape[1], head_dim, page_size)
        self.ref = byref(self.args)

    @classmethod
    def zeros(cls, pages: int, kv_heads: int, head_dim: int, page_size: int, device="cuda") -> "PagedKV":
        torch = _torch()
        each = int(load().symar_kv_page_bytes(1, head_dim, page_size))
        return cls(torch.zeros(pages, kv_heads, each, dtype=torch.uint8, device=device), head_dim, page_size)


class KVBatch:
    """The sequences of a call: int32 CUDA tensors lengths [seqs], page_table [seqs, columns] and, where sequences
    have other than one new token each, token_start [seqs + 1]."""

    def __init__(self, lengths, page_table, token_start=None):
        i32 = (_T or _torch()).int32
        ls, ps = lengths.shape, page_table.shape
        index = lengths.get_device()
        # (the row stride doubles as the number of columns that the kernels may read)
        if lengths.dtype is not i32 or page_table.dtype is not i32 or len(ls) != 1 or len(ps) != 2 or ps[0] != ls[0] or \
                not lengths.is_contiguous() or not page_table.is_contiguous() or index < 0 or page_table.get_device() != index:
            _bad("KVBatch", "lengths [seqs] and page_table [seqs, columns] are contiguous int32 CUDA tensors")
        seqs = ls[0]
        start = None
        if token_start is not None:
            if token_start.dtype is not i32 or token_start.shape != (seqs + 1,) or not token_start.is_contiguous() or \
                    token_start.get_device() != index:
                _bad("KVBatch", "token_start [seqs + 1] is a contiguous int32 CUDA tensor")
            start = token_start.data_ptr()
        self.lengths, self.page_table, self.token_start, self.seqs, self.index = lengths, page_table, token_start, seqs, index
        self._fields = lengths.data_ptr(), start, page_table.data_ptr(), ps[1], seqs
        self._last = (None, None)

    def of(self, tokens: int):
        """What a call with that many rows hands to the library.  Nothing that is handed out changes any more: calls of several threads
        may share a batch."""
        last = self._last
        if last[0] == tokens:
            return last[1]
        lengths, start, table, columns, seqs = self._fields
        ref = byref(KVBatchArgs(lengths, start, table, columns, seqs, tokens))
        self._last = (tokens, ref)
        return ref


class KVContext:
    """Owner of one ``symar_kv_t``: what the cache operators of one stream share."""

    def __init__(self, device_mem: int | None = None, device_bytes: int = 0, keepalive=None):
        _torch()
        self._lib = load()
        self._h = c_void_p()
        self._keepalive = keepalive
        if device_mem is None:
            _ck(self._lib.symar_kv_create(byref(self._h)), "symar_kv_create")
        else:
            _ck(self._lib.symar_kv_create_on(byref(self._h), device_mem, device_bytes), "symar_kv_create_on")
        self.index = _device()

    @classmethod
    def on_torch(cls, device="cuda:0") -> "KVContext":
        """Context in a torch uint8 tensor."""
        torch = _torch()
        n = int(load().symar_kv_required_bytes())
        buf = torch.empty(n + 256, dtype=torch.uint8, device=device)
        with torch.cuda.device(buf.device):
            return cls((buf.data_ptr() + 255) // 256 * 256, n, keepalive=buf)

    def destroy(self) -> None:
        """Gives the context back; its memory, where that is torch's, once no kernel of any stream uses it."""
        if self._h:
            self._lib.symar_kv_destroy(self._h)
            self._h = c_void_p()
            if self._keepalive is not None:
                if _T.cuda.is_current_stream_capturing():
                    _late.append((self.index, self._keepalive))     # (waiting would end the capture: kept until the next that may)
                else:
                    for index in sorted({self.index, *(i for i, _ in _late)}):
                        _T.cuda.synchronize(index)
                    _late.clear()
            self._keepalive = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def reset(self, stream=None) -> None:
        """Clear the status and the counters, on torch's current stream unless another is given: behind this context's calls
        there, and before those that follow."""
        _call(self._lib.symar_kv_reset, "symar_kv_reset", self.index, stream, self._h)

    def status(self):
        """(code, sequence, position) of the first offence since the last reset; waits for the device."""
        code, seq, position = c_int(), c_int(), c_int()
        with _T.cuda.device(self.index):
            _ck(self._lib.symar_kv_status(self._h, byref(code), byref(seq), byref(position)), "symar_kv_status")
        return code.value, seq.value, position.value

    def _devices(self, where, cache, batch):
        _bad(where, f"the context is of device {self.index}, the cache of {cache.index}, the batch of {batch.index}")

    @staticmethod
    def _refuse(where, name, t, shape, dtype):
        _bad(where, f"{name} is {list(shape)} {dtype} on the batch's device with contiguous channels, not {tuple(t.shape)} {t.dtype} on "
                    f"{t.device}")

    def append(self, cache: PagedKV, batch: KVBatch, k, v, *, q=None, q_out=None, rotations=None, interleaved: bool = False,
               stream=None):
        """Rotate q and k, store k and v (``symar_kv_append``); returns the rotated q (``q_out``, new unless given)."""
        where = "symar_kv_append"
        dtype, index, dim, ks, vs = k.dtype, batch.index, cache.head_dim, k.stride(), v.stride()
        code = _dtype_code(dtype, where)
        if cache.index != index or self.index != index:
            self._devices(where, cache, batch)
        tokens = k.shape[0] if len(ks) else 0
        shape = (tokens, cache.kv_heads, dim)
        if k.shape != shape or ks[2] != 1 or k.get_device() != index:
            self._refuse(where, "k", k, shape, dtype)
        if v.shape != shape or vs[2] != 1 or v.dtype is not dtype or v.get_device() != index:
            self._refuse(where, "v", v, shape, dtype)
        qp = op = q_heads = rp = rows = rot = 0
        qs = os = (0, 0)
        if q is not None:
            qs, shape = q.stride(), q.shape
            q_heads = shape[1] if len(shape) > 1 else 0
            if len(shape) != 3 or shape[0] != tokens or shape[2] != dim or qs[2] != 1 or q.dtype is not dtype or q.get_device() != index:
                self._refuse(where, "q", q, (tokens, q_heads, dim), dtype)
            if q_out is None:
                q_out = q.new_empty(shape) if stream is None else _new(q, shape, dtype, index, stream)
                os = (q_heads * dim, dim)
            else:
                os = q_out.stride()
                if q_out.shape != shape or os[2] != 1 or q_out.dtype is not dtype or q_out.get_device() != index:
                    self._refuse(where, "q_out", q_out, shape, dtype)
            qp, op = q.data_ptr(), q_out.data_ptr()
        if rotations is not None:
            rs = rotations.shape
            if len(rs) != 3 or rs[2] != 2 or rotations.dtype is not _T.float32 or not rotations.is_contiguous() or \
                    rotations.get_device() != index:
                _bad(where, "rotations are a contiguous float32 tensor [positions, rot_dim / 2, 2]")
            rp, rows, rot = rotations.data_ptr(), rs[0], 2 * rs[1]
        args = KVAppendArgs(qp, qs[0], qs[1], op, os[0], os[1], k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], rp, rows, rot,
                            1 if interleaved else 0, q_heads, code)
        _call(self._lib.symar_kv_append, where, index, stream, self._h, cache.ref, batch.of(tokens), byref(args))
        return q_out

    def read(self, cache: PagedKV, batch: KVBatch, tokens: int, *, dtype=None, stream=None):
        """(k, v) of the batch's new tokens as the cache holds them (``symar_kv_read``)."""
        if cache.index != batch.index or self.index != batch.index:
            self._devices("symar_kv_read", cache, batch)
        heads, dim = cache.kv_heads, cache.head_dim
        dtype, shape = dtype or (_T or _torch()).bfloat16, (tokens, heads, dim)
        if stream is None:
            k, v = cache.pages.new_empty(shape, dtype=dtype), cache.pages.new_empty(shape, dtype=dtype)
        else:
            k, v = (_new(cache.pages, shape, dtype, batch.index, stream) for _ in range(2))
        args = KVReadArgs(k.data_ptr(), heads * dim, dim, v.data_ptr(), heads * dim, dim, _dtype_code(dtype, "symar_kv_read"))
        _call(self._lib.symar_kv_read, "symar_kv_read", batch.index, stream, self._h, cache.ref, batch.of(tokens), byref(args))
        return k, v

    def attention(self, cache: PagedKV, batch: KVBatch, q, *, out=None, scale: float = 0.0, window: int = 0, stream=None):
        """Attention of the batch's new tokens over the cache (``symar_kv_attention``)."""
        where = "symar_kv_attention"
        shape, dtype, index = q.shape, q.dtype, batch.index
        if cache.index != index or self.index != index:
            self._devices(where, cache, batch)
        code, qs = _dtype_code(dtype, where), q.stride()
        if len(shape) != 3 or shape[2] != cache.head_dim or qs[2] != 1 or q.get_device() != index:
            _bad(where, f"q is [tokens, q_heads, {cache.head_dim}] on the batch's device with contiguous channels, not {tuple(shape)}")
        if out is None:
            out = q.new_empty(shape) if stream is None else _new(q, shape, dtype, index, stream)
        os = out.stride()
        if out.shape != shape or os[2] != 1 or out.dtype is not dtype or out.get_device() != index:
            self._refuse(where, "out", out, shape, dtype)
        args = KVAttentionArgs(q.data_ptr(), qs[0], qs[1], out.data_ptr(), os[0], os[1], scale, shape[1], window, code)
        _call(self._lib.symar_kv_attention, where, index, stream, self._h, cache.ref, batch.of(shape[0]), byref(args))
        return out


# -- probes --

def probe_empty(grid_x: int, grid_y: int, block: int, stream: int = 0) -> None:
    _ck(load().symar_probe_empty(grid_x, grid_y, block, stream), "symar_probe_empty")


def probe_empty_pdl(grid_x: int, grid_y: int, block: int, stream: int = 0) -> None:
    _ck(load().symar_probe_empty_pdl(grid_x, grid_y, block, stream), "symar_probe_empty_pdl")


def probe_empty_cluster(grid_x: int, grid_y: int, block: int, stream: int = 0) -> None:
    _ck(load().symar_probe_empty_cluster(grid_x, grid_y, block, stream), "symar_probe_empty_cluster")


def probe_fence(iterations: int = 20000) -> float:
    v = c_double()
    _ck(load().symar_probe_fence(iterations, byref(v)), "symar_probe_fence")
    return v.value


def probe_pingpong(iterations: int = 20000) -> float:
    v = c_double()
    _ck(load().symar_probe_pingpong(iterations, byref(v)), "symar_probe_pingpong")
    return v.value


def llbuffer_bytes(sync_mode: int, elem_bytes: int, slots_per_cta: int, ctas: int, round_robin: int) -> int:
    return int(load().symar_llbuffer_bytes(sync_mode, elem_bytes, slots_per_cta, ctas, round_robin))


def llbuffer_init_sentinel(device_ptr: int, nbytes: int, stream: int = 0) -> None:
    _ck(load().symar_llbuffer_init_sentinel(device_ptr, nbytes, stream), "symar_llbuffer_init_sentinel")


def probe_barrier(ranks: int, iterations: int = 5000, ordered: bool = False) -> float:
    """ns per all-to-all flag barrier among `ranks` CTAs (the barrier the method removes)."""
    v = c_double()
    _ck(load().symar_probe_barrier(ranks, iterations, 1 if ordered else 0, byref(v)), "symar_probe_barrier")
    return v.value


def probe_pingpong_blocks(first_block: int, partner_block: int, grid_blocks: int, iterations: int = 20000):
    """(ns per round trip, (smid_first, smid_partner)); only the two named blocks of the launch play."""
    v = c_double()
    sm = (c_int * 2)()
    _ck(load().symar_probe_pingpong_blocks(iterations, first_block, partner_block, grid_blocks, byref(v), sm),
        "symar_probe_pingpong_blocks")
    return v.value, (sm[0], sm[1])


def probe_pingpong_pair(partner_block: int, iterations: int = 20000):
    """(ns per round trip, (smid0, smid1)) between block 0 and block `partner_block`."""
    v = c_double()
    sm = (c_int * 2)()
    _ck(load().symar_probe_pingpong_pair(iterations, partner_block, byref(v), sm), "symar_probe_pingpong_pair")
    return v.value, (sm[0], sm[1])
