"""Python binding of libdck (ctypes): argument marshalling only.

Every function here has the name of the C entry point it calls and passes
raw device pointers (taken from torch tensors) and the current CUDA stream.
No step of the computation runs in Python: if ``libdck.so`` is missing the
import of this module's entry points raises.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "_build", "libdck.so")

DCK_OK = 0
DCK_ERR_INVALID = -1
DCK_ERR_UNSUPPORTED = -2
DCK_ERR_WORKSPACE = -3
DCK_ERR_CUDA = -4
DCK_ERR_TIMEOUT = -5
DCK_BF16 = 0
DCK_F32 = 1

EXPORTED = (
    "dck_status_string", "dck_validate_desc", "dck_latent_append_workspace_size", "dck_latent_append",
    "dck_decode_workspace_size", "dck_decode_attention", "dck_last_device_error", "dck_set_decode_kernel",
    "dck_last_launch_count", "dck_synth_gaussian", "dck_set_timing_events", "dck_decode_attention_noalloc",
    "dck_selftest_bounded_wait", "dck_selftest_append_timeout", "dck_decode_step", "dck_decode_step_workspace_size",
    "dck_prefill_workspace_size", "dck_prefill_attention", "dck_validate_paged_desc", "dck_page_update",
    "dck_rope_init", "dck_rope", "dck_paged_append", "dck_paged_decode_workspace_size", "dck_paged_decode_attention",
)


class DckError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


class LayerDesc(ctypes.Structure):
    _fields_ = [
        ("hidden", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("n_groups", ctypes.c_int32),
        ("group_offsets", ctypes.POINTER(ctypes.c_int32)),
        ("group_heads", ctypes.POINTER(ctypes.c_int32)),
        ("ranks", ctypes.POINTER(ctypes.c_int32)),
        ("rank_v", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
    ]


class PagedDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "page_size", "n_pages", "dtype")] + [
        (n, ctypes.c_int64) for n in ("k_page_stride", "k_token_stride", "k_head_stride", "v_page_stride",
                                      "v_token_stride", "v_head_stride")]


class RopeTable(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("initialised", ctypes.c_int32), ("turns", ctypes.c_uint64 * 128)]


_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """The loaded libdck.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"libdck.so is not built ({LIB_PATH}); run __graft_entry__.build()")
    L = ctypes.CDLL(LIB_PATH)
    P, I32, I64, U64, F32, SZ = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64,
                                 ctypes.c_float, ctypes.c_size_t)
    D = ctypes.POINTER(LayerDesc)
    L.dck_status_string.restype = ctypes.c_char_p
    L.dck_status_string.argtypes = [I32]
    L.dck_validate_desc.restype = I32
    L.dck_validate_desc.argtypes = [D]
    L.dck_latent_append_workspace_size.restype = SZ
    L.dck_latent_append_workspace_size.argtypes = [D, I32]
    L.dck_latent_append.restype = I32
    L.dck_latent_append.argtypes = [D, P, I32, P, P, P, P, P, I64, P, SZ, P]
    L.dck_decode_workspace_size.restype = SZ
    L.dck_decode_workspace_size.argtypes = [D, I32, I64]
    L.dck_decode_attention.restype = I32
    L.dck_decode_attention.argtypes = [D, P, P, P, I64, P, P, P, P, I32, F32, P, P, SZ, P]
    L.dck_prefill_workspace_size.restype = SZ
    L.dck_prefill_workspace_size.argtypes = [D, I64]
    L.dck_prefill_attention.restype = I32
    L.dck_prefill_attention.argtypes = [D, P, P, I32, P, P, I64, P, P, P, P, I32, I32, F32, P, P, SZ, P]
    L.dck_decode_step_workspace_size.restype = SZ
    L.dck_decode_step_workspace_size.argtypes = [D, I32, I64]
    L.dck_decode_step.restype = I32
    L.dck_decode_step.argtypes = [D, P, P, P, P, P, P, P, I64, P, P, P, P, I32, F32, P, P, SZ, P]
    L.dck_decode_attention_noalloc.restype = I32
    L.dck_decode_attention_noalloc.argtypes = [D, P, P, P, I64, P, P, P, P, I32, F32, P, P]
    L.dck_last_device_error.restype = I32
    L.dck_last_device_error.argtypes = [P]
    L.dck_set_decode_kernel.restype = I32
    L.dck_set_decode_kernel.argtypes = [I32]
    L.dck_last_launch_count.restype = I32
    L.dck_last_launch_count.argtypes = []
    L.dck_set_timing_events.restype = I32
    L.dck_set_timing_events.argtypes = [P, I32]
    L.dck_selftest_bounded_wait.restype = I32
    L.dck_selftest_bounded_wait.argtypes = [I64, P]
    L.dck_selftest_append_timeout.restype = I32
    L.dck_selftest_append_timeout.argtypes = [D, P, I32, P, P, P, P, P, I64, I64, P]
    L.dck_synth_gaussian.restype = I32
    L.dck_synth_gaussian.argtypes = [P, I64, U64, I64, F32, I32, P]
    G, R, F64 = ctypes.POINTER(PagedDesc), ctypes.POINTER(RopeTable), ctypes.c_double
    L.dck_validate_paged_desc.restype = I32
    L.dck_validate_paged_desc.argtypes = [G]
    L.dck_page_update.restype = I32
    L.dck_page_update.argtypes = [I32, I32, I32, P, P, P, P, I64, P, P, P, I64, P, P, P, P]
    L.dck_rope_init.restype = I32
    L.dck_rope_init.argtypes = [R, I32, I32, F64, I32, F64, F64, F64, I32, F64]
    L.dck_rope.restype = I32
    L.dck_rope.argtypes = [R, P, I32, I32, I32, I32, I64, I64, P, P, I64, I64, I32, P]
    L.dck_paged_append.restype = I32
    L.dck_paged_append.argtypes = [G, R, P, I64, P, I64, P, I64, I32, P, P, P, P, P, P]
    L.dck_paged_decode_workspace_size.restype = SZ
    L.dck_paged_decode_workspace_size.argtypes = [G, I32, I32]
    L.dck_paged_decode_attention.restype = I32
    L.dck_paged_decode_attention.argtypes = [G, P, I64, P, P, P, I64, P, I32, I32, F32, I32, F32, P, P, P, SZ, P]
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().dck_status_string(int(status)).decode()


class Layer:
    """A dck_layer_desc and the host arrays it points to (kept alive here)."""

    def __init__(self, hidden: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                 groups: Sequence[Sequence[int]], ranks: Sequence[int], rank_v: int, dtype: str):
        self.groups = [list(g) for g in groups]
        offs = [0]
        for g in self.groups:
            offs.append(offs[-1] + len(g))
        heads = [h for g in self.groups for h in g]
        self._offs = (ctypes.c_int32 * len(offs))(*offs)
        self._heads = (ctypes.c_int32 * max(1, len(heads)))(*heads)
        self._ranks = (ctypes.c_int32 * max(1, len(ranks)))(*ranks)
        self.dtype = dtype
        self.desc = LayerDesc(hidden, n_q_heads, n_kv_heads, head_dim, len(self.groups),
                              ctypes.cast(self._offs, ctypes.POINTER(ctypes.c_int32)),
                              ctypes.cast(self._heads, ctypes.POINTER(ctypes.c_int32)),
                              ctypes.cast(self._ranks, ctypes.POINTER(ctypes.c_int32)),
                              rank_v, DCK_F32 if dtype == "f32" else DCK_BF16)

    @classmethod
    def from_spec(cls, spec) -> "Layer":
        return cls(spec.hidden, spec.n_q_heads, spec.n_kv_heads, spec.head_dim, spec.groups,
                   spec.ranks, spec.rank_v, spec.dtype)

    @property
    def ref(self):
        return ctypes.byref(self.desc)


class PagedCache:
    """A dck_paged_desc: one uncompressed layer's key and value caches in pages.

    ``k_strides`` and ``v_strides`` are the elements between pages, tokens of a page
    and heads; by default caches are dense [n_pages, page_size, n_kv_heads, head_dim].
    """

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, dtype: str,
                 k_strides: Optional[Sequence[int]] = None, v_strides: Optional[Sequence[int]] = None):
        if dtype not in ("bf16", "f32"):
            raise ValueError(f"dtype: bf16 or f32, not {dtype!r}")
        row = n_kv_heads * head_dim
        dense = (page_size * row, row, head_dim)
        self.desc = PagedDesc(n_q_heads, n_kv_heads, head_dim, page_size, n_pages,
                              DCK_F32 if dtype == "f32" else DCK_BF16, *(k_strides or dense), *(v_strides or dense))
        self.ref = ctypes.byref(self.desc)

    @classmethod
    def from_tensors(cls, kcache, vcache, n_q_heads: int) -> "PagedCache":
        """The descriptor of torch caches (or views) [n_pages, page_size, n_kv_heads, head_dim], bf16 or fp32,
        whose head elements are consecutive."""
        name = {"torch.bfloat16": "bf16", "torch.float32": "f32"}.get(str(kcache.dtype))
        if kcache.shape != vcache.shape or kcache.dtype != vcache.dtype or kcache.dim() != 4 or name is None:
            raise ValueError("kcache and vcache: [n_pages, page_size, n_kv_heads, head_dim], bfloat16 or float32 alike")
        if kcache.stride(3) != 1 or vcache.stride(3) != 1:
            raise ValueError("the elements of a head must be consecutive")
        n_pages, page_size, n_kv_heads, head_dim = kcache.shape
        return cls(n_q_heads, n_kv_heads, head_dim, page_size, n_pages, name, kcache.stride()[:3], vcache.stride()[:3])


class Rope:
    """A dck_rope_table (dck_rope_init): rotary dimension, base, layout and the scaling for long contexts."""

    LAYOUTS = {"half": 0, "interleaved": 1}
    SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "bands": 3, "yarn": 4}

    def __init__(self, rotary_dim: int, theta: float, layout: str = "half", scaling: str = "none", factor: float = 1.0,
                 slow: float = 1.0, fast: float = 32.0, trained_len: int = 0, magnitude: float = 1.0):
        self.table = RopeTable()
        check(lib().dck_rope_init(ctypes.byref(self.table), self.LAYOUTS[layout], int(rotary_dim), float(theta),
                                  self.SCALINGS[scaling], float(factor), float(slow), float(fast), int(trained_len),
                                  float(magnitude)), "dck_rope_init")
        self.ref = ctypes.byref(self.table)


def _ptr(t) -> Optional[int]:
    try:
        return t.data_ptr()
    except AttributeError:
        if t is None or isinstance(t, int):  # an address
            return t
        raise  # ctypes would take bytes or str for one


_torch = None


def _stream(stream) -> Optional[int]:
    if stream is None:
        global _torch
        if _torch is None:
            import torch as _torch
        if _torch.cuda.is_initialized():  # the handle alone: a Stream object takes 3 us to make, a fifth of a short call
            return _torch._C._cuda_getCurrentRawStream(_torch._C._cuda_getDevice())
        return _torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def dck_validate_desc(layer: Layer) -> int:
    return lib().dck_validate_desc(layer.ref)


def dck_decode_workspace_size(layer: Layer, batch: int, n_rows: int) -> int:
    return lib().dck_decode_workspace_size(layer.ref, batch, n_rows)


def dck_latent_append_workspace_size(layer: Layer, n_tok: int) -> int:
    return lib().dck_latent_append_workspace_size(layer.ref, n_tok)


def dck_decode_attention(layer: Layer, q, kcache, vcache, n_rows: int, B_k, B_v, seq_start, seq_len,
                         batch: int, rope_theta: float, out, workspace, ws_bytes: int, stream=None) -> int:
    return lib().dck_decode_attention(layer.ref, _ptr(q), _ptr(kcache), _ptr(vcache), int(n_rows), _ptr(B_k),
                                      _ptr(B_v), _ptr(seq_start), _ptr(seq_len), int(batch), float(rope_theta),
                                      _ptr(out), _ptr(workspace), int(ws_bytes), _stream(stream))


def dck_decode_step_workspace_size(layer: Layer, batch: int, n_rows: int) -> int:
    return lib().dck_decode_step_workspace_size(layer.ref, batch, n_rows)


def dck_decode_step(layer: Layer, x, A_k, A_v, rows, q, kcache, vcache, n_rows: int, B_k, B_v, seq_start, seq_len,
                    batch: int, rope_theta: float, out, workspace, ws_bytes: int, stream=None) -> int:
    """Latent append of the batch's new tokens, then decode attention (one call)."""
    return lib().dck_decode_step(layer.ref, _ptr(x), _ptr(A_k), _ptr(A_v), _ptr(rows), _ptr(q), _ptr(kcache),
                                 _ptr(vcache), int(n_rows), _ptr(B_k), _ptr(B_v), _ptr(seq_start), _ptr(seq_len),
                                 int(batch), float(rope_theta), _ptr(out), _ptr(workspace), int(ws_bytes),
                                 _stream(stream))


def dck_prefill_workspace_size(layer: Layer, n_rows: int) -> int:
    return lib().dck_prefill_workspace_size(layer.ref, int(n_rows))


def dck_prefill_attention(layer: Layer, q, q_len, q_max: int, kcache, vcache, n_rows: int, B_k, B_v, seq_start,
                          seq_len, batch: int, max_seq_len: int, rope_theta: float, out, workspace, ws_bytes: int,
                          stream=None) -> int:
    return lib().dck_prefill_attention(layer.ref, _ptr(q), _ptr(q_len), int(q_max), _ptr(kcache), _ptr(vcache),
                                       int(n_rows), _ptr(B_k), _ptr(B_v), _ptr(seq_start), _ptr(seq_len), int(batch),
                                       int(max_seq_len), float(rope_theta), _ptr(out), _ptr(workspace),
                                       int(ws_bytes), _stream(stream))


def dck_decode_attention_noalloc(layer: Layer, q, kcache, vcache, n_rows: int, B_k, B_v, seq_start, seq_len,
                                 batch: int, rope_theta: float, out, stream=None) -> int:
    """dck_decode_attention without a workspace argument (library-owned fixed scratch)."""
    return lib().dck_decode_attention_noalloc(layer.ref, _ptr(q), _ptr(kcache), _ptr(vcache), int(n_rows),
                                              _ptr(B_k), _ptr(B_v), _ptr(seq_start), _ptr(seq_len), int(batch),
                                              float(rope_theta), _ptr(out), _stream(stream))


def dck_latent_append(layer: Layer, x, n_tok: int, A_k, A_v, rows, kcache, vcache, n_rows: int,
                      workspace, ws_bytes: int, stream=None) -> int:
    return lib().dck_latent_append(layer.ref, _ptr(x), int(n_tok), _ptr(A_k), _ptr(A_v), _ptr(rows), _ptr(kcache),
                                   _ptr(vcache), int(n_rows), _ptr(workspace), int(ws_bytes), _stream(stream))


def dck_validate_paged_desc(cache: PagedCache) -> int:
    return lib().dck_validate_paged_desc(cache.ref)


def dck_page_update(batch: int, page_size: int, n_pages: int, old_len, new_len, seq_len, block_table,
                    table_stride: int, free_pages, free_in, free_out, n_tok: int, slots, positions, cu_new,
                    stream=None) -> int:
    """A step's page bookkeeping: tables, free list, lengths, slots and positions of the new tokens."""
    return lib().dck_page_update(batch, page_size, n_pages, _ptr(old_len), _ptr(new_len), _ptr(seq_len),
                                 _ptr(block_table), table_stride, _ptr(free_pages), _ptr(free_in), _ptr(free_out),
                                 n_tok, _ptr(slots), _ptr(positions), _ptr(cu_new), _stream(stream))


def dck_rope(rope: Rope, x, n_tok: int, n_heads: int, head_dim: int, dtype: int, x_token_stride: int,
             x_head_stride: int, positions, out, out_token_stride: int, out_head_stride: int, transpose: bool = False,
             stream=None) -> int:
    """Rotation of x at the given positions, or its transpose (the gradient)."""
    return lib().dck_rope(rope.ref, _ptr(x), n_tok, n_heads, head_dim, dtype, x_token_stride,
                          x_head_stride, _ptr(positions), _ptr(out), out_token_stride, out_head_stride,
                          transpose, _stream(stream))


def dck_paged_append(cache: PagedCache, rope: Optional[Rope], q, q_stride: int, k, k_stride: int, v, v_stride: int,
                     n_tok: int, positions, slots, q_out, kcache, vcache, stream=None) -> int:
    """New tokens' queries rotated to q_out, their keys (rotated) and values written to the slots' cache rows."""
    return lib().dck_paged_append(cache.ref, rope.ref if rope is not None else None, _ptr(q), q_stride, _ptr(k),
                                  k_stride, _ptr(v), v_stride, n_tok, _ptr(positions), _ptr(slots),
                                  _ptr(q_out), _ptr(kcache), _ptr(vcache), _stream(stream))


def dck_paged_decode_workspace_size(cache: PagedCache, batch: int, max_seq_len: int) -> int:
    return lib().dck_paged_decode_workspace_size(cache.ref, batch, max_seq_len)


def dck_paged_decode_attention(cache: PagedCache, q, q_stride: int, kcache, vcache, block_table, table_stride: int,
                               seq_len, batch: int, max_seq_len: int, scale: float, window: int, softcap: float, out,
                               lse, workspace, ws_bytes: int, stream=None) -> int:
    """One query per sequence over its pages; lse (optional): the log of the softmax's sum."""
    return lib().dck_paged_decode_attention(cache.ref, _ptr(q), q_stride, _ptr(kcache), _ptr(vcache),
                                            _ptr(block_table), table_stride, _ptr(seq_len), batch,
                                            max_seq_len, scale, window, softcap, _ptr(out),
                                            _ptr(lse), _ptr(workspace), ws_bytes, _stream(stream))


def dck_last_device_error(stream=None) -> int:
    return lib().dck_last_device_error(_stream(stream))


def dck_set_decode_kernel(which: int) -> int:
    return lib().dck_set_decode_kernel(int(which))


def dck_last_launch_count() -> int:
    return lib().dck_last_launch_count()


def dck_synth_gaussian(dst, n: int, key: int, start: int, scale: float, dtype: int, stream=None) -> int:
    return lib().dck_synth_gaussian(_ptr(dst), int(n), int(key) & ((1 << 64) - 1), int(start), float(scale),
                                    int(dtype), _stream(stream))


def dck_set_timing_events(events) -> int:
    """``events``: torch.cuda.Event objects (already recorded once, so that the CUDA
    events exist), or None / [] to switch this thread's hook off."""
    if not events:
        return lib().dck_set_timing_events(None, 0)
    arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    return lib().dck_set_timing_events(arr, len(events))


def dck_selftest_bounded_wait(limit_cycles: int, stream=None) -> int:
    """One kernel whose bounded wait on a barrier nothing arrives at gives up after
    ``limit_cycles`` SM cycles; the timeout shows in the next dck_last_device_error."""
    return lib().dck_selftest_bounded_wait(int(limit_cycles), _stream(stream))


def dck_selftest_append_timeout(layer: Layer, x, n_tok: int, A_k, A_v, rows, kcache, vcache, n_rows: int,
                                limit_cycles: int, stream=None) -> int:
    """A tensor-core append whose last operand block is never loaded: its wait gives up
    after ``limit_cycles`` SM cycles, no row is written, the timeout is reported."""
    return lib().dck_selftest_append_timeout(layer.ref, _ptr(x), int(n_tok), _ptr(A_k), _ptr(A_v), _ptr(rows),
                                             _ptr(kcache), _ptr(vcache), int(n_rows), int(limit_cycles),
                                             _stream(stream))


def check(status: int, what: str) -> None:
    if status != DCK_OK:
        raise DckError(status, what)
