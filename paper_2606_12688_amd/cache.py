"""Python binding of the operators on paged caches (``include/mstar_cache.h``):
a KV cache held in 4 bits and block tables built on the GPU.

Like :mod:`attn`, argument marshalling only, over the same library, plans and
streams.  The names follow the C entry points: :func:`kv4_append`
(``mstar_kv4_append``), :func:`kv4_fwd` (``mstar_kv4_fwd``),
:func:`kv4_fwd_noalloc` (``mstar_kv4_fwd_noalloc``), :func:`kv4_unpack`
(``mstar_kv4_unpack``), :func:`block_tables` (``mstar_block_tables``) and
:func:`block_tables_pages` (``mstar_block_tables_pages``).  A step with both::

    plan = attn.plan(...)                                    # the step's requests
    cache.block_tables(plan, free_pages, block_table)        # pages of the new tokens
    for layer in layers:
        cache.kv4_append(plan, k, v, block_table, *pools[layer])
        cache.kv4_fwd(plan, q, *pools[layer], block_table, out, lse, workspace)
"""
from __future__ import annotations

import ctypes

from . import attn
from .attn import _check_rc, _need, _stream_handle

DEVERR_NONFINITE = 2

EXPORTS = [
    "mstar_kv4_append",
    "mstar_kv4_fwd",
    "mstar_kv4_fwd_noalloc",
    "mstar_kv4_unpack",
    "mstar_block_tables_pages",
    "mstar_block_tables",
]

_lib = None


def lib() -> ctypes.CDLL:
    """The built library (raises if it is missing) with this module's functions declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = attn.lib()
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    L.mstar_kv4_append.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.mstar_kv4_append.restype = ctypes.c_int
    L.mstar_kv4_fwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.mstar_kv4_fwd.restype = ctypes.c_int
    L.mstar_kv4_fwd_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    L.mstar_kv4_fwd_noalloc.restype = ctypes.c_int
    L.mstar_kv4_unpack.argtypes = [i32, i32, i32, vp, vp, vp, i32, vp, vp, vp]
    L.mstar_kv4_unpack.restype = ctypes.c_int
    L.mstar_block_tables_pages.argtypes = [vp]
    L.mstar_block_tables_pages.restype = i64
    L.mstar_block_tables.argtypes = [vp, vp, i64, vp, vp, vp]
    L.mstar_block_tables.restype = ctypes.c_int
    _lib = L
    return L


def record_bytes(head_dim: int) -> int:
    """Bytes of a record of the 4-bit cache: one page and KV head of a K or V pool."""
    return 17 * head_dim // 2


def kv4_pages(num_pages: int, num_kv_heads: int, head_dim: int, device):
    """A K and a V pool of a 4-bit cache, every value 0."""
    import torch

    shape = (num_pages, num_kv_heads, record_bytes(head_dim))
    return torch.zeros(shape, dtype=torch.uint8, device=device), torch.zeros(shape, dtype=torch.uint8, device=device)


def _check(tensors, stream):
    """``(name, tensor, shape, dtype)`` of a call: right shapes and types, dense, and all on the current device.
    Returns the stream's handle."""
    import torch

    dev = torch.cuda.current_device() if torch.cuda.is_available() else -1
    for name, t, shape, dtype in tensors:
        if t.get_device() == dev and t.is_cuda and t.dtype is dtype and t.shape == shape and t.is_contiguous():
            continue
        _need(t.is_cuda and t.get_device() == dev, f"{name} must be on the current device")
        _need(t.dtype == dtype, f"{name} must be {dtype}")
        _need(tuple(t.shape) == tuple(shape), f"{name} must be {list(shape)}")
        _need(t.is_contiguous(), f"{name} must be contiguous")
    return _stream_handle(stream)


def _pool_shape(pl: attn.Plan):
    p = pl.params
    return p.num_pages, p.num_kv_heads, record_bytes(p.head_dim)


def kv4_append(pl: attn.Plan, k_new, v_new, block_table, k_pages, v_pages, stream=None):
    """``mstar_kv4_append`` on torch tensors: round the plan's new K/V rows
    (bf16 ``[total_q, Hkv, d]``, the row numbering of q) to 4 bits and write
    them into their pages of a 4-bit cache."""
    import torch

    pool = _pool_shape(pl)
    s = _check((("k_new", k_new, pl._new_shape, torch.bfloat16), ("v_new", v_new, pl._new_shape, torch.bfloat16),
                ("block_table", block_table, pl._table_shape, torch.int32),
                ("k_pages", k_pages, pool, torch.uint8), ("v_pages", v_pages, pool, torch.uint8)), stream)
    _check_rc(lib().mstar_kv4_append(pl.handle, k_new.data_ptr(), v_new.data_ptr(), block_table.data_ptr(),
                                     k_pages.data_ptr(), v_pages.data_ptr(), s))


def _check_fwd(pl, q, k_pages, v_pages, block_table, out, lse, stream):
    import torch

    pool = _pool_shape(pl)
    return _check((("q", q, pl._q_shape, torch.bfloat16), ("k_pages", k_pages, pool, torch.uint8),
                   ("v_pages", v_pages, pool, torch.uint8),
                   ("block_table", block_table, pl._table_shape, torch.int32),
                   ("out", out, pl._q_shape, torch.bfloat16), ("lse", lse, pl._lse_shape, torch.float32)), stream)


def kv4_fwd(pl: attn.Plan, q, k_pages, v_pages, block_table, out, lse, workspace=None, stream=None):
    """``mstar_kv4_fwd`` on torch tensors: :func:`attn.fwd` over a 4-bit cache.
    ``workspace`` as there (:func:`attn.workspace`)."""
    s = _check_fwd(pl, q, k_pages, v_pages, block_table, out, lse, stream)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        _need(workspace.is_cuda and workspace.device == q.device and workspace.is_contiguous(), "bad workspace")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.nbytes
    _check_rc(lib().mstar_kv4_fwd(pl.handle, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                  block_table.data_ptr(), out.data_ptr(), lse.data_ptr(), ws_ptr, ws_bytes, s))


def kv4_fwd_noalloc(pl: attn.Plan, q, k_pages, v_pages, block_table, out, lse, stream=None):
    """``mstar_kv4_fwd_noalloc`` on torch tensors: :func:`attn.fwd_noalloc` over a 4-bit cache."""
    s = _check_fwd(pl, q, k_pages, v_pages, block_table, out, lse, stream)
    _check_rc(lib().mstar_kv4_fwd_noalloc(pl.handle, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                          block_table.data_ptr(), out.data_ptr(), lse.data_ptr(), s))


def kv4_unpack(k_pages, v_pages, page_ids, k_out, v_out, stream=None):
    """``mstar_kv4_unpack`` on torch tensors: pages ``page_ids`` (int32 ``[n]``) of a 4-bit cache as bf16 pages
    ``[n, 16, Hkv, d]``; an index outside the pool gives zeros."""
    import torch

    _need(k_pages.dim() == 3 and k_out.dim() == 4 and page_ids.dim() == 1, "k_pages, k_out or page_ids has wrong dims")
    hkv, d = k_pages.shape[1], k_out.shape[3]
    pool, pages = (k_pages.shape[0], hkv, record_bytes(d)), (page_ids.shape[0], 16, hkv, d)
    s = _check((("k_pages", k_pages, pool, torch.uint8), ("v_pages", v_pages, pool, torch.uint8),
                ("page_ids", page_ids, page_ids.shape, torch.int32), ("k_out", k_out, pages, torch.bfloat16),
                ("v_out", v_out, pages, torch.bfloat16)), stream)
    _check_rc(lib().mstar_kv4_unpack(hkv, d, k_pages.shape[0], k_pages.data_ptr(), v_pages.data_ptr(),
                                     page_ids.data_ptr(), page_ids.shape[0], k_out.data_ptr(), v_out.data_ptr(), s))


def block_tables_pages(pl: attn.Plan) -> int:
    """``mstar_block_tables_pages``: how many pages of the free list the plan's new rows take."""
    return int(lib().mstar_block_tables_pages(pl.handle))


def block_tables(pl: attn.Plan, free_pages, block_table, slots=None, stream=None) -> int:
    """``mstar_block_tables`` on torch tensors: the pages of the plan's new rows,
    taken from the front of ``free_pages`` (int32 ``[m]``), are entered into
    ``block_table`` (int32 ``[num_seqs, max_blocks]``), and ``slots`` (int64
    ``[total_q]``, optional) gets every new row's flat slot.  Returns the number
    of pages taken."""
    import torch

    _need(free_pages.dim() == 1, "free_pages must have one dimension")
    tensors = [("free_pages", free_pages, free_pages.shape, torch.int32),
               ("block_table", block_table, pl._table_shape, torch.int32)]
    if slots is not None:
        tensors.append(("slots", slots, (pl.total_q,), torch.int64))
    s = _check(tensors, stream)
    _check_rc(lib().mstar_block_tables(pl.handle, free_pages.data_ptr(), free_pages.shape[0],
                                       block_table.data_ptr(), None if slots is None else slots.data_ptr(), s))
    return block_tables_pages(pl)
