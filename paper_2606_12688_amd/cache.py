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


_torch = None
_current_device = None  # the current device's index; torch's own function behind torch.cuda.current_device where it is there


def _init():
    global _torch, _current_device
    import torch

    _torch = torch
    _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    lib()


def _explain(*tensors):
    """A call that is not in order, taken apart for its message: ``(name, tensor, shape, dtype)`` each."""
    dev = _torch.cuda.current_device() if _torch.cuda.is_available() else -1
    for name, t, shape, dtype in tensors:
        _need(t.is_cuda and t.get_device() == dev, f"{name} must be on the current device")
        _need(t.dtype == dtype, f"{name} must be {dtype}")
        _need(tuple(t.shape) == tuple(shape), f"{name} must be {list(shape)}")
        _need(t.is_contiguous(), f"{name} must be contiguous")


def _pool_shape(pl: attn.Plan):
    shape = getattr(pl, "_kv4_shape", None)
    if shape is None:
        p = pl.params
        shape = pl._kv4_shape = (p.num_pages, p.num_kv_heads, record_bytes(p.head_dim))
    return shape


def kv4_append(pl: attn.Plan, k_new, v_new, block_table, k_pages, v_pages, stream=None):
    """``mstar_kv4_append`` on torch tensors: round the plan's new K/V rows
    (bf16 ``[total_q, Hkv, d]``, the row numbering of q) to 4 bits and write
    them into their pages of a 4-bit cache."""
    if _torch is None:
        _init()
    pool, dev, bf16, u8, i32 = _pool_shape(pl), k_new.get_device(), _torch.bfloat16, _torch.uint8, _torch.int32
    if not (dev >= 0 and v_new.get_device() == dev and block_table.get_device() == dev
            and k_pages.get_device() == dev and v_pages.get_device() == dev and _current_device() == dev
            and k_new.dtype is bf16 and v_new.dtype is bf16 and block_table.dtype is i32
            and k_pages.dtype is u8 and v_pages.dtype is u8
            and k_new.shape == pl._new_shape and v_new.shape == pl._new_shape
            and block_table.shape == pl._table_shape and k_pages.shape == pool and v_pages.shape == pool
            and k_new.is_contiguous() and v_new.is_contiguous() and block_table.is_contiguous()
            and k_pages.is_contiguous() and v_pages.is_contiguous()):
        _explain(("k_new", k_new, pl._new_shape, bf16), ("v_new", v_new, pl._new_shape, bf16),
                 ("block_table", block_table, pl._table_shape, i32), ("k_pages", k_pages, pool, u8),
                 ("v_pages", v_pages, pool, u8))
    rc = _lib.mstar_kv4_append(pl.handle, k_new.data_ptr(), v_new.data_ptr(), block_table.data_ptr(),
                               k_pages.data_ptr(), v_pages.data_ptr(), _stream_handle(stream))
    if rc:
        _check_rc(rc)


def _check_fwd(pl, q, k_pages, v_pages, block_table, out, lse):
    if _torch is None:
        _init()
    pool, dev, bf16, u8 = _pool_shape(pl), q.get_device(), _torch.bfloat16, _torch.uint8
    if not (dev >= 0 and k_pages.get_device() == dev and v_pages.get_device() == dev
            and block_table.get_device() == dev and out.get_device() == dev and lse.get_device() == dev
            and _current_device() == dev
            and q.dtype is bf16 and out.dtype is bf16 and k_pages.dtype is u8 and v_pages.dtype is u8
            and lse.dtype is _torch.float32 and block_table.dtype is _torch.int32
            and q.shape == pl._q_shape and out.shape == pl._q_shape and lse.shape == pl._lse_shape
            and k_pages.shape == pool and v_pages.shape == pool and block_table.shape == pl._table_shape
            and q.is_contiguous() and k_pages.is_contiguous() and v_pages.is_contiguous()
            and block_table.is_contiguous() and out.is_contiguous() and lse.is_contiguous()):
        _explain(("q", q, pl._q_shape, bf16), ("k_pages", k_pages, pool, u8), ("v_pages", v_pages, pool, u8),
                 ("block_table", block_table, pl._table_shape, _torch.int32), ("out", out, pl._q_shape, bf16),
                 ("lse", lse, pl._lse_shape, _torch.float32))
    return dev


def kv4_fwd(pl: attn.Plan, q, k_pages, v_pages, block_table, out, lse, workspace=None, stream=None):
    """``mstar_kv4_fwd`` on torch tensors: :func:`attn.fwd` over a 4-bit cache, for
    values of up to 2^64 in magnitude.  ``workspace`` as there (:func:`attn.workspace`)."""
    dev = _check_fwd(pl, q, k_pages, v_pages, block_table, out, lse)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        _need(workspace.get_device() == dev and workspace.is_contiguous(), "bad workspace")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.nbytes
    rc = _lib.mstar_kv4_fwd(pl.handle, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(),
                            out.data_ptr(), lse.data_ptr(), ws_ptr, ws_bytes, _stream_handle(stream))
    if rc:
        _check_rc(rc)


def kv4_fwd_noalloc(pl: attn.Plan, q, k_pages, v_pages, block_table, out, lse, stream=None):
    """``mstar_kv4_fwd_noalloc`` on torch tensors: :func:`attn.fwd_noalloc` over a 4-bit cache."""
    _check_fwd(pl, q, k_pages, v_pages, block_table, out, lse)
    rc = _lib.mstar_kv4_fwd_noalloc(pl.handle, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                    block_table.data_ptr(), out.data_ptr(), lse.data_ptr(), _stream_handle(stream))
    if rc:
        _check_rc(rc)


def kv4_unpack(k_pages, v_pages, page_ids, k_out, v_out, stream=None):
    """``mstar_kv4_unpack`` on torch tensors: pages ``page_ids`` (int32 ``[n]``) of a 4-bit cache as bf16 pages
    ``[n, 16, Hkv, d]``; an index outside the pool gives zeros."""
    if _torch is None:
        _init()
    shape, pages = k_pages.shape, k_out.shape
    _need(len(shape) == 3 and len(pages) == 4 and page_ids.dim() == 1, "k_pages, k_out or page_ids has wrong dims")
    (num_pages, hkv, record), n, d = shape, page_ids.shape[0], pages[3]
    dev, bf16, u8 = k_pages.get_device(), _torch.bfloat16, _torch.uint8
    if not (dev >= 0 and v_pages.get_device() == dev and page_ids.get_device() == dev and k_out.get_device() == dev
            and v_out.get_device() == dev and _current_device() == dev
            and k_pages.dtype is u8 and v_pages.dtype is u8 and page_ids.dtype is _torch.int32
            and k_out.dtype is bf16 and v_out.dtype is bf16
            and record == record_bytes(d) and v_pages.shape == shape and pages == (n, 16, hkv, d)
            and v_out.shape == pages
            and k_pages.is_contiguous() and v_pages.is_contiguous() and page_ids.is_contiguous()
            and k_out.is_contiguous() and v_out.is_contiguous()):
        pool, out = (num_pages, hkv, record_bytes(d)), (n, 16, hkv, d)
        _explain(("k_pages", k_pages, pool, u8), ("v_pages", v_pages, pool, u8),
                 ("page_ids", page_ids, (n,), _torch.int32), ("k_out", k_out, out, bf16), ("v_out", v_out, out, bf16))
    rc = _lib.mstar_kv4_unpack(hkv, d, num_pages, k_pages.data_ptr(), v_pages.data_ptr(), page_ids.data_ptr(), n,
                               k_out.data_ptr(), v_out.data_ptr(), _stream_handle(stream))
    if rc:
        _check_rc(rc)


def block_tables_pages(pl: attn.Plan) -> int:
    """``mstar_block_tables_pages``: how many pages of the free list the plan's new rows take."""
    return int(lib().mstar_block_tables_pages(pl.handle))


def block_tables(pl: attn.Plan, free_pages, block_table, slots=None, stream=None):
    """``mstar_block_tables`` on torch tensors: the pages of the plan's new rows,
    taken from the front of ``free_pages`` (int32 ``[m]``; :func:`block_tables_pages`
    says how many), are entered into ``block_table`` (int32 ``[num_seqs,
    max_blocks]``), and ``slots`` (int64 ``[total_q]``, optional) gets every new
    row's flat slot."""
    if _torch is None:
        _init()
    dev, i32 = block_table.get_device(), _torch.int32
    if not (dev >= 0 and free_pages.get_device() == dev and _current_device() == dev
            and free_pages.dtype is i32 and block_table.dtype is i32
            and free_pages.dim() == 1 and block_table.shape == pl._table_shape
            and free_pages.is_contiguous() and block_table.is_contiguous()):
        _explain(("free_pages", free_pages, (free_pages.numel(),), i32),
                 ("block_table", block_table, pl._table_shape, i32))
    slots_ptr = None
    if slots is not None:
        if not (slots.get_device() == dev and slots.dtype is _torch.int64 and slots.shape == (pl.total_q,)
                and slots.is_contiguous()):
            _explain(("slots", slots, (pl.total_q,), _torch.int64))
        slots_ptr = slots.data_ptr()
    rc = _lib.mstar_block_tables(pl.handle, free_pages.data_ptr(), free_pages.shape[0], block_table.data_ptr(),
                                 slots_ptr, _stream_handle(stream))
    if rc:
        _check_rc(rc)
