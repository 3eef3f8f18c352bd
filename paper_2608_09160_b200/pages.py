"""Python side of include/qknorm_pages.h: the life of a paged cache's pages -- copying, forking a sequence, freeing, compacting.

Argument marshalling only, as in ``attn``: every step runs in the library's kernels, a bad argument raises ``QKNormError``, every
tensor of a call is on the current device.  What the calls share:

    pools        the cache: a tensor, or several, with the pages along axis `page_dim` and any axes beside it (layers, K and V, heads), whose
                 page is at most two axes of contiguous pieces
    refs         int32 [num_pages]: rows that hold a page; 0 or less: free
    block_table  int32 [rows, cols], lens int32 [rows]: a row holds the first ceil(lens / page_size) entries

Eight samples of one prompt, dropped and drawn again::

    pages.qknorm_pages_free(refs, block_table, lens, children, 16)
    pages.qknorm_pages_fork(kv_cache, refs, block_table, lens, parents, children, 16, page_dim=2)
"""
from __future__ import annotations

import ctypes
import functools
import struct
from typing import Tuple

import torch

from . import binding
from .attn import _current, _device, _empty, _flat, _int32, _refuse, _rows
from .binding import _check, _invoke

EXPORTS = (
    "qknorm_pages_copy",
    "qknorm_pages_fork",
    "qknorm_pages_free",
    "qknorm_pages_compact",
    "qknorm_pages_workspace",
)

_vp = ctypes.c_void_p
_SHAPE = binding.QKNORM_ERR_SHAPE


class CPagePool(ctypes.Structure):
    """qknorm_page_pool"""
    _fields_ = [("base", _vp), ("page", ctypes.c_int64), ("count", ctypes.c_int64 * 2), ("stride", ctypes.c_int64 * 2), ("bytes", ctypes.c_int64)]


_POOL = struct.Struct("Pqqqqqq")
assert _POOL.size == ctypes.sizeof(CPagePool)

_ready = False


def lib() -> ctypes.CDLL:
    """The loaded library with the prototypes of qknorm_pages.h declared."""
    global _ready
    L = binding.load()
    if _ready:
        return L
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    L.qknorm_pages_copy.argtypes = [_vp, i32, i64, _vp, _vp, i32, _vp]
    L.qknorm_pages_fork.argtypes = [_vp, i32, i64, _vp, _vp, i32, i64, _vp, i32, i32, _vp, _vp, i32, _vp, _vp, i64, _vp]
    L.qknorm_pages_free.argtypes = [_vp, i64, _vp, i32, i64, _vp, i32, i32, _vp, i32, _vp]
    L.qknorm_pages_compact.argtypes = [_vp, i32, i64, _vp, _vp, i32, i64, _vp, i32, i32, _vp, _vp, i64, _vp]
    L.qknorm_pages_workspace.argtypes = [i64, i32, i32, ctypes.POINTER(i64)]
    for name in EXPORTS:
        getattr(L, name).restype = ctypes.c_int
    _ready = True
    return L


@functools.lru_cache(maxsize=256)
def _pieces(shape: Tuple[int, ...], stride: Tuple[int, ...], item: int, page_dim: int):
    """How a page lies: (bytes between pages, two counts, two strides in bytes, bytes of a piece), or None."""
    axes = sorted((s * item, n) for d, (n, s) in enumerate(zip(shape, stride)) if d != page_dim and n > 1)
    piece, outer = item, []
    for s, n in axes:
        if not outer and s == piece:
            piece *= n
        elif outer and s == outer[-1][0] * outer[-1][1]:
            outer[-1] = (outer[-1][0], outer[-1][1] * n)
        else:
            outer.append((s, n))
    if len(outer) > 2 or any(n == 0 for n in shape):
        return None
    outer = [(0, 1)] * (2 - len(outer)) + outer[::-1]
    return stride[page_dim] * item, outer[0][1], outer[1][1], outer[0][0], outer[1][0], piece


def _pools(pools, page_dim: int, dev: int, num_pages: int = -1):
    """The pools as the C ABI takes them: (structs, how many, pages), and the tensors themselves, to be kept as long as the call is."""
    pools = (pools,) if isinstance(pools, torch.Tensor) else tuple(pools)
    packed = []
    for t in pools:
        if not isinstance(t, torch.Tensor) or t.get_device() != dev or not -t.dim() <= page_dim < t.dim():
            _refuse(_SHAPE, f"pools: expected tensors with axis {page_dim} on cuda:{dev}")
        d = page_dim % t.dim()
        if num_pages < 0:
            num_pages = t.shape[d]
        if t.shape[d] != num_pages:
            _refuse(_SHAPE, f"pools: {t.shape[d]} pages along axis {page_dim}, expected {num_pages}")
        how = _pieces(tuple(t.shape), t.stride(), t.element_size(), d)
        if how is None:
            _refuse(_SHAPE, f"pools: a page of {tuple(t.shape)} with strides {t.stride()} is more than two axes of contiguous pieces")
        packed.append(_POOL.pack(t.data_ptr(), *how))
    return b"".join(packed), len(packed), num_pages, pools


def _books(refs, block_table, lens, dev: int):
    """refs, block_table and lens: (pages, addresses, cols, row stride, rows)."""
    if not isinstance(refs, torch.Tensor) or refs.dim() != 1:
        _refuse(_SHAPE, "refs: expected an int32 CUDA tensor [num_pages]")
    if not isinstance(lens, torch.Tensor) or lens.dim() != 1:
        _refuse(_SHAPE, "lens: expected an int32 CUDA tensor [rows]")
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
        _refuse(_SHAPE, "block_table: expected an int32 CUDA tensor [rows, pages per row]")
    n, rows = refs.shape[0], lens.shape[0]
    prefs, plens = _flat(refs, (n,), torch.int32, "refs", dev), _flat(lens, (rows,), torch.int32, "lens", dev)
    ptable, cols, ld = _rows(block_table, rows, "block_table", torch.int32, dev)
    return n, prefs, ptable, cols, ld, plens, rows


def _list(t, what: str, dev: int):
    if not isinstance(t, torch.Tensor) or t.dim() != 1:
        _refuse(_SHAPE, f"{what}: expected a 1-D int32 CUDA tensor")
    return _flat(t, (t.shape[0],), torch.int32, what, dev)


def pages_workspace(num_pages: int, rows: int, n: int = 0) -> int:
    """qknorm_pages_workspace: bytes that n forks, or (n = 0) compacting, need."""
    return _workspace(int(num_pages), _int32(rows, "rows"), _int32(n, "n"))


@functools.lru_cache(maxsize=256)
def _workspace(num_pages: int, rows: int, n: int) -> int:
    out = ctypes.c_int64(0)
    _check(lib().qknorm_pages_workspace(num_pages, rows, n, ctypes.byref(out)))
    return out.value


def _scratch(workspace, num_pages: int, rows: int, n: int, device, stream, dev: int):
    if workspace is None:
        workspace = _empty((_workspace(num_pages, rows, n),), torch.uint8, device, stream)
    elif not workspace.is_contiguous() or workspace.get_device() != dev:
        _refuse(binding.QKNORM_ERR_SCRATCH, f"workspace: expected a contiguous tensor on cuda:{dev}")
    return workspace, workspace.numel() * workspace.element_size()


def qknorm_pages_copy(pools, src, dst, *, page_dim: int = 0, stream=None) -> None:
    """qknorm_pages_copy: page src[i] to page dst[i] in every pool; src, dst int32 [n].  Pairs outside the pool copy nothing."""
    L = lib()
    dev = _device()
    packed, k, n, pools = _pools(pools, page_dim, dev)
    psrc, pdst = _list(src, "src", dev), _list(dst, "dst", dev)
    if src.shape != dst.shape:
        _refuse(_SHAPE, f"src, dst: {src.shape[0]} and {dst.shape[0]} pages")
    if k == 0:
        return
    _invoke(L.qknorm_pages_copy, (packed, k, n, psrc, pdst, src.shape[0]), _current(stream), (pools, src, dst))


def qknorm_pages_fork(pools, refs, block_table, lens, parents, children, page_size: int, *, page_dim: int = 0, ok=None, workspace=None,
                      stream=None):
    """qknorm_pages_fork: row children[i] becomes a copy of row parents[i] that can grow by itself, sharing full pages; the
    children have to be empty (qknorm_pages_free).  ok int32 [n] to fill: 1 for forks made, 0 for those left out.
    workspace: uint8 tensor of pages_workspace(num_pages, rows, n) bytes, by default a new one per call.  Returns ok."""
    L = lib()
    dev = _device()
    N, prefs, ptable, cols, ld, plens, rows = _books(refs, block_table, lens, dev)
    packed, k, _, pools = _pools(pools, page_dim, dev, N)
    pp, pc = _list(parents, "parents", dev), _list(children, "children", dev)
    n = parents.shape[0]
    if children.shape[0] != n:
        _refuse(_SHAPE, f"parents, children: {n} and {children.shape[0]} rows")
    pok = None if ok is None else _flat(ok, (n,), torch.int32, "ok", dev)
    workspace, nbytes = _scratch(workspace, N, rows, n, refs.device, stream, dev)
    _invoke(L.qknorm_pages_fork, (packed, k, N, prefs, ptable, cols, ld, plens, rows, _int32(page_size, "page_size"), pp, pc, n, pok,
                                  workspace.data_ptr(), nbytes), _current(stream),
            (pools, refs, block_table, lens, parents, children, ok, workspace))
    return ok


def qknorm_pages_free(refs, block_table, lens, rows, page_size: int, *, stream=None) -> None:
    """qknorm_pages_free: the rows named (int32 [n]) give up their pages; their lens become 0."""
    L = lib()
    dev = _device()
    N, prefs, ptable, cols, ld, plens, R = _books(refs, block_table, lens, dev)
    plist = _list(rows, "rows", dev)
    _invoke(L.qknorm_pages_free, (prefs, N, ptable, cols, ld, plens, R, _int32(page_size, "page_size"), plist, rows.shape[0]), _current(stream),
            (refs, block_table, lens, rows))


def qknorm_pages_compact(pools, refs, block_table, lens, page_size: int, *, page_dim: int = 0, live=None, workspace=None, stream=None):
    """qknorm_pages_compact: the held pages move together at the pool's start, tables and refs with them.  Returns live, int32 [1] on the
    device (a new tensor unless given): the number of pages held, all below it now."""
    L = lib()
    dev = _device()
    N, prefs, ptable, cols, ld, plens, R = _books(refs, block_table, lens, dev)
    packed, k, _, pools = _pools(pools, page_dim, dev, N)
    if live is None:
        live = _empty((1,), torch.int32, refs.device, stream)
    plive = _flat(live, (1,), torch.int32, "live", dev)
    workspace, nbytes = _scratch(workspace, N, R, 0, refs.device, stream, dev)
    _invoke(L.qknorm_pages_compact, (packed, k, N, prefs, ptable, cols, ld, plens, R, _int32(page_size, "page_size"), plive, workspace.data_ptr(),
                                     nbytes), _current(stream), (pools, refs, block_table, lens, live, workspace))
    return live
