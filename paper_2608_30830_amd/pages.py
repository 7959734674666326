"""Binding of the entry points for a cache's pages, in the manner of ``kv``: argument
marshalling only, streams, ``check`` and ``status`` alike.

One pool of pages serves the caches of all layers.  Its state is three int32 tensors that the
calls change in place: ``refs`` [n_pages], how many rows hold each page (0: free), ``page_table``
[n_seqs, entries] and ``kv_len`` [n_seqs], which attention takes.  ``kvr_pages_resize`` takes and
gives back pages, ``kvr_pages_fork`` lets rows share them, ``kvr_pages_compact`` brings them
together; the last two name pages that ``kvr_pages_copy`` then copies in every layer.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Union

from . import kv
from .kv import KvCache
from .latent import LatentCache

EXPORTS = ("kvr_pages_fork", "kvr_pages_resize", "kvr_pages_compact", "kvr_pages_copy")


class kvr_page_pool(ctypes.Structure):
    _fields_ = [("d_refs", ctypes.c_void_p), ("d_pages", ctypes.c_void_p),
                ("d_kv_len", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
                ("pages_stride", ctypes.c_int64), ("max_pages", ctypes.c_int32),
                ("n_seqs", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class kvr_page_buffer(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("outer_stride", ctypes.c_int64), ("inner_stride", ctypes.c_int64),
                ("run_bytes", ctypes.c_int64), ("outer", ctypes.c_int32), ("inner", ctypes.c_int32)]


def declare(lib) -> None:
    """Argument types of the entry points above."""
    P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    C, Z = ctypes.POINTER(kvr_page_pool), ctypes.POINTER(ctypes.c_size_t)
    lib.kvr_pages_fork.argtypes = [C, P, P, P]
    lib.kvr_pages_resize.argtypes = [C, P, P, P, P, Z, P]
    lib.kvr_pages_compact.argtypes = [C, P, I64, P, P, P, Z, P]
    lib.kvr_pages_copy.argtypes = [ctypes.POINTER(kvr_page_buffer), I32, I64, P, I64, P, P]
    for name in EXPORTS:
        getattr(lib, name).restype = ctypes.c_int


class PageBuffers:
    """The tensors of one pool's caches (a KvCache or LatentCache of each layer, all with the
    same number of pages), kept alive with the C view of their pages."""

    def __init__(self, caches: Union[KvCache, LatentCache, Sequence]):
        if isinstance(caches, (KvCache, LatentCache)):
            caches = [caches]
        caches = list(caches)
        if not caches or not all(isinstance(c, (KvCache, LatentCache)) for c in caches):
            raise ValueError("caches must be KvCache or LatentCache objects")
        if any(c.n_pages != caches[0].n_pages for c in caches):
            raise ValueError("the caches of a pool must have the same number of pages")
        if any(c.device != caches[0].device for c in caches):
            raise ValueError("the caches of a pool must be on one device")
        tensors = [t for c in caches for t in c.tensors if t is not None]
        # tensors whose pages are alike next to each other: they are copied together
        tensors.sort(key=lambda t: (-t.element_size() * t.shape[1:].numel(), tuple(t.stride())))
        self.caches, self.n_pages, self.device = caches, caches[0].n_pages, caches[0].device
        self.c = c = (kvr_page_buffer * len(tensors))()
        for b, t in zip(c, tensors):
            e = t.element_size()
            b.data, b.page_stride, b.run_bytes = t.data_ptr(), e * t.stride(0), e * t.shape[-1]
            b.inner, b.inner_stride = t.shape[-2], e * t.stride(-2)
            b.outer, b.outer_stride = (t.shape[1], e * t.stride(1)) if t.dim() == 4 else (1, 0)
        self.handle = (ctypes.addressof(c), len(tensors), self.n_pages, tuple(tensors), c)


def kvr_pages_fork(refs, page_table, kv_len, parent, page_size: int, status=None, stream=None,
                   check: bool = True) -> None:
    """Rows b with ``parent[b]`` >= 0 ([n_seqs] int32) take that row's length and pages, which they
    then hold too.  They must be empty, and their parents rows without one."""
    c = kv._context()
    if check:
        status = kv._status(c, refs, check, status, stream)
    rc, = c.fast.pages_fork(refs, page_table, kv_len, parent, page_size, status, kv._handle(stream))
    if rc or check or stream is not None:
        kv._finish(c, "kvr_pages_fork", rc, check, status, stream)


def kvr_pages_resize(refs, page_table, kv_len, new_len, page_size: int, copies=None, workspace=None,
                     status=None, stream=None, check: bool = True):
    """Rows to ``new_len`` [n_seqs] int32 tokens (below 0: as they are; 0: given back whole).

    Pages are taken lowest first, in the order of rows.  A row that grows and whose last, partly
    filled page is held by others too takes one in its place: returns ``copies`` [n_seqs, 2] int32,
    the pages to copy for each row (kvr_pages_copy, before the row is written to), or -1.  A row
    that the free pages are too few for stays as it is: with ``check`` an error, whose ``copies`` are
    those of the rows that did grow."""
    c = kv._context()
    if check:
        status = kv._status(c, refs, check, status, stream)
    rc, copies, ws = c.fast.pages_resize(refs, page_table, kv_len, new_len, page_size, copies, workspace,
                                         status, kv._handle(stream))
    if rc or check or stream is not None:
        try:
            kv._finish(c, "kvr_pages_resize", rc, check, status, stream, copies, ws)
        except c.pkg.KvrError as e:   # of the device: the other rows have their new pages
            if not rc:
                e.copies = copies
            raise
    return copies


def kvr_pages_compact(refs, page_table, kv_len, page_size: int, max_moves: Optional[int] = None,
                      moves=None, used=None, workspace=None, status=None, stream=None,
                      check: bool = True):
    """The highest pages in use into the lowest free ones, while those are lower and at most
    ``max_moves`` (all that there are by default).  Returns (``moves`` [max_moves, 2] int32, the pages to
    copy, -1 from the last on; ``used`` [1] int32, the pages in use).  With ``check`` a row that does not
    fit is an error, whose ``moves`` and ``used`` are what was done all the same."""
    c = kv._context()
    if check:
        status = kv._status(c, refs, check, status, stream)
    rc, moves, used, ws = c.fast.pages_compact(refs, page_table, kv_len, page_size, max_moves, moves, used,
                                               workspace, status, kv._handle(stream))
    if rc or check or stream is not None:
        try:
            kv._finish(c, "kvr_pages_compact", rc, check, status, stream, moves, used, ws)
        except c.pkg.KvrError as e:
            if not rc:
                e.moves, e.used = moves, used
            raise
    return moves, used


def kvr_pages_copy(buffers: PageBuffers, pairs, status=None, stream=None, check: bool = True) -> None:
    """Copies page ``pairs[i, 0]`` to page ``pairs[i, 1]`` ([n, 2] int32; below 0: left out) in every
    tensor of ``buffers``.  No page may be written twice, or written and read."""
    c = kv._context()
    if check:
        status = kv._status(c, buffers, check, status, stream)
    rc, = c.fast.pages_copy(buffers.handle, pairs, status, kv._handle(stream))
    if rc or check or stream is not None:
        kv._finish(c, "kvr_pages_copy", rc, check, status, stream)
