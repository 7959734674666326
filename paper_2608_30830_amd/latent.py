"""Binding of the latent cache's entry points of libkvr, in the manner of ``kv``: argument
marshalling only, streams, ``check`` and ``status`` alike, no gradients recorded.

A latent cache keeps one row a token for all heads: a latent, from which every head's key and
value follow by a product with a weight, and a rotated key that all heads share.
``kvr_latent_write`` and ``kvr_latent_read`` move rows, ``kvr_latent_attention`` attends to them
as they are (the absorbed form), ``kvr_latent_prompt`` attends to keys and values that were
expanded for each head (prompts).
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import kv
from .kv import BLOCK, KVR_KV_BF16, KVR_KV_FP16, KVR_KV_FP8

EXPORTS = ("kvr_latent_write", "kvr_latent_read", "kvr_latent_attention", "kvr_latent_prompt")


class kvr_latent_cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("scale_page_stride", ctypes.c_int64), ("scale_token_stride", ctypes.c_int64),
                ("n_pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("rank", ctypes.c_int32),
                ("rot", ctypes.c_int32), ("format", ctypes.c_int32)]


class kvr_prompt(ctypes.Structure):
    _fields_ = [("d_cu_q", ctypes.c_void_p), ("d_cu_k", ctypes.c_void_p),
                ("n_queries", ctypes.c_int64), ("n_keys", ctypes.c_int64),
                ("n_seqs", ctypes.c_int32), ("max_q", ctypes.c_int32), ("max_k", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("nope", ctypes.c_int32), ("rot", ctypes.c_int32), ("causal", ctypes.c_int32)]


def declare(lib) -> None:
    """Argument types of the entry points above."""
    P, I32, I64, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    C, Z = ctypes.POINTER(kvr_latent_cache), ctypes.POINTER(ctypes.c_size_t)
    lib.kvr_latent_write.argtypes = [C, P, P, I32, I64, I64, I64, P, F, P, P, P, I64, I32, I32, P, P]
    lib.kvr_latent_read.argtypes = [C, P, I64, P, I32, I64, P, P]
    lib.kvr_latent_attention.argtypes = [C, ctypes.POINTER(kv.kvr_sequences), P, I32, I32, I64, I64,
                                         P, I32, F, P, I64, I64, P, P, P, Z, P]
    lib.kvr_latent_prompt.argtypes = [ctypes.POINTER(kvr_prompt), P, I32, I64, I64, P, I64, I64, P,
                                      I64, P, I64, I64, F, P, I64, I64, P, P, P, Z, P]
    for name in EXPORTS:
        getattr(lib, name).restype = ctypes.c_int


class LatentCache:
    """The tensors of a paged latent cache, kept alive with the C view of them.

    ``rows``: [n_pages, page_size, rank + rot], any strides with adjacent rows; bfloat16 or
    float16, or uint8 codes (e4m3) with ``scale`` [n_pages, page_size, (rank + rot) / 32] uint8.
    ``rot``: elements of the shared key, the last ones of a row."""

    def __init__(self, rows, rot: int, scale=None):
        import torch
        if rows.dim() != 3 or not rows.is_cuda or rows.stride(2) != 1:
            raise ValueError("rows must be a [n_pages, page_size, rank + rot] CUDA tensor with adjacent rows")
        pages, page, dim = rows.shape
        if not 0 < rot < dim:
            raise ValueError(f"rows of {dim} elements have no room for a shared key of {rot}")
        self.rows, self.scale = rows, scale
        self.c = c = kvr_latent_cache()
        if rows.dtype == torch.uint8:
            if scale is None:
                raise ValueError("a quantised cache needs its scales")
            if scale.dim() != 3 or tuple(scale.shape) != (pages, page, dim // BLOCK) or \
                    scale.dtype != torch.uint8 or not scale.is_cuda or scale.stride(2) != 1:
                raise ValueError("scale must be a [n_pages, page_size, (rank + rot) / 32] uint8 CUDA tensor "
                                 "with adjacent rows")
            if scale.device != rows.device:
                raise ValueError("the tensors of a cache must be on one device")
            c.format = KVR_KV_FP8
            c.scale = scale.data_ptr()
            c.scale_page_stride, c.scale_token_stride = scale.stride()[:2]
        elif rows.dtype in (torch.bfloat16, torch.float16):
            if scale is not None:
                raise ValueError("a 16-bit cache has no scales")
            c.format = KVR_KV_BF16 if rows.dtype == torch.bfloat16 else KVR_KV_FP16
        else:
            raise ValueError(f"a cache holds bfloat16, float16 or uint8, not {rows.dtype}")
        e = rows.element_size()
        c.data = rows.data_ptr()
        c.page_stride, c.token_stride = (e * x for x in rows.stride()[:2])
        c.n_pages, c.page_size, c.rank, c.rot = pages, page, dim - rot, rot
        self.n_pages, self.page_size, self.rank, self.rot = pages, page, dim - rot, rot
        self.format = c.format
        self.device = rows.device
        self.handle = (ctypes.addressof(c), rows, scale, c)   # what calls take

    @classmethod
    def allocate(cls, fmt: int, n_pages: int, page_size: int, rank: int, rot: int):
        """An empty cache (zeros) on the current device."""
        torch = kv._context().torch
        lead = (n_pages, page_size)
        if fmt in (KVR_KV_BF16, KVR_KV_FP16):
            dt = torch.bfloat16 if fmt == KVR_KV_BF16 else torch.float16
            return cls(torch.zeros(lead + (rank + rot,), dtype=dt, device="cuda"), rot)
        if fmt != KVR_KV_FP8:
            raise ValueError(f"a latent cache has no format {fmt}")
        new = [torch.zeros(lead + (n,), dtype=torch.uint8, device="cuda")
               for n in (rank + rot, (rank + rot) // BLOCK)]
        return cls(new[0], rot, new[1])

    @property
    def tensors(self):
        return self.rows, self.scale


def latent_bytes_per_token(fmt: int, layers: int, rank: int, rot: int) -> int:
    """Bytes of one token's rows over all layers, scale bytes included: the
    kv_bytes_per_token of kvr_prices_from_platform."""
    dim = rank + rot
    return layers * {KVR_KV_BF16: 2 * dim, KVR_KV_FP16: 2 * dim, KVR_KV_FP8: dim + dim // BLOCK}[fmt]


def kvr_latent_write(cache: LatentCache, latent, key, slots, positions=None, table=None,
                     norm_weight=None, eps: float = 1e-6, interleaved: bool = False,
                     adjoint: bool = False, status=None, stream=None, check: bool = True) -> None:
    """latent [tokens, rank] and key [tokens, rot] into ``slots`` [tokens] int64 (page *
    page_size + row; below 0: not written; each once).  With ``norm_weight`` [rank] (of the latents' type)
    latents are normalised, c w / sqrt(mean(c^2) + eps); with ``table`` keys are rotated by
    ``positions``; both in 32 bits on the way."""
    c = kv._context()
    if check:
        status = kv._status(c, cache, check, status, stream)
    rc, = c.fast.latent_write(cache.handle, latent, key, slots, positions, table, norm_weight, eps,
                              kv._flags(interleaved, adjoint), status, kv._handle(stream))
    if rc or check or stream is not None:
        kv._finish(c, "kvr_latent_write", rc, check, status, stream)


def kvr_latent_read(cache: LatentCache, slots, dtype=None, out=None, status=None, stream=None,
                    check: bool = True):
    """Rows [tokens, rank + rot] of ``slots`` [tokens] int64 in ``dtype`` (bfloat16 by default);
    below 0: zeros."""
    c = kv._context()
    if check:
        status = kv._status(c, cache, check, status, stream)
    if dtype is not None:
        if dtype not in c.codes:
            raise ValueError(f"out must be bfloat16, float16 or float32, not {dtype}")
        dtype = c.codes[dtype]
    rc, out = c.fast.latent_read(cache.handle, slots, dtype, out, status, kv._handle(stream))
    if rc or check or stream is not None:
        kv._finish(c, "kvr_latent_read", rc, check, status, stream, out)
    return out


def kvr_latent_attention(cache: LatentCache, q, cu_q, kv_len, page_table, max_q: int, max_kv: int,
                         scale: float, tree_mask=None, want_lse: bool = False, out=None,
                         workspace=None, status=None, stream=None, check: bool = True):
    """Attention of each sequence's newest tokens over its pages of the latent cache, in the
    latent's space.

    ``q`` [n_queries, n_heads, rank + rot]: each head's query times its key weight, then its
    rotated part; the other arguments as kvr_tree_attention's, but ``scale``, which the sizes of
    the cache do not tell.  Returns out [n_queries, n_heads, rank] (to be multiplied by each head's
    value weight), or (out, lse [n_queries, n_heads] float32) with ``want_lse``."""
    c = kv._context()
    if check:
        status = kv._status(c, cache, check, status, stream)
    rc, out, lse, ws = c.fast.latent_attention(cache.handle, q, cu_q, kv_len, page_table, max_q, max_kv,
                                               scale, tree_mask, want_lse, out, workspace, status,
                                               kv._handle(stream))
    if rc or check or stream is not None:
        kv._finish(c, "kvr_latent_attention", rc, check, status, stream, out, lse, ws)
    return (out, lse) if want_lse else out


def kvr_latent_prompt(q, k, k_rot, v, cu_q, cu_k, max_q: int, max_k: int, causal: bool = True,
                      scale: Optional[float] = None, want_lse: bool = False, out=None,
                      workspace=None, status=None, stream=None, check: bool = True):
    """Attention of prompts, or of their next chunks, over keys and values of each head.

    ``q`` [n_queries, n_q_heads, nope + rot]; ``k``, ``v`` [n_keys, n_kv_heads, nope]; ``k_rot``
    [n_keys, rot], shared by all heads; ``cu_q``, ``cu_k`` [n_seqs + 1] int32, first query and
    first key of each sequence; ``max_q``, ``max_k``: bounds on a sequence's.  With ``causal`` a
    sequence's queries are its last keys' tokens, and each sees the keys up to its own.  ``scale``
    defaults to (nope + rot) ** -0.5.  Returns out [n_queries, n_q_heads, nope], or (out, lse
    [n_queries, n_q_heads] float32) with ``want_lse``."""
    c = kv._context()
    if check:
        status = kv._status(c, q, check, status, stream)
    rc, out, lse, ws = c.fast.latent_prompt(q, k, k_rot, v, cu_q, cu_k, max_q, max_k, causal, scale,
                                            want_lse, out, workspace, status, kv._handle(stream))
    if rc or check or stream is not None:
        kv._finish(c, "kvr_latent_prompt", rc, check, status, stream, out, lse, ws)
    return (out, lse) if want_lse else out
