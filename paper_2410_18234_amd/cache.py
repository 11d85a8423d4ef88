"""The paged 8-bit cache of keys and values: its pool and the calls on it.

A decoding loop holds a ``PagedCache`` (the pool of pages, for all layers), and for its sequences a page table
``[S][width]`` int32, lengths ``[S]`` int32 and reference counts ``[pages]`` int32 (0: a free page):

    table, lengths, refs = cache_fork(cache, table, lengths, refs, parent, grow=grow)   # once a step
    for layer in range(layers):
        cache_append(cache, layer, k, v, starts, table, lengths)                        # the new tokens
        out = cache_attention(q, cache, layer, starts, table, lengths)                  # over all of them

New tokens are ragged: sequence s owns tokens ``starts[s] .. starts[s + 1] - 1`` of q, k and v (``starts`` None: as
many for each), the last of its ``lengths[s]`` tokens.
"""
from __future__ import annotations

import math
import struct
from typing import Optional

import torch

from .binding import _check, _need, _ptr, _stream, _ws_arg, load_library

_DTYPES = {torch.bfloat16: 1, torch.float16: 2}


# mdss_cache of the C ABI: k, v, k_exp, v_exp, pages, layers, heads, head_dim, page_size
_DESC = struct.Struct("PPPPqiiii")


class PagedCache:
    """A pool of pages: e4m3 codes of keys and values, and an int8 exponent for each layer, page and head.

    k      [layers][pages][heads][page_size / 16][head_dim / 16][16][16]  uint8 (unit, 16 of head_dim, token)
    v      [layers][pages][heads][page_size / 16][head_dim][16]           uint8 (unit, head_dim, token)
    k_exp, v_exp [layers][pages][heads]                                   int8; a value is code * 2**exp

    The calls go by the addresses that the tensors had here: the attributes cannot be set anew, and the tensors are not to be
    given other memory (``set_``, ``resize_``).
    """

    __slots__ = ("k", "v", "k_exp", "v_exp", "layers", "pages", "heads", "head_dim", "page_size", "device", "_ref")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor):
        shape = k.shape
        if len(shape) != 7 or shape[5] != 16 or shape[6] != 16:
            raise ValueError("k must be [layers][pages][heads][page_size / 16][head_dim / 16][16][16]")
        if not k.is_cuda:
            raise ValueError("k must be a GPU tensor")
        layers, pages, heads, units, chunks = shape[:5]
        device = k.device
        _need(k, "k", torch.uint8, shape, device)
        _need(v, "v", torch.uint8, (layers, pages, heads, units, 16 * chunks, 16), device)
        _need(k_exp, "k_exp", torch.int8, (layers, pages, heads), device)
        _need(v_exp, "v_exp", torch.int8, (layers, pages, heads), device)
        ref = _DESC.pack(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(), pages, layers, heads,
                         16 * chunks, 16 * units)
        for name, x in zip(self.__slots__, (k, v, k_exp, v_exp, layers, pages, heads, 16 * chunks, 16 * units, device, ref)):
            object.__setattr__(self, name, x)

    def __setattr__(self, name, value):
        raise AttributeError(f"a PagedCache keeps its {name}: make another one of the new tensors")

    def __delattr__(self, name):
        raise AttributeError(f"a PagedCache keeps its {name}")

    def __reduce__(self):  # copies go by their own tensors' addresses
        return PagedCache, (self.k, self.v, self.k_exp, self.v_exp)

    @classmethod
    def empty(cls, layers: int, pages: int, heads: int, head_dim: int, page_size: int = 64,
              device: torch.device = "cuda") -> "PagedCache":
        """A pool with nothing in it."""
        if head_dim % 16 or page_size % 16:
            raise ValueError("head_dim and page_size must be multiples of 16")
        lead = (layers, pages, heads)
        return cls(torch.zeros(lead + (page_size // 16, head_dim // 16, 16, 16), dtype=torch.uint8, device=device),
                   torch.zeros(lead + (page_size // 16, head_dim, 16), dtype=torch.uint8, device=device),
                   torch.full(lead, -40, dtype=torch.int8, device=device),
                   torch.full(lead, -40, dtype=torch.int8, device=device))


def _rows(cache: PagedCache, starts: Optional[torch.Tensor], table: torch.Tensor, lengths: torch.Tensor):
    if table.dim() != 2:
        raise ValueError("table must be [S][width]")
    S, width = table.shape
    _need(table, "table", torch.int32, (S, width), cache.device)
    _need(lengths, "lengths", torch.int32, (S,), cache.device)
    if starts is not None:
        _need(starts, "starts", torch.int32, (S + 1,), cache.device)
    return S, width


def _tokens(x: torch.Tensor, name: str, cache: PagedCache, dtype: Optional[torch.dtype] = None):
    """x is [T][heads][head_dim], its last dimension contiguous; the others may have any stride."""
    if x.dim() != 3 or x.shape[2] != cache.head_dim:
        raise ValueError(f"{name} must be [T][heads][{cache.head_dim}]")
    if x.dtype not in _DTYPES or (dtype is not None and x.dtype != dtype):
        raise TypeError(f"{name} must be {dtype or 'torch.bfloat16 or torch.float16'}, got {x.dtype}")
    if x.device != cache.device:
        raise ValueError(f"{name} must be on {cache.device}, got {x.device}")
    if x.stride(2) != 1 and x.numel():
        raise ValueError(f"{name}'s last dimension must be contiguous")


def _status(row_status: Optional[torch.Tensor], S: int, device: torch.device):
    if row_status is not None:
        _need(row_status, "row_status", torch.int32, (S,), device)


def _scratch(device: torch.device, need: int, workspace: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    return None if workspace is None and not need else _ws_arg(device, need, workspace)


def cache_append(cache: PagedCache, layer: int, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor],
                 table: torch.Tensor, lengths: torch.Tensor, row_status: Optional[torch.Tensor] = None) -> None:
    """Rounds the new tokens' keys and values ``[T][heads][head_dim]`` into their pages of ``layer``."""
    lib = load_library()
    S, width = _rows(cache, starts, table, lengths)
    _tokens(k, "k", cache)
    _tokens(v, "v", cache, k.dtype)
    T = k.shape[0]
    if k.shape[1] != cache.heads or v.shape != k.shape:
        raise ValueError(f"k and v must be [T][{cache.heads}][{cache.head_dim}]")
    _status(row_status, S, cache.device)
    _check("mdss_cache_append",
           lib.mdss_cache_append(cache._ref, layer, _ptr(k), k.stride(0), k.stride(1), _ptr(v), v.stride(0),
                                 v.stride(1), _DTYPES[k.dtype], T, _ptr(starts), _ptr(table), width, _ptr(lengths), S,
                                 _ptr(row_status), _stream(cache.device)))


def cache_attention(q: torch.Tensor, cache: PagedCache, layer: int, starts: Optional[torch.Tensor],
                    table: torch.Tensor, lengths: torch.Tensor, scale: Optional[float] = None, max_new: int = 0,
                    max_length: int = 0, want_lse: bool = False, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None):
    """Attention of the new tokens ``q [T][heads_q][head_dim]`` over their sequences' cached tokens up to their own.

    ``scale`` defaults to ``head_dim ** -0.5``.  ``max_new`` and ``max_length`` (0: unknown) say how many new tokens
    and how many tokens a sequence has at most; they only choose how the work is cut.  Returns ``out`` (q's type), or
    ``(out, lse)`` with ``want_lse``; tokens of q that belong to no sequence are not written there."""
    lib = load_library()
    S, width = _rows(cache, starts, table, lengths)
    _tokens(q, "q", cache)
    T, heads_q = q.shape[0], q.shape[1]
    dev = cache.device
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        _need(out, "out", q.dtype, (T, heads_q, cache.head_dim), dev)
    lse = torch.empty((T, heads_q), dtype=torch.float32, device=dev) if want_lse else None
    need = lib.mdss_workspace_bytes_attention(cache._ref, T, S, width, heads_q, starts is None, max_new, max_length)
    workspace = _scratch(dev, need, workspace)
    _check("mdss_cache_attention",
           lib.mdss_cache_attention(cache._ref, layer, _ptr(q), q.stride(0), q.stride(1), _DTYPES[q.dtype], T, heads_q,
                                    _ptr(starts), _ptr(table), width, _ptr(lengths), S,
                                    1.0 / math.sqrt(cache.head_dim) if scale is None else scale, max_new, max_length,
                                    _ptr(out), _ptr(lse), _ptr(workspace),
                                    workspace.numel() if workspace is not None else 0, _stream(dev)))
    return (out, lse) if want_lse else out


def cache_fork(cache: PagedCache, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor,
               parent: Optional[torch.Tensor] = None, keep: Optional[torch.Tensor] = None,
               grow: Optional[torch.Tensor] = None, row_status: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None):
    """(table, lengths, refs) of rows that take over their parents' and get room for ``grow`` more tokens.

    Row i holds the first ``keep[i]`` tokens (None: all) of row ``parent[i]`` (None: row i; -1: nothing, its pages are
    given back), and pages for ``grow[i]`` more; a partly filled page that others hold is replaced by a copy.  Rows
    for which there is no page are flagged MDSS_ROW_NO_PAGE and do not grow (none does if the pool lacks the
    pages for all)."""
    lib = load_library()
    S, width = _rows(cache, None, table, lengths)
    dev = cache.device
    _need(refs, "refs", torch.int32, (cache.pages,), dev)
    S_out = S if parent is None else parent.shape[0]
    for name, x in (("parent", parent), ("keep", keep), ("grow", grow)):
        if x is not None:
            _need(x, name, torch.int32, (S_out,), dev)
    _status(row_status, S_out, dev)
    table_out = torch.empty_strided((S_out, width), (width, 1), dtype=torch.int32, device=dev)
    lengths_out = torch.empty_strided((S_out,), (1,), dtype=torch.int32, device=dev)
    refs_out = torch.empty_like(refs)
    workspace = _scratch(dev, lib.mdss_workspace_bytes_cache_fork(cache._ref, S_out), workspace)
    _check("mdss_cache_fork",
           lib.mdss_cache_fork(cache._ref, _ptr(table), _ptr(lengths), S, width, _ptr(refs), _ptr(parent), _ptr(keep),
                               _ptr(grow), S_out, _ptr(table_out), _ptr(lengths_out), _ptr(refs_out), _ptr(row_status),
                               _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream(dev)))
    return table_out, lengths_out, refs_out


def cache_compact(cache: PagedCache, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor,
                  workspace: Optional[torch.Tensor] = None):
    """(table, refs, used): the used pages moved to the ids 0 .. used - 1 (``used`` a one-element int32 tensor).

    What moves goes by ``refs``: every table that holds pages of the pool has to follow, as rows of this one (rows that
    list all ids come back as the map from old to new ids, -1 for free pages)."""
    lib = load_library()
    S, width = _rows(cache, None, table, lengths)
    dev = cache.device
    _need(refs, "refs", torch.int32, (cache.pages,), dev)
    table_out, refs_out = torch.empty_like(table), torch.empty_like(refs)
    used = torch.empty_strided((), (), dtype=torch.int32, device=dev)
    workspace = _scratch(dev, lib.mdss_workspace_bytes_cache_compact(cache._ref), workspace)
    _check("mdss_cache_compact",
           lib.mdss_cache_compact(cache._ref, _ptr(table), _ptr(lengths), S, width, _ptr(refs), _ptr(table_out),
                                  _ptr(refs_out), _ptr(used), _ptr(workspace),
                                  workspace.numel() if workspace is not None else 0, _stream(dev)))
    return table_out, refs_out, used


def cache_copy(cache: PagedCache, src: torch.Tensor, dst: torch.Tensor) -> None:
    """Copies pages ``src[i]`` to ``dst[i]`` (int32 ids) in every layer."""
    lib = load_library()
    if src.dim() != 1:
        raise ValueError("src must be [n]")
    _need(src, "src", torch.int32, tuple(src.shape), cache.device)
    _need(dst, "dst", torch.int32, tuple(src.shape), cache.device)
    _check("mdss_cache_copy",
           lib.mdss_cache_copy(cache._ref, _ptr(src), _ptr(dst), src.shape[0], _stream(cache.device)))
