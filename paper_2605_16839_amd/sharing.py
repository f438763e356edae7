"""Requests that share pages of a paged cache (section 6 of include/compactattn.h).

``page_shares`` int32 ``[num_pages]`` counts, for every page, the requests that hold it
besides the first: zeros at the start.  ``assign_slots`` goes on from what these calls leave;
requests that may share pages end here (``parent[b] = -1``), not by ``release_pages``.

    cache = ca.Cache(...)
    shares = torch.zeros(cache.num_pages, dtype=torch.int32, device="cuda")
    state = dict(seq_len=seq_len, page_table=page_table, page_shares=shares,
                 free_pages=free_pages, free_count=free_count)
    ca.sharing.fork_requests(cache, parent, **state, kv_pool=pools, bufs=dict(state))   # in place
    share_len = seq_len[:1].clone()   # what all have in common: as it is at the fork
    # a step's tokens: assign_slots, rotary_append
    out, _ = ca.sharing.prefix_decode_attention(cache, q, pools, page_table, seq_len, share,
                                                share_len, sm_scale)

Every call is enqueued on torch's current stream, or on ``stream=``.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from .binding import Cache, _check, _here, _nbytes, _need, _on, load

__all__ = ["fork_workspace_bytes", "fork_requests", "compact_workspace_bytes", "compact_pages",
           "prefix_decode_workspace_bytes", "prefix_decode_attention"]


def _workspace(ws: Optional[torch.Tensor], nbytes: int, like: torch.Tensor, index: int):
    if ws is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=like.device) if nbytes else None
    if ws.get_device() != index or not ws.is_contiguous():
        raise ValueError(f"ws must be contiguous on cuda:{index}")
    return ws


def _pool_ptrs(c: Cache, kv_pool, index: int):
    return (_need("k_pool", kv_pool[0], torch.bfloat16, c._k_pool, index),
            _need("v_pool", kv_pool[1], torch.bfloat16, c._v_pool, index))


def _state(c: Cache, given: dict, bufs: Optional[dict], names: Tuple[str, ...], index: int):
    """Addresses of the state before (``given``) and after the call (``bufs``, made where missing)."""
    shapes = dict(seq_len=(c.batch,), page_table=c._table, page_shares=(c.num_pages,),
                  free_pages=(given["free_pages"].numel(),), free_count=(1,), new_page=(c.num_pages,))
    before = {k: None if t is None else _need(k, t, torch.int32, shapes[k], index) for k, t in given.items()}
    b = bufs if bufs is not None else {}
    for k in names:
        if k not in b and not (k in given and given[k] is None):
            b[k] = torch.full(shapes[k], -1, dtype=torch.int32, device=given["free_pages"].device)
    after = {k: _need(k, b[k], torch.int32, shapes[k], index) if b.get(k) is not None else None for k in names}
    return before, after, b


def fork_workspace_bytes(c: Cache) -> int:
    return load().ca_fork_workspace_bytes(c.ref)


def fork_requests(c: Cache, parent: torch.Tensor, seq_len: torch.Tensor, page_table: torch.Tensor,
                  page_shares: torch.Tensor, free_pages: torch.Tensor, free_count: torch.Tensor,
                  kv_pool: Tuple[torch.Tensor, torch.Tensor],
                  keep_len: Optional[torch.Tensor] = None, bufs: Optional[dict] = None,
                  ws: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Request b goes on from request parent[b] as it was (-1: it ends), with its first keep_len[b]
    tokens (None: all): whole pages are shared, a part-filled last one is copied where someone else has it
    too, and pages that no one holds any more become free.

    Returns ``bufs`` (made where missing): int32 seq_len, page_table, page_shares, free_pages and
    free_count after it; each may be the input itself."""
    if stream is not None:
        return _on(stream, fork_requests, locals())
    index, st = _here(parent)
    names = ("seq_len", "page_table", "page_shares", "free_pages", "free_count")
    given = dict(zip(names, (seq_len, page_table, page_shares, free_pages, free_count)))
    at, to, b = _state(c, given, bufs, names, index)
    k, v = _pool_ptrs(c, kv_pool, index)
    ws = _workspace(ws, fork_workspace_bytes(c) if ws is None else 0, parent, index)
    _check(load().ca_fork_requests(
        c.ref, _need("parent", parent, torch.int32, (c.batch,), index),
        None if keep_len is None else _need("keep_len", keep_len, torch.int32, (c.batch,), index),
        at["seq_len"], at["page_table"], at["page_shares"], at["free_pages"], free_pages.numel(),
        at["free_count"], k, v, to["seq_len"], to["page_table"], to["page_shares"], to["free_pages"],
        to["free_count"], None if ws is None else ws.data_ptr(), _nbytes(ws), st))
    return b


def compact_workspace_bytes(c: Cache) -> int:
    return load().ca_compact_workspace_bytes(c.ref)


def compact_pages(c: Cache, seq_len: torch.Tensor, page_table: torch.Tensor,
                  page_shares: Optional[torch.Tensor], free_pages: torch.Tensor,
                  free_count: torch.Tensor, kv_pool: Tuple[torch.Tensor, torch.Tensor],
                  bufs: Optional[dict] = None, ws: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Moves the pages in use (those that are not in the free list) to the lowest ids.

    Returns ``bufs`` (made where missing): int32 page_table, page_shares (None without),
    free_pages and free_count after it, each of which may be the input itself, and new_page
    [num_pages], where each page is now (-1: free)."""
    if stream is not None:
        return _on(stream, compact_pages, locals())
    index, st = _here(seq_len)
    names = ("page_table", "page_shares", "free_pages", "free_count")
    given = dict(zip(names, (page_table, page_shares, free_pages, free_count)), seq_len=seq_len)
    at, to, b = _state(c, given, bufs, names + ("new_page",), index)
    if (at["page_shares"] is None) != (to["page_shares"] is None):
        raise ValueError("page_shares before and after the call come together")
    k, v = _pool_ptrs(c, kv_pool, index)
    ws = _workspace(ws, compact_workspace_bytes(c) if ws is None else 0, seq_len, index)
    _check(load().ca_compact_pages(
        c.ref, at["seq_len"], at["page_table"], at["page_shares"], at["free_pages"],
        free_pages.numel(), at["free_count"], k, v, to["new_page"], to["page_table"],
        to["page_shares"], to["free_pages"], to["free_count"],
        None if ws is None else ws.data_ptr(), _nbytes(ws), st))
    return b


def prefix_decode_workspace_bytes(c: Cache, num_shares: int) -> int:
    return load().ca_prefix_decode_workspace_bytes(c.ref, num_shares)


def prefix_decode_attention(c: Cache, q: torch.Tensor, kv_pool: Tuple[torch.Tensor, torch.Tensor],
                            page_table: torch.Tensor, kv_len: torch.Tensor, share: torch.Tensor,
                            share_len: torch.Tensor, sm_scale: float,
                            out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                            ws: Optional[torch.Tensor] = None, stream=None):
    """``decode_attention`` for requests that share prefixes: share[b] names the share of request b (-1:
    none), whose first share_len[share[b]] tokens it has in common with the share's others; their whole
    pages are read once for all of them.  After a fork that is the length at the fork: tokens that a
    request adds later are its own, and a share_len that counts them reads the first member's for all.
    Where the prefixes read again for every request would be less than some 100 to 250 MB,
    ``decode_attention`` is faster.
    Returns (out bf16, lse fp32 or None)."""
    if stream is not None:
        return _on(stream, prefix_decode_attention, locals())
    index, st = _here(q)
    bf, i32, shares = torch.bfloat16, torch.int32, share_len.numel()
    shape = (c.batch, c.num_q_heads, c.head_dim)
    qp = _need("q", q, bf, shape, index)
    if out is None:
        out = torch.empty_like(q)
    ws = _workspace(ws, prefix_decode_workspace_bytes(c, shares) if ws is None else 0, q, index)
    k, v = _pool_ptrs(c, kv_pool, index)
    _check(load().ca_prefix_decode_attention(
        c.ref, qp, k, v, _need("page_table", page_table, i32, c._table, index),
        _need("kv_len", kv_len, i32, (c.batch,), index),
        _need("share", share, i32, (c.batch,), index),
        _need("share_len", share_len, i32, (shares,), index), shares, sm_scale,
        _need("out", out, bf, shape, index),
        None if lse is None else _need("lse", lse, torch.float32, shape[:2], index),
        None if ws is None else ws.data_ptr(), _nbytes(ws), st))
    return out, lse
