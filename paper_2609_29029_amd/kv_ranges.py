"""Attention over ranges of the paged key-value cache (include/rift_kv.h): after a prefix that
all sequences share, and over the pages that promise the largest scores.

Argument marshalling only, as in kv: the same tensors, checks and errors."""
from __future__ import annotations

from typing import Optional

from . import kv
from ._lib import _check
from .kv import KvCache, _dense, _elsewhere, _row_type, _rows, _stream


def _tensors(cache, q, page_table, lens, status):
    """What the calls below have in common: (device, row type, the table's shape, q's address and stride)."""
    dev, i32 = cache.device, kv._I32
    n_seq, max_pages = page_table.shape
    dt = kv._ROWS.get(q.dtype)
    if dt is None:
        _row_type(q, "q")
    pq, ldq = _rows(q, q.dtype, (n_seq, q.shape[1], cache.head_dim), dev, "q")
    if page_table.dtype is not i32 or not page_table.is_contiguous() or page_table.get_device() != dev:
        _dense(page_table, i32, None, dev, "page_table")
    if lens.dtype is not i32 or lens.shape != (n_seq,) or not lens.is_contiguous() or lens.get_device() != dev:
        _dense(lens, i32, (n_seq,), dev, "lens")
    if status.dtype is not i32 or status.shape != (1,) or status.get_device() != dev:
        _dense(status, i32, (1,), dev, "status")
    return dev, dt, n_seq, max_pages, pq, ldq


def _call(name, dev, stream, *args):
    fn = getattr(kv._lib, name)
    st = kv._raw_stream(dev) or None if stream is None else _stream(stream, dev)
    st = fn(*args, st) if dev == kv._device() else _elsewhere(dev, fn, *args, st)
    if st:
        _check(st, name)


# ----------------------------------------------------------------------------- a shared prefix
def riftkv_attention_shared_workspace_size(cache: KvCache, n_seq: int, n_heads: int, prefix_len: int, max_pages: int) -> int:
    return int(kv._lib.riftkv_attention_shared_workspace_size(cache.ref, int(n_heads), int(n_seq), int(prefix_len), int(max_pages)))


def riftkv_attention_shared(cache: KvCache, q, prefix_table, prefix_len: int, page_table, lens, out, workspace, status,
                            scale: Optional[float] = None, stream=None) -> None:
    """out[i] := attention of q[i] [n_heads][head_dim] over the prefix_len tokens of the pages prefix_table [pages] i32
    and then the first lens[i] tokens of sequence i's own pages; scale None: 1 / sqrt(head_dim)."""
    dev, dt, n_seq, max_pages, pq, ldq = _tensors(cache, q, page_table, lens, status)
    prefix_len = int(prefix_len)
    if prefix_table.dim() != 1 or prefix_table.shape[0] * cache.page_size < prefix_len:
        raise ValueError("prefix_table: expected the pages of prefix_len tokens")
    front = _dense(prefix_table, kv._I32, None, dev, "prefix_table")
    po, ldo = _rows(out, q.dtype, q.shape, dev, "out")
    ws = _dense(workspace, kv._U8, None, dev, "workspace")
    _call("riftkv_attention_shared", dev, stream, cache.ref, pq, ldq, q.shape[1], dt, front, prefix_len, page_table.data_ptr(), n_seq,
          max_pages, lens.data_ptr(), cache.head_dim ** -0.5 if scale is None else scale, po, ldo, status.data_ptr(), ws,
          workspace.numel())


# ----------------------------------------------------------------------------- some pages of a long context
def riftkv_page_bounds(cache: KvCache, bounds, page_table, lens, status, begins=None, stream=None) -> None:
    """bounds [n_pages][n_kv_heads][2][head_dim] (float32 with float32 pages, else bf16) := the smallest and largest key values
    of the pages that hold tokens begins[i] (None: 0) .. lens[i] - 1 of every sequence."""
    dev, i32 = cache.device, kv._I32
    n_seq, max_pages = page_table.shape
    to = _dense(bounds, kv.torch.float32 if cache.dt == kv.RIFTKV_F32 else kv.torch.bfloat16,
                (cache.n_pages, cache.n_kv_heads, 2, cache.head_dim), dev, "bounds")
    table = _dense(page_table, i32, None, dev, "page_table")
    n = _dense(lens, i32, (n_seq,), dev, "lens")
    first = None if begins is None else _dense(begins, i32, (n_seq,), dev, "begins")
    word = _dense(status, i32, (1,), dev, "status")
    _call("riftkv_page_bounds", dev, stream, cache.ref, to, table, n_seq, max_pages, first, n, word)


def riftkv_select_pages_workspace_size(cache: KvCache, n_seq: int, max_pages: int) -> int:
    return int(kv._lib.riftkv_select_pages_workspace_size(cache.ref, int(n_seq), int(max_pages)))


def riftkv_select_pages(cache: KvCache, bounds, q, page_table, lens, pages, workspace, status, keep_first: int = 1,
                        keep_last: int = 1, stream=None) -> None:
    """pages [n_seq][n_kv_heads][top] i32 := the places in its row of page_table of the `top` pages that each sequence's
    token needs most of each key head, ascending, -1 behind them; the first keep_first and last keep_last always."""
    dev, dt, n_seq, max_pages, pq, ldq = _tensors(cache, q, page_table, lens, status)
    of = _dense(bounds, kv.torch.float32 if cache.dt == kv.RIFTKV_F32 else kv.torch.bfloat16,
                (cache.n_pages, cache.n_kv_heads, 2, cache.head_dim), dev, "bounds")
    if pages.dim() != 3:
        raise ValueError("pages: expected [n_seq][n_kv_heads][top]")
    to = _dense(pages, kv._I32, (n_seq, cache.n_kv_heads, pages.shape[2]), dev, "pages")
    ws = _dense(workspace, kv._U8, None, dev, "workspace")
    _call("riftkv_select_pages", dev, stream, cache.ref, of, pq, ldq, q.shape[1], dt, page_table.data_ptr(), n_seq, max_pages,
          lens.data_ptr(), int(keep_first), int(keep_last), to, pages.shape[2], status.data_ptr(), ws, workspace.numel())


def riftkv_attention_pages_workspace_size(cache: KvCache, n_seq: int, n_heads: int, top: int) -> int:
    return int(kv._lib.riftkv_attention_pages_workspace_size(cache.ref, int(n_heads), int(n_seq), int(top)))


def riftkv_attention_pages(cache: KvCache, q, page_table, lens, pages, out, workspace, status, scale: Optional[float] = None,
                           stream=None) -> None:
    """out[i] := attention of q[i] [n_heads][head_dim] over the tokens before lens[i] of the pages listed for it:
    pages [n_seq][n_kv_heads][top] i32, places in sequence i's row of page_table; scale None: 1 / sqrt(head_dim)."""
    dev, dt, n_seq, max_pages, pq, ldq = _tensors(cache, q, page_table, lens, status)
    if pages.dim() != 3:
        raise ValueError("pages: expected [n_seq][n_kv_heads][top]")
    of = _dense(pages, kv._I32, (n_seq, cache.n_kv_heads, pages.shape[2]), dev, "pages")
    po, ldo = _rows(out, q.dtype, q.shape, dev, "out")
    ws = _dense(workspace, kv._U8, None, dev, "workspace")
    _call("riftkv_attention_pages", dev, stream, cache.ref, pq, ldq, q.shape[1], dt, page_table.data_ptr(), n_seq, max_pages,
          lens.data_ptr(), of, pages.shape[2], cache.head_dim ** -0.5 if scale is None else scale, po, ldo, status.data_ptr(), ws,
          workspace.numel())
