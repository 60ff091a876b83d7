"""The paged key-value cache (include/rift_kv.h): rotary positions, rows into
pages and out of them, attention of one new token a sequence.

Argument marshalling only, as in _lib: tensors are checked, raw pointers and the
stream go to the C ABI, and a non-OK status raises RiftError.  Rows are
[rows][heads][head_dim] tensors whose heads and elements are contiguous; the
rows themselves may be any stride apart (slices of a projection).  All tensors
of a call are on one device, which need not be the current one."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from ._lib import RIFT_BF16, RIFT_F32, LayerWeights, ModelCfg, _check, layer_struct, load

RIFTKV_F32, RIFTKV_BF16, RIFTKV_FP8, RIFTKV_INT8 = 0, 1, 2, 3
# Every symbol include/rift_kv.h declares, in declaration order.
KV_EXPORTS = ("riftkv_abi_version", "riftkv_rope_freqs", "riftkv_rope", "riftkv_rope_axes", "riftkv_write", "riftkv_read",
              "riftkv_attention_workspace_size", "riftkv_attention", "riftkv_attention_shared_workspace_size",
              "riftkv_attention_shared", "riftkv_page_bounds", "riftkv_select_pages_workspace_size",
              "riftkv_select_pages", "riftkv_attention_pages_workspace_size", "riftkv_attention_pages",
              "riftkv_decode_workspace_size", "riftkv_decode_step")
ROPE_SCALINGS = ("none", "linear", "base", "ramp", "bands")
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}


class _CacheStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")] + \
        [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "dt")]


class _RopeStruct(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int32)] + \
        [(n, ctypes.c_double) for n in ("base", "factor", "original_len", "low", "high")]


_lib: Optional[ctypes.CDLL] = None
# Set by the first call: importing the package does not import torch.
torch = _ROWS = _STORES = _I32 = _U8 = _F8 = _I4 = _device = _raw_stream = None


def _load() -> ctypes.CDLL:
    global _lib, torch, _ROWS, _STORES, _I32, _U8, _F8, _I4, _device, _raw_stream
    if _lib is None:
        import numpy as np
        import torch as t
        _F8, _I4 = np.dtype("<f8"), np.dtype("<i4")
        torch, _I32, _U8 = t, t.int32, t.uint8
        _device, _raw_stream = t._C._cuda_getDevice, t._C._cuda_getCurrentRawStream
        _ROWS = {t.bfloat16: RIFT_BF16, t.float32: RIFT_F32}
        _STORES = {t.float32: RIFTKV_F32, t.bfloat16: RIFTKV_BF16, t.float8_e4m3fn: RIFTKV_FP8, t.int8: RIFTKV_INT8}
        L = load()
        P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        F32, F64 = ctypes.c_float, ctypes.c_double
        L.riftkv_abi_version.restype = I32
        L.riftkv_abi_version.argtypes = []
        L.riftkv_rope_freqs.restype = I32
        L.riftkv_rope_freqs.argtypes = [P, P, P]
        L.riftkv_rope.restype = I32
        L.riftkv_rope.argtypes = [P, I64, I32, P, I64, P, I64, I32, P, I64, I32, P, I32, I32, I32, I32, P, F64, P]
        L.riftkv_rope_axes.restype = I32
        L.riftkv_rope_axes.argtypes = [P, I64, I32, P, I64, P, I64, I32, P, I64, I32, P, I32, I32, I32, I32, I32, P, P, F64, P]
        for name in ("riftkv_write", "riftkv_read"):
            getattr(L, name).restype = I32
            getattr(L, name).argtypes = [P, P, I64, P, I64, I32, P, I32, I32, P, P, I32, P, P]
        L.riftkv_attention_workspace_size.restype = SZ
        L.riftkv_attention_workspace_size.argtypes = [P, I32, I32, I32]
        L.riftkv_attention.restype = I32
        L.riftkv_attention.argtypes = [P, P, I64, I32, I32, P, I32, I32, P, F32, P, I64, P, P, SZ, P]
        L.riftkv_attention_shared_workspace_size.restype = SZ
        L.riftkv_attention_shared_workspace_size.argtypes = [P, I32, I32, I32, I32]
        L.riftkv_attention_shared.restype = I32
        L.riftkv_attention_shared.argtypes = [P, P, I64, I32, I32, P, I32, P, I32, I32, P, F32, P, I64, P, P, SZ, P]
        L.riftkv_page_bounds.restype = I32
        L.riftkv_page_bounds.argtypes = [P, P, P, I32, I32, P, P, P, P]
        L.riftkv_select_pages_workspace_size.restype = SZ
        L.riftkv_select_pages_workspace_size.argtypes = [P, I32, I32]
        L.riftkv_select_pages.restype = I32
        L.riftkv_select_pages.argtypes = [P, P, P, I64, I32, I32, P, I32, I32, P, I32, I32, P, I32, P, P, SZ, P]
        L.riftkv_attention_pages_workspace_size.restype = SZ
        L.riftkv_attention_pages_workspace_size.argtypes = [P, I32, I32, I32]
        L.riftkv_attention_pages.restype = I32
        L.riftkv_attention_pages.argtypes = [P, P, I64, I32, I32, P, I32, I32, P, P, I32, F32, P, I64, P, P, SZ, P]
        L.riftkv_decode_workspace_size.restype = SZ
        L.riftkv_decode_workspace_size.argtypes = [P, P, I32, I32]
        L.riftkv_decode_step.restype = I32
        L.riftkv_decode_step.argtypes = [P, P, P, P, P, I32, I32, P, P, P, P, SZ, P]
        _lib = L
    return _lib


# ----------------------------------------------------------------------------- checks
# A call's checks are part of its cost: devices are compared by index, and what the calls of a decode
# step check of each tensor stands in them in line (a write 7.3 -> 6.7 us a call, 3.1 of it the launch); these functions then say what is
# wrong, or that nothing is.
def _int32(x, name):
    """A number that the C ABI takes in 32 bits: ctypes would cut a larger one off."""
    if not -0x80000000 <= x <= 0x7FFFFFFF:
        raise ValueError(f"{name}: {x} does not fit 32 bits")
    return x


def _too_many():
    raise ValueError("more rows, heads, sequences or pages than 31 bits count")


def _dense(t, dtype, shape, device, name):
    """Address of a contiguous device tensor; shape None: any."""
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if t.get_device() != device:
        raise ValueError(f"{name}: must be on device {device}")
    return t.data_ptr()


def _rows(t, dtype, shape, device, name):
    """[rows][heads][head_dim], the last two contiguous: (address, elements between rows)."""
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name}: must be on device {device}")
    n, heads, hd = shape
    ld, sh, se = t.stride()
    if (se != 1 and hd > 1) or (sh != hd and heads > 1):
        raise ValueError(f"{name}: heads and elements must be contiguous")
    return t.data_ptr(), (ld if n > 1 else heads * hd)


def _device_of(t, name):
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a device tensor")
    return t.get_device()


def _row_type(t, name):
    dt = _ROWS.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}")
    return dt


def _stream(stream, device):
    if stream.device.index != device:
        raise ValueError(f"stream: must be on device {device}")
    return stream.cuda_stream or None


def _elsewhere(device, fn, *args):
    """fn with `device` as the current one."""
    with torch.cuda.device(device):
        return fn(*args)


# ----------------------------------------------------------------------------- the pages
class KvCache:
    """One layer's pages, or several layers', as riftkv_cache made them: what the calls
    take.  riftkv_decode_step goes through all layers, the others act on the first;
    layer(l) is layer l on its own."""

    def __init__(self, k, v, k_scale, v_scale):
        _load()
        dev = _device_of(k, "k")
        dt = _STORES.get(k.dtype)
        if dt is None:
            raise TypeError(f"k: unsupported storage dtype {k.dtype}")
        shape = tuple(k.shape)
        if len(shape) not in (4, 5) or 0 in shape:
            raise ValueError("k: expected [n_pages][n_kv_heads][page_size][head_dim], or several layers of these")
        scaled = dt in (RIFTKV_FP8, RIFTKV_INT8)
        if scaled != (k_scale is not None) or scaled != (v_scale is not None):
            raise ValueError("k_scale and v_scale go with 8-bit pages, and only with them")
        p = [_dense(k, k.dtype, shape, dev, "k"), _dense(v, k.dtype, shape, dev, "v"), None, None]
        if scaled:
            p[2] = _dense(k_scale, torch.uint8, shape[:-1], dev, "k_scale")
            p[3] = _dense(v_scale, torch.uint8, shape[:-1], dev, "v_scale")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self.dt = dev, dt
        self.n_layers = shape[0] if len(shape) == 5 else 1
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = shape[-4:]
        self.struct = _CacheStruct(*p, shape[-4], shape[-2], shape[-3], shape[-1], dt)
        self.ref = ctypes.byref(self.struct)

    def layer(self, l: int) -> "KvCache":
        if self.k.dim() == 4:
            if l != 0:
                raise IndexError(f"layer {l} of 1")
            return self
        return KvCache(*(None if t is None else t[l] for t in (self.k, self.v, self.k_scale, self.v_scale)))


def riftkv_cache(k, v, k_scale=None, v_scale=None) -> KvCache:
    """A handle on pages k, v [n_pages][n_kv_heads][page_size][head_dim], or [n_layers] of
    these (bf16, f32, float8_e4m3fn or int8; 8-bit ones with scale bytes
    [n_pages][n_kv_heads][page_size], uint8).  It keeps the tensors; make it once."""
    return KvCache(k, v, k_scale, v_scale)


# ----------------------------------------------------------------------------- positions
def riftkv_rope_freqs(rotary_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                      original_len: float = 0.0, low: float = 0.0, high: float = 0.0):
    """Host-only call: (float64 numpy array of rotary_dim / 2 angles a position,
    magnitude) for riftkv_rope."""
    import numpy as np
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling: one of {ROPE_SCALINGS}")
    rotary_dim = _int32(int(rotary_dim), "rotary_dim")
    cfg = _RopeStruct(rotary_dim, ROPE_SCALINGS.index(scaling), float(base), float(factor), float(original_len),
                      float(low), float(high))
    out = np.zeros(max(1, rotary_dim // 2), dtype=np.float64)
    mag = ctypes.c_double(0.0)
    _check(_load().riftkv_rope_freqs(ctypes.byref(cfg), out.ctypes.data, ctypes.byref(mag)), "riftkv_rope_freqs")
    return out, float(mag.value)


def _rope_rows(t, dtype, rows, heads, hd, dev, name):
    """_rows, for rows whose strides are as they mostly are."""
    if t.dtype is dtype and t.shape == (rows, heads, hd) and t.get_device() == dev:
        ld, sh, se = t.stride()
        if se == 1 and sh == hd and rows > 1:
            return t.data_ptr(), ld
    return _rows(t, dtype, (rows, heads, hd), dev, name)


def _rope(name, fn, q, k, positions, freqs, q_out, k_out, layout, magnitude, stream, axes=None):
    x = q if q is not None else k
    if x is None:
        raise ValueError("q or k is needed")
    if x.dim() != 3:
        raise ValueError("rows: expected [rows][heads][head_dim]")
    dev, dtype, (rows, heads, hd) = x.get_device(), x.dtype, x.shape
    if (rows | heads | hd) >> 31:
        _too_many()
    dt = _ROWS.get(dtype)
    if dt is None or dev < 0:
        _device_of(x, "rows")
        _row_type(x, "rows")
    pq = lq = nq = poq = loq = pk = lk = nk = pok = lok = 0
    if q is not None:
        nq = heads
        pq, lq = _rope_rows(q, dtype, rows, nq, hd, dev, "q")
        poq, loq = (pq, lq) if q_out is None else _rope_rows(q_out, dtype, rows, nq, hd, dev, "q_out")
    elif q_out is not None:
        raise ValueError("q_out without q")
    if k is not None:
        if k.dim() != 3:
            raise ValueError("rows: expected [rows][heads][head_dim]")
        nk = k.shape[1]
        if nk >> 31:
            _too_many()
        pk, lk = _rope_rows(k, dtype, rows, nk, hd, dev, "k")
        pok, lok = (pk, lk) if k_out is None else _rope_rows(k_out, dtype, rows, nk, hd, dev, "k_out")
    elif k_out is not None:
        raise ValueError("k_out without k")
    lay = ROPE_LAYOUTS.get(layout)
    if lay is None:
        raise ValueError(f"layout: one of {tuple(ROPE_LAYOUTS)}")
    fp = _host(freqs, _F8, ctypes.c_double, "freqs: expected a contiguous float64 array")
    if axes is None:
        shape, places, by_axis = (rows,), (rows,), ()
    else:
        if axes.shape != freqs.shape:
            raise ValueError("axes: expected as many as freqs")
        shape = (positions.shape[0], rows)
        if shape[0] >> 31:
            _too_many()
        places = shape
        by_axis = (_host(axes, _I4, ctypes.c_int32, "axes: expected a contiguous int32 array"),)
    if positions.dtype is not _I32 or positions.shape != shape or not positions.is_contiguous() or positions.get_device() != dev:
        _dense(positions, _I32, shape, dev, "positions")
    st = _raw_stream(dev) or None if stream is None else _stream(stream, dev)
    args = (pq, lq, nq, poq, loq, pk, lk, nk, pok, lok, dt, positions.data_ptr(), *places, hd, 2 * freqs.size, lay, fp, *by_axis,
            magnitude, st)
    st = fn(*args) if dev == _device() else _elsewhere(dev, fn, *args)
    if st:
        _check(st, name)


def _host(a, dtype, ctype, what):
    """Address of a numpy array (its own .ctypes takes three times as long)."""
    if a.dtype is dtype:
        try:
            return ctypes.byref(ctype.from_buffer(a))
        except (TypeError, ValueError, BufferError):   # not writeable, or not what it has to be
            pass
    if a.dtype.str != dtype.str or not a.flags.c_contiguous or a.size == 0:
        raise TypeError(what)
    return a.ctypes.data


def riftkv_rope(q, k, positions, freqs, q_out=None, k_out=None, layout: str = "half", magnitude: float = 1.0,
                stream=None) -> None:
    """Rotates the rows q and k (either may be None) into q_out and k_out (None: in
    place) by positions [rows] i32.  freqs: float64 numpy array of rotary_dim / 2
    angles a position (riftkv_rope_freqs)."""
    _rope("riftkv_rope", (_lib or _load()).riftkv_rope, q, k, positions, freqs, q_out, k_out, layout, magnitude, stream)


def riftkv_rope_axes(q, k, positions, freqs, axes, q_out=None, k_out=None, layout: str = "half", magnitude: float = 1.0,
                     stream=None) -> None:
    """The same by positions [n_axes][rows] i32 on several axes: pair j turns by
    positions[axes[j]].  axes: int32 numpy array of rotary_dim / 2."""
    _rope("riftkv_rope_axes", (_lib or _load()).riftkv_rope_axes, q, k, positions, freqs, q_out, k_out, layout, magnitude, stream, axes)


# ----------------------------------------------------------------------------- rows
def _move(name, fn, cache, k, v, page_table, positions, status, seq_ids, stream):
    dev, hd, dtype, i32, rows = cache.device, cache.head_dim, k.dtype, _I32, k.shape[0]
    shape, one = (rows, cache.n_kv_heads, hd), (rows,)
    n_seq, max_pages = page_table.shape
    if (rows | n_seq | max_pages) >> 31:
        _too_many()
    dt = _ROWS.get(dtype)
    if dt is None:
        _row_type(k, "k")
    if k.shape != shape or k.get_device() != dev:
        _rows(k, dtype, shape, dev, "k")
    if v.dtype is not dtype or v.shape != shape or v.get_device() != dev:
        _rows(v, dtype, shape, dev, "v")
    pk, pv = k.data_ptr(), v.data_ptr()
    ldk, sh, se = k.stride()
    if se != 1 or sh != hd:
        pk, ldk = _rows(k, dtype, shape, dev, "k")
    elif rows < 2:
        ldk = shape[1] * hd
    ldv, sh, se = v.stride()
    if se != 1 or sh != hd:
        pv, ldv = _rows(v, dtype, shape, dev, "v")
    elif rows < 2:
        ldv = shape[1] * hd
    if page_table.dtype is not i32 or not page_table.is_contiguous() or page_table.get_device() != dev:
        _dense(page_table, i32, None, dev, "page_table")
    if positions.dtype is not i32 or positions.shape != one or not positions.is_contiguous() or positions.get_device() != dev:
        _dense(positions, i32, one, dev, "positions")
    ids = None
    if seq_ids is not None:
        if seq_ids.dtype is not i32 or seq_ids.shape != one or not seq_ids.is_contiguous() or seq_ids.get_device() != dev:
            _dense(seq_ids, i32, one, dev, "seq_ids")
        ids = seq_ids.data_ptr()
    if status.dtype is not i32 or status.shape != (1,) or status.get_device() != dev:
        _dense(status, i32, (1,), dev, "status")
    st = _raw_stream(dev) or None if stream is None else _stream(stream, dev)
    args = (cache.ref, pk, ldk, pv, ldv, dt, page_table.data_ptr(), n_seq, max_pages, ids, positions.data_ptr(), rows,
            status.data_ptr(), st)
    st = fn(*args) if dev == _device() else _elsewhere(dev, fn, *args)
    if st:
        _check(st, name)


def riftkv_write(cache: KvCache, k, v, page_table, positions, status, seq_ids=None, stream=None) -> None:
    """Rows k, v [rows][n_kv_heads][head_dim] into the pages of their sequences:
    row i is at positions[i] of sequence seq_ids[i] (None: i); page_table
    [n_seq][max_pages], all i32.  Negative ones are skipped."""
    _move("riftkv_write", _lib.riftkv_write, cache, k, v, page_table, positions, status, seq_ids, stream)


def riftkv_read(cache: KvCache, page_table, positions, k_out, v_out, status, seq_ids=None, stream=None) -> None:
    """The same rows out of the pages, into k_out and v_out."""
    _move("riftkv_read", _lib.riftkv_read, cache, k_out, v_out, page_table, positions, status, seq_ids, stream)


# ----------------------------------------------------------------------------- attention
def riftkv_attention_workspace_size(cache: KvCache, n_seq: int, n_heads: int, max_pages: int) -> int:
    return int(_load().riftkv_attention_workspace_size(cache.ref, _int32(int(n_heads), "n_heads"), _int32(int(n_seq), "n_seq"),
                                                       _int32(int(max_pages), "max_pages")))


def riftkv_attention(cache: KvCache, q, page_table, lens, out, workspace, status, scale: Optional[float] = None,
                     stream=None) -> None:
    """out[i] := attention of q[i] [n_heads][head_dim] over the first lens[i] tokens of
    sequence i's pages; scale None: 1 / sqrt(head_dim)."""
    dev, hd, dtype, i32 = cache.device, cache.head_dim, q.dtype, _I32
    n_seq, max_pages = page_table.shape
    n_heads = q.shape[1]
    if (n_seq | max_pages | n_heads) >> 31:
        _too_many()
    shape = (n_seq, n_heads, hd)
    dt = _ROWS.get(dtype)
    if dt is None:
        _row_type(q, "q")
    if q.shape != shape or q.get_device() != dev:
        _rows(q, dtype, shape, dev, "q")
    if out.dtype is not dtype or out.shape != shape or out.get_device() != dev:
        _rows(out, dtype, shape, dev, "out")
    pq, po = q.data_ptr(), out.data_ptr()
    ldq, sh, se = q.stride()
    if se != 1 or sh != hd:
        pq, ldq = _rows(q, dtype, shape, dev, "q")
    elif n_seq < 2:
        ldq = n_heads * hd
    ldo, sh, se = out.stride()
    if se != 1 or sh != hd:
        po, ldo = _rows(out, dtype, shape, dev, "out")
    elif n_seq < 2:
        ldo = n_heads * hd
    if page_table.dtype is not i32 or not page_table.is_contiguous() or page_table.get_device() != dev:
        _dense(page_table, i32, None, dev, "page_table")
    if lens.dtype is not i32 or lens.shape != (n_seq,) or not lens.is_contiguous() or lens.get_device() != dev:
        _dense(lens, i32, (n_seq,), dev, "lens")
    if status.dtype is not i32 or status.shape != (1,) or status.get_device() != dev:
        _dense(status, i32, (1,), dev, "status")
    if workspace.dtype is not _U8 or not workspace.is_contiguous() or workspace.get_device() != dev:
        _dense(workspace, _U8, None, dev, "workspace")
    st = _raw_stream(dev) or None if stream is None else _stream(stream, dev)
    args = (cache.ref, pq, ldq, n_heads, dt, page_table.data_ptr(), n_seq, max_pages, lens.data_ptr(),
            hd ** -0.5 if scale is None else scale, po, ldo, status.data_ptr(), workspace.data_ptr(), workspace.numel(), st)
    st = _lib.riftkv_attention(*args) if dev == _device() else _elsewhere(dev, _lib.riftkv_attention, *args)
    if st:
        _check(st, "riftkv_attention")


# ----------------------------------------------------------------------------- ranges of pages
def _queries(cache, q, page_table, lens, status):
    """What the calls below check alike: (device, row type, sequences, the table's width, q's address and stride)."""
    dev, hd, dtype, i32 = cache.device, cache.head_dim, q.dtype, _I32
    n_seq, max_pages = page_table.shape
    dt = _ROWS.get(dtype)
    if dt is None:
        _row_type(q, "q")
    n, n_heads, width = q.shape
    if (n_seq | max_pages | n_heads) >> 31:
        _too_many()
    pq = q.data_ptr()
    ldq, sh, se = q.stride()
    if n != n_seq or width != hd or q.get_device() != dev or se != 1 or sh != hd:
        pq, ldq = _rows(q, dtype, (n_seq, n_heads, hd), dev, "q")
    elif n_seq < 2:
        ldq = n_heads * hd
    if page_table.dtype is not i32 or not page_table.is_contiguous() or page_table.get_device() != dev:
        _dense(page_table, i32, None, dev, "page_table")
    if lens.dtype is not i32 or lens.shape != (n_seq,) or not lens.is_contiguous() or lens.get_device() != dev:
        _dense(lens, i32, (n_seq,), dev, "lens")
    if status.dtype is not i32 or status.shape != (1,) or status.get_device() != dev:
        _dense(status, i32, (1,), dev, "status")
    return dev, dt, n_seq, max_pages, n_heads, pq, ldq


def _output(out, q, dev):
    """Address and stride of rows like q's."""
    shape = q.shape
    ld, sh, se = out.stride()
    if out.dtype is not q.dtype or out.shape != shape or out.get_device() != dev or se != 1 or sh != shape[2]:
        return _rows(out, q.dtype, shape, dev, "out")
    return out.data_ptr(), (ld if shape[0] > 1 else shape[1] * shape[2])


def _space(workspace, dev):
    if workspace.dtype is not _U8 or not workspace.is_contiguous() or workspace.get_device() != dev:
        _dense(workspace, _U8, None, dev, "workspace")
    return workspace.data_ptr()


def _lists(cache, pages, n_seq, dev):
    shape = pages.shape
    if len(shape) != 3:
        raise ValueError("pages: expected [n_seq][n_kv_heads][top]")
    if shape[2] >> 31:
        _too_many()
    if shape[0] != n_seq or shape[1] != cache.n_kv_heads or pages.dtype is not _I32 or not pages.is_contiguous() or pages.get_device() != dev:
        _dense(pages, _I32, (n_seq, cache.n_kv_heads, shape[2]), dev, "pages")
    return pages.data_ptr(), shape[2]


def _bounds(cache, bounds):
    """Address of the pages' bounds."""
    return _dense(bounds, torch.float32 if cache.dt == RIFTKV_F32 else torch.bfloat16,
                  (cache.n_pages, cache.n_kv_heads, 2, cache.head_dim), cache.device, "bounds")


def riftkv_attention_shared_workspace_size(cache: KvCache, n_seq: int, n_heads: int, prefix_len: int, max_pages: int) -> int:
    return int(_lib.riftkv_attention_shared_workspace_size(cache.ref, _int32(int(n_heads), "n_heads"), _int32(int(n_seq), "n_seq"),
                                                           _int32(int(prefix_len), "prefix_len"), _int32(int(max_pages), "max_pages")))


def riftkv_attention_shared(cache: KvCache, q, prefix_table, prefix_len: int, page_table, lens, out, workspace, status,
                            scale: Optional[float] = None, stream=None) -> None:
    """out[i] := attention of q[i] [n_heads][head_dim] over the prefix_len tokens of the pages prefix_table [pages] i32
    and then the first lens[i] tokens of sequence i's own pages; scale None: 1 / sqrt(head_dim)."""
    _int32(prefix_len, "prefix_len")
    dev, dt, n_seq, max_pages, n_heads, pq, ldq = _queries(cache, q, page_table, lens, status)
    if prefix_table.dtype is not _I32 or not prefix_table.is_contiguous() or prefix_table.get_device() != dev:
        _dense(prefix_table, _I32, None, dev, "prefix_table")
    if prefix_table.dim() != 1 or prefix_table.shape[0] * cache.page_size < prefix_len:
        raise ValueError("prefix_table: expected the pages of prefix_len tokens")
    po, ldo = _output(out, q, dev)
    ws = _space(workspace, dev)
    st = _raw_stream(dev) or None if stream is None else _stream(stream, dev)
    args = (cache.ref, pq, ldq, n_heads, dt, prefix_table.data_ptr(), prefix_len, page_table.data_ptr(), n_seq, max_pages,
            lens.data_ptr(), cache.head_dim ** -0.5 if scale is None else scale, po, ldo, status.data_ptr(), ws, workspace.numel(), st)
    st = _lib.riftkv_attention_shared(*args) if dev == _device() else _elsewhere(dev, _lib.riftkv_attention_shared, *args)
    if st:
        _check(st, "riftkv_attention_shared")


def riftkv_page_bounds(cache: KvCache, bounds, page_table, lens, status, begins=None, stream=None) -> None:
    """bounds [n_pages][n_kv_heads][2][head_dim] (float32 with float32 pages, else bf16) := the smallest and largest key values
    of the pages that hold tokens begins[i] (None: 0) .. lens[i] - 1 of every sequence."""
    dev, i32 = cache.device, _I32
    n_seq, max_pages = page_table.shape
    if (n_seq | max_pages) >> 31:
        _too_many()
    to = _bounds(cache, bounds)
    table = _dense(page_table, i32, None, dev, "page_table")
    n = _dense(lens, i32, (n_seq,), dev, "lens")
    first = None if begins is None else _dense(begins, i32, (n_seq,), dev, "begins")
    word = _dense(status, i32, (1,), dev, "status")
    st = _raw_stream(dev) or None if stream is None else _stream(stream, dev)
    args = (cache.ref, to, table, n_seq, max_pages, first, n, word, st)
    st = _lib.riftkv_page_bounds(*args) if dev == _device() else _elsewhere(dev, _lib.riftkv_page_bounds, *args)
    if st:
        _check(st, "riftkv_page_bounds")


def riftkv_select_pages_workspace_size(cache: KvCache, n_seq: int, max_pages: int) -> int:
    return int(_lib.riftkv_select_pages_workspace_size(cache.ref, _int32(int(n_seq), "n_seq"), _int32(int(max_pages), "max_pages")))


def riftkv_select_pages(cache: KvCache, bounds, q, page_table, lens, pages, workspace, status, keep_first: int = 1,
                        keep_last: int = 1, stream=None) -> None:
    """pages [n_seq][n_kv_heads][top] i32 := the places in its row of page_table of the `top` pages that each sequence's
    token needs most of each key head, ascending, -1 behind them; the first keep_first and last keep_last always."""
    _int32(keep_first, "keep_first")
    _int32(keep_last, "keep_last")
    dev, dt, n_seq, max_pages, n_heads, pq, ldq = _queries(cache, q, page_table, lens, status)
    of = _bounds(cache, bounds)
    to, top = _lists(cache, pages, n_seq, dev)
    ws = _space(workspace, dev)
    st = _raw_stream(dev) or None if stream is None else _stream(stream, dev)
    args = (cache.ref, of, pq, ldq, n_heads, dt, page_table.data_ptr(), n_seq, max_pages, lens.data_ptr(), keep_first, keep_last, to,
            top, status.data_ptr(), ws, workspace.numel(), st)
    st = _lib.riftkv_select_pages(*args) if dev == _device() else _elsewhere(dev, _lib.riftkv_select_pages, *args)
    if st:
        _check(st, "riftkv_select_pages")


def riftkv_attention_pages_workspace_size(cache: KvCache, n_seq: int, n_heads: int, top: int) -> int:
    return int(_lib.riftkv_attention_pages_workspace_size(cache.ref, _int32(int(n_heads), "n_heads"), _int32(int(n_seq), "n_seq"), _int32(int(top), "top")))


def riftkv_attention_pages(cache: KvCache, q, page_table, lens, pages, out, workspace, status, scale: Optional[float] = None,
                           stream=None) -> None:
    """out[i] := attention of q[i] [n_heads][head_dim] over the tokens before lens[i] of the pages listed for it:
    pages [n_seq][n_kv_heads][top] i32, places in sequence i's row of page_table; scale None: 1 / sqrt(head_dim)."""
    dev, dt, n_seq, max_pages, n_heads, pq, ldq = _queries(cache, q, page_table, lens, status)
    of, top = _lists(cache, pages, n_seq, dev)
    po, ldo = _output(out, q, dev)
    ws = _space(workspace, dev)
    st = _raw_stream(dev) or None if stream is None else _stream(stream, dev)
    args = (cache.ref, pq, ldq, n_heads, dt, page_table.data_ptr(), n_seq, max_pages, lens.data_ptr(), of, top,
            cache.head_dim ** -0.5 if scale is None else scale, po, ldo, status.data_ptr(), ws, workspace.numel(), st)
    st = _lib.riftkv_attention_pages(*args) if dev == _device() else _elsewhere(dev, _lib.riftkv_attention_pages, *args)
    if st:
        _check(st, "riftkv_attention_pages")


# ----------------------------------------------------------------------------- decode
def riftkv_decode_workspace_size(cfg: ModelCfg, cache: KvCache, n_seq: int, max_pages: int) -> int:
    return int(_load().riftkv_decode_workspace_size(ctypes.byref(cfg), cache.ref, _int32(int(n_seq), "n_seq"), _int32(int(max_pages), "max_pages")))


def riftkv_decode_step(cfg: ModelCfg, layers: Sequence[dict], x_new, cache: KvCache, page_table, positions, hidden_out,
                       workspace, status, stream=None) -> None:
    """One generated token of every sequence through the decoder layers, its keys and
    values in pages (include/rift_kv.h).  x_new [n_seq][d] bf16; cache of cfg.n_layers
    layers; positions [n_seq] i32: the tokens each sequence holds already."""
    dev = cache.device
    if len(layers) != cfg.n_layers or cache.n_layers != cfg.n_layers:
        raise ValueError("need one weight set and one layer of pages per layer")
    for w in layers:
        for n, t in w.items():
            _dense(t, torch.bfloat16, None, dev, n)
    n_seq, max_pages = page_table.shape
    if (n_seq | max_pages) >> 31:
        _too_many()
    x = _dense(x_new, torch.bfloat16, (n_seq, cfg.d), dev, "x_new")
    out = _dense(hidden_out, torch.float32, (n_seq, cfg.d), dev, "hidden_out")
    table = _dense(page_table, torch.int32, None, dev, "page_table")
    pos = _dense(positions, torch.int32, (n_seq,), dev, "positions")
    word = _dense(status, torch.int32, (1,), dev, "status")
    ws = _dense(workspace, torch.uint8, None, dev, "workspace")
    arr = (LayerWeights * max(1, len(layers)))(*[layer_struct(w) for w in layers])
    st = _raw_stream(dev) or None if stream is None else _stream(stream, dev)
    args = (ctypes.byref(cfg), arr, x, cache.ref, table, n_seq, max_pages, pos, out, word, ws, workspace.numel(), st)
    st = _lib.riftkv_decode_step(*args) if dev == _device() else _elsewhere(dev, _lib.riftkv_decode_step, *args)
    if st:
        _check(st, "riftkv_decode_step")
