"""The entry points of a step over a stream of tokens (include/fqvit.h): the
root-mean-square norm with the residual's addition, the paged cache of keys and
values, attention of new tokens over it, eviction from it.  Argument marshalling
only, as in binding.py.

A cache is three tensors, k_pages int8 [pages, Hkv, page, d], v_pages int8
[pages, Hkv, d, page] and, where it is evicted by attention weight, weight int64
[pages, Hkv, page]; table int32 [B, max_pages] names each sequence's pages and
length int32 [B] counts its keys.
"""
from __future__ import annotations

from typing import Optional

from . import binding as _b


def _fits(t, dtype, shape, dev) -> bool:
    return (t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == dev)


def _check(dev: int, specs) -> None:
    """Raises for the first of (name, tensor, dtype, shape) that does not fit."""
    try:
        if dev >= 0 and all(_fits(t, dtype, shape, dev) for _, t, dtype, shape in specs):
            return
    except AttributeError:
        pass
    _b._refuse(dev, *specs)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _norm(name, r, gamma, eps, given, more, bits, x, zp_x, alpha, K, m_x, h, y, stream, prepare):
    import torch
    i8, i16, f32 = torch.int8, torch.int16, torch.float32
    T, C = _b._dims(r, 2, "r")
    dev = r.get_device()
    new = r.new_empty if stream is None else lambda s, dtype: _b._empty(r, stream, s, dtype)
    if h is None:
        h = new((T, C), dtype=i16)
    if y is None:
        y = new((T, C), dtype=i8)
    rows = more is not None
    if rows and more[0] is None:
        more = (new((T,), dtype=f32),)
    specs = [("r", r, i16, (T, C)), ("gamma", gamma, f32, (C,)), ("h", h, i16, (T, C)),
             ("y", y, i8, (T, C))]
    if x is not None:
        specs.append(("x", x, i8, (T, C)))
    if alpha is not None:
        if x is None:
            raise ValueError("alpha belongs to a branch: give x with it")
        specs.append(("alpha", alpha, torch.uint8, (C,)))
    if rows:
        specs.append(("scales", more[0], f32, (T,)))
    _check(dev, specs)
    args = (_ptr(x), zp_x, _ptr(alpha), K, m_x, r.data_ptr(), T, C, gamma.data_ptr(), eps, *given, bits,
            h.data_ptr(), y.data_ptr(), *(t.data_ptr() for t in more or ()), _b._raw_stream(stream, dev))
    return _b._invoke(name, args, (x, alpha, r, gamma, h, y, more), prepare, (h, y, *(more or ())), dev)


def rmsnorm_int8(r, gamma, eps: float, s_out: float, zp_out: int = 0, bits: int = 8, x=None,
                 zp_x: int = 0, alpha=None, K: int = 3, m_x: float = 1.0, h=None, y=None, stream=None,
                 prepare: bool = False):
    """Root-mean-square norm of the int16 stream r [T, C] with the int8 branch x
    added (zero point zp_x, power-of-two factors alpha uint8 [C], m_x = s_x / s_r):
    (h int16 [T, C], the new stream, which may be r; y int8 [T, C] of scale s_out
    and zero point zp_out).  eps in steps of the stream, squared."""
    return _norm("rmsnorm_int8", r, gamma, eps, (s_out, zp_out), None, bits, x, zp_x, alpha, K, m_x, h,
                 y, stream, prepare)


def rmsnorm_rows_int8(r, gamma, eps: float, bits: int = 8, x=None, zp_x: int = 0, alpha=None,
                      K: int = 3, m_x: float = 1.0, h=None, y=None, scales=None, stream=None,
                      prepare: bool = False):
    """rmsnorm_int8 with a scale for each row, its largest value at the grid's end:
    (h, y, scales float [T])."""
    return _norm("rmsnorm_rows_int8", r, gamma, eps, (), (scales,), bits, x, zp_x, alpha, K, m_x, h, y,
                 stream, prepare)


def _cache_specs(k_pages, v_pages, weight, table, length, B):
    """(pages, Hkv, page, d, max_pages) of a cache and what its tensors have to be."""
    import torch
    pages, Hkv, page, d = _b._dims(k_pages, 4, "k_pages")
    max_pages = _b._dims(table, 2, "table")[1]
    specs = [("k_pages", k_pages, torch.int8, (pages, Hkv, page, d)),
             ("v_pages", v_pages, torch.int8, (pages, Hkv, d, page)),
             ("table", table, torch.int32, (B, max_pages)), ("length", length, torch.int32, (B,))]
    if weight is not None:
        specs.append(("weight", weight, torch.int64, (pages, Hkv, page)))
    return (pages, Hkv, page, d, max_pages), specs


def kv_cache_append_int8(k, v, k_pages, v_pages, table, length, n_new=None, weight=None, stream=None,
                         prepare: bool = False):
    """Writes k, v int8 [B, Hkv, L, d] (rope_qkv_int8's) into the cache: token
    i < n_new[b] (all L where n_new is None) to place length[b] - n_new[b] + i, so
    length counts the new tokens already; their weight becomes 0."""
    import torch
    B, Hkv, L, d = _b._dims(k, 4, "k")
    dev = k.get_device()
    (pages, Hc, page, dc, max_pages), specs = _cache_specs(k_pages, v_pages, weight, table, length, B)
    if (Hc, dc) != (Hkv, d):
        raise ValueError(f"k_pages must hold {Hkv} heads of {d}, got {Hc} of {dc}")
    specs += [("k", k, torch.int8, (B, Hkv, L, d)), ("v", v, torch.int8, (B, Hkv, L, d))]
    if n_new is not None:
        specs.append(("n_new", n_new, torch.int32, (B,)))
    _check(dev, specs)
    args = (k.data_ptr(), v.data_ptr(), B, Hkv, L, d, _ptr(n_new), k_pages.data_ptr(),
            v_pages.data_ptr(), _ptr(weight), pages, page, table.data_ptr(), max_pages,
            length.data_ptr(), _b._raw_stream(stream, dev))
    return _b._invoke("kv_cache_append_int8", args, (k, v, n_new, k_pages, v_pages, weight, table,
                                                     length), prepare, None, dev)


def lis_attention_paged_workspace_bytes(B: int, Hq: int, Hkv: int, L: int, d: int,
                                        max_keys: int) -> int:
    """Bytes of device scratch that lis_attention_paged needs (max_keys: keys that a
    table's row can name); 0 where it needs none, and for invalid sizes."""
    return int(_b.lib().fq_lis_attention_paged_workspace_bytes(B, Hq, Hkv, L, d, max_keys))


def lis_attention_paged(q, k_pages, v_pages, table, length, s_logit: float, n_new=None, zp_q: int = 0,
                        zp_k: int = 0, zp_v: int = 0, bits: int = 4, exp_n: int = 20,
                        causal: bool = True, weight=None, out=None, workspace=None, stream=None,
                        prepare: bool = False):
    """Integer-only attention of the queries q int8 [B, Hq, L, d] of new tokens over
    the cache: int32 [B, Hq, L, d].  Token i < n_new[b] (all L where n_new is None)
    stands at place length[b] - n_new[b] + i and sees the places up to it (causal) or
    all; rows behind n_new[b] are left as they are (unspecified where out is not
    given).  weight: the cache's, which adds up what each key receives.  The
    workspace is allocated here with torch when not given."""
    import torch
    i8, i32 = torch.int8, torch.int32
    B, Hq, L, d = _b._dims(q, 4, "q")
    dev = q.get_device()
    (pages, Hkv, page, dc, max_pages), specs = _cache_specs(k_pages, v_pages, weight, table, length, B)
    if dc != d:
        raise ValueError(f"k_pages must hold heads of {d}, got {dc}")
    if out is None:
        out = _b._empty(q, stream, (B, Hq, L, d), i32)
    specs += [("q", q, i8, (B, Hq, L, d)), ("out", out, i32, (B, Hq, L, d))]
    if n_new is not None:
        specs.append(("n_new", n_new, i32, (B,)))
    if workspace is None:
        need = lis_attention_paged_workspace_bytes(B, Hq, Hkv, L, d, max_pages * page)
        if need:
            workspace = _b._empty(q, stream, need, torch.uint8)
    size = 0 if workspace is None else workspace.numel()
    if workspace is not None:
        specs.append(("workspace", workspace, torch.uint8, (size,)))
    _check(dev, specs)
    args = (q.data_ptr(), B, Hq, Hkv, L, d, _ptr(n_new), k_pages.data_ptr(), v_pages.data_ptr(),
            _ptr(weight), pages, page, table.data_ptr(), max_pages, length.data_ptr(), zp_q, zp_k, zp_v,
            1 if causal else 0, s_logit, bits, exp_n, out.data_ptr(), _ptr(workspace), size,
            _b._raw_stream(stream, dev))
    return _b._invoke("lis_attention_paged", args, (q, n_new, k_pages, v_pages, weight, table, length,
                                                    out, workspace), prepare, out, dev)


def kv_cache_evict(k_pages, v_pages, weight, table, length, keep: int, recent: int = 0, table_out=None,
                   length_out=None, kept=None, stream=None, prepare: bool = False):
    """Cuts each sequence to at most `keep` keys, by each key head on its own: the
    `recent` last ones and the heaviest of the others (of equal ones the first), in
    their order, brought together in the pages of table_out (None: in place).
    Returns (length_out int32 [B], kept int32 [B, Hkv, keep]: the places that stayed,
    -1 behind the last).  length_out may be length."""
    import torch
    i32 = torch.int32
    B, _ = _b._dims(table, 2, "table")
    dev = k_pages.get_device()
    (pages, Hkv, page, d, max_pages), specs = _cache_specs(k_pages, v_pages, weight, table, length, B)
    if weight is None:
        raise TypeError("weight must be a torch.Tensor")
    table_out: Optional[object] = table if table_out is None else table_out
    max_out = _b._dims(table_out, 2, "table_out")[1]
    if length_out is None:
        length_out = _b._empty(length, stream, (B,), i32)
    if kept is None:
        kept = _b._empty(length, stream, (B, Hkv, keep), i32)
    specs += [("table_out", table_out, i32, (B, max_out)), ("length_out", length_out, i32, (B,)),
              ("kept", kept, i32, (B, Hkv, keep))]
    _check(dev, specs)
    args = (k_pages.data_ptr(), v_pages.data_ptr(), weight.data_ptr(), pages, Hkv, page, d,
            table.data_ptr(), max_pages, length.data_ptr(), B, keep, recent, table_out.data_ptr(),
            max_out, length_out.data_ptr(), kept.data_ptr(), _b._raw_stream(stream, dev))
    return _b._invoke("kv_cache_evict", args, (k_pages, v_pages, weight, table, length, table_out,
                                               length_out, kept), prepare, (length_out, kept), dev)
