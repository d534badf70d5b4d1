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

from . import binding as _b


def _ptr(t):
    return None if t is None else t.data_ptr()


def _norm(name, r, gamma, eps, given, scales, bits, x, zp_x, alpha, K, m_x, h, y, stream, prepare):
    import torch
    i8, i16, f32, u8 = torch.int8, torch.int16, torch.float32, torch.uint8
    T, C = size = _b._dims(r, 2, "r")
    dev = r.get_device()
    new = r.new_empty if stream is None else lambda shape, dtype: _b._empty(r, stream, shape, dtype)
    if h is None:
        h = new(size, dtype=i16)
    if y is None:
        y = new(size, dtype=i8)
    rows = not given
    if rows and scales is None:
        scales = new((T,), dtype=f32)
    if alpha is not None and x is None:
        raise ValueError("alpha belongs to a branch: give x with it")
    try:
        fits = (r.dtype is i16 and r.is_contiguous() and dev >= 0
                and gamma.dtype is f32 and gamma.shape == (C,) and gamma.is_contiguous()
                and gamma.get_device() == dev
                and h.dtype is i16 and h.shape == size and h.is_contiguous() and h.get_device() == dev
                and y.dtype is i8 and y.shape == size and y.is_contiguous() and y.get_device() == dev
                and (x is None or x.dtype is i8 and x.shape == size and x.is_contiguous()
                     and x.get_device() == dev)
                and (alpha is None or alpha.dtype is u8 and alpha.shape == (C,)
                     and alpha.is_contiguous() and alpha.get_device() == dev)
                and (not rows or scales.dtype is f32 and scales.shape == (T,)
                     and scales.is_contiguous() and scales.get_device() == dev))
    except AttributeError:
        fits = False
    if not fits:
        _b._refuse(dev, ("r", r, i16, size), ("gamma", gamma, f32, (C,)), ("h", h, i16, size),
                   ("y", y, i8, size),
                   *[s for s in (("x", x, i8, size), ("alpha", alpha, u8, (C,))) if s[1] is not None],
                   *([("scales", scales, f32, (T,))] if rows else []))
    args = (None if x is None else x.data_ptr(), zp_x, None if alpha is None else alpha.data_ptr(), K,
            m_x, r.data_ptr(), T, C, gamma.data_ptr(), eps, *given, bits, h.data_ptr(), y.data_ptr(),
            *((scales.data_ptr(),) if rows else ()), _b._raw_stream(stream, dev))
    return _b._invoke(name, args, (x, alpha, r, gamma, h, y, scales), prepare,
                      (h, y, scales) if rows else (h, y), dev)


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
    return _norm("rmsnorm_rows_int8", r, gamma, eps, (), scales, bits, x, zp_x, alpha, K, m_x, h, y,
                 stream, prepare)


def _cache_fits(k_pages, v_pages, weight, table, length, B, dev) -> bool:
    """Whether the tensors are a cache of B sequences on device `dev`."""
    import torch
    i8, i32 = torch.int8, torch.int32
    try:
        pages, Hkv, page, d = k_pages.shape
        return (k_pages.dtype is i8 and k_pages.is_contiguous() and k_pages.get_device() == dev >= 0
                and v_pages.dtype is i8 and v_pages.shape == (pages, Hkv, d, page)
                and v_pages.is_contiguous() and v_pages.get_device() == dev
                and table.dtype is i32 and table.shape[0] == B and table.is_contiguous()
                and table.get_device() == dev
                and length.dtype is i32 and length.shape == (B,) and length.is_contiguous()
                and length.get_device() == dev
                and (weight is None or weight.dtype is torch.int64
                     and weight.shape == (pages, Hkv, page) and weight.is_contiguous()
                     and weight.get_device() == dev))
    except AttributeError:
        return False


def _cache_specs(k_pages, v_pages, weight, table, length, B):
    """What a cache's tensors have to be, for _refuse."""
    import torch
    pages, Hkv, page, d = k_pages.shape
    specs = [("k_pages", k_pages, torch.int8, (pages, Hkv, page, d)),
             ("v_pages", v_pages, torch.int8, (pages, Hkv, d, page)),
             ("table", table, torch.int32, (B, table.shape[1])), ("length", length, torch.int32, (B,))]
    if weight is not None:
        specs.append(("weight", weight, torch.int64, (pages, Hkv, page)))
    return specs


def kv_cache_append_int8(k, v, k_pages, v_pages, table, length, n_new=None, weight=None, stream=None,
                         prepare: bool = False):
    """Writes k, v int8 [B, Hkv, L, d] (rope_qkv_int8's) into the cache: token
    i < n_new[b] (all L where n_new is None) to place length[b] - n_new[b] + i, so
    length counts the new tokens already; their weight becomes 0."""
    import torch
    i8, i32 = torch.int8, torch.int32
    B, Hkv, L, d = size = _b._dims(k, 4, "k")
    pages, Hc, page, dc = _b._dims(k_pages, 4, "k_pages")
    max_pages = _b._dims(table, 2, "table")[1]
    dev = k.get_device()
    if Hc != Hkv or dc != d:
        raise ValueError(f"k_pages must hold {Hkv} heads of {d}, got {Hc} of {dc}")
    try:
        fits = (k.dtype is i8 and k.is_contiguous()
                and v.dtype is i8 and v.shape == size and v.is_contiguous() and v.get_device() == dev
                and (n_new is None or n_new.dtype is i32 and n_new.shape == (B,)
                     and n_new.is_contiguous() and n_new.get_device() == dev)
                and _cache_fits(k_pages, v_pages, weight, table, length, B, dev))
    except AttributeError:
        fits = False
    if not fits:
        _b._refuse(dev, *_cache_specs(k_pages, v_pages, weight, table, length, B),
                   ("k", k, i8, size), ("v", v, i8, size),
                   *([] if n_new is None else [("n_new", n_new, i32, (B,))]))
    args = (k.data_ptr(), v.data_ptr(), B, Hkv, L, d, _ptr(n_new), k_pages.data_ptr(),
            v_pages.data_ptr(), _ptr(weight), pages, page, table.data_ptr(), max_pages,
            length.data_ptr(), _b._raw_stream(stream, dev))
    return _b._invoke("kv_cache_append_int8", args, (k, v, n_new, k_pages, v_pages, weight, table,
                                                     length), prepare, None, dev)


def lis_attention_paged_workspace_bytes(B: int, Hq: int, Hkv: int, L: int, d: int,
                                        max_keys: int) -> int:
    """Bytes of device scratch that lis_attention_paged needs (max_keys: keys that a
    table's row can name, which it grows with, to 1 GiB); 0 where it needs none, and
    for invalid sizes."""
    return _workspace_bytes(B, Hq, Hkv, L, d, max_keys)


def _workspace_bytes(*sizes) -> int:
    if max(sizes) > 0x7fffffff or min(sizes) < 0:       # the call itself refuses these
        return 0
    return (_b._lib or _b.lib()).fq_lis_attention_paged_workspace_bytes(*sizes)


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
    i8, i32, u8 = torch.int8, torch.int32, torch.uint8
    B, Hq, L, d = size = _b._dims(q, 4, "q")
    pages, Hkv, page, dc = _b._dims(k_pages, 4, "k_pages")
    max_pages = _b._dims(table, 2, "table")[1]
    dev = q.get_device()
    if dc != d:
        raise ValueError(f"k_pages must hold heads of {d}, got {dc}")
    if out is None:
        out = q.new_empty(size, dtype=i32) if stream is None else _b._empty(q, stream, size, i32)
    if workspace is None:
        need = _workspace_bytes(B, Hq, Hkv, L, d, max_pages * page)
        if need:
            workspace = _b._empty(q, stream, need, u8)
    held = 0 if workspace is None else workspace.numel()
    try:
        fits = (q.dtype is i8 and q.is_contiguous()
                and out.dtype is i32 and out.shape == size and out.is_contiguous()
                and out.get_device() == dev
                and (n_new is None or n_new.dtype is i32 and n_new.shape == (B,)
                     and n_new.is_contiguous() and n_new.get_device() == dev)
                and (workspace is None or workspace.dtype is u8 and workspace.shape == (held,)
                     and workspace.is_contiguous() and workspace.get_device() == dev)
                and _cache_fits(k_pages, v_pages, weight, table, length, B, dev))
    except AttributeError:
        fits = False
    if not fits:
        _b._refuse(dev, *_cache_specs(k_pages, v_pages, weight, table, length, B),
                   ("q", q, i8, size), ("out", out, i32, size),
                   *([] if n_new is None else [("n_new", n_new, i32, (B,))]),
                   *([] if workspace is None else [("workspace", workspace, u8, (held,))]))
    args = (q.data_ptr(), B, Hq, Hkv, L, d, _ptr(n_new), k_pages.data_ptr(), v_pages.data_ptr(),
            _ptr(weight), pages, page, table.data_ptr(), max_pages, length.data_ptr(), zp_q, zp_k, zp_v,
            1 if causal else 0, s_logit, bits, exp_n, out.data_ptr(), _ptr(workspace), held,
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
    B, max_pages = _b._dims(table, 2, "table")
    pages, Hkv, page, d = _b._dims(k_pages, 4, "k_pages")
    dev = k_pages.get_device()
    if weight is None:
        raise TypeError("weight must be a torch.Tensor")
    if table_out is None:
        table_out = table
    max_out = _b._dims(table_out, 2, "table_out")[1]
    new = k_pages.new_empty if stream is None else lambda s, dtype: _b._empty(k_pages, stream, s, dtype)
    if length_out is None:
        length_out = new((B,), dtype=i32)
    if kept is None:
        kept = new((B, Hkv, keep), dtype=i32)
    try:
        fits = (table_out.dtype is i32 and table_out.shape[0] == B and table_out.is_contiguous()
                and table_out.get_device() == dev
                and length_out.dtype is i32 and length_out.shape == (B,)
                and length_out.is_contiguous() and length_out.get_device() == dev
                and kept.dtype is i32 and kept.shape == (B, Hkv, keep) and kept.is_contiguous()
                and kept.get_device() == dev
                and _cache_fits(k_pages, v_pages, weight, table, length, B, dev))
    except AttributeError:
        fits = False
    if not fits:
        _b._refuse(dev, *_cache_specs(k_pages, v_pages, weight, table, length, B),
                   ("table_out", table_out, i32, (B, max_out)), ("length_out", length_out, i32, (B,)),
                   ("kept", kept, i32, (B, Hkv, keep)))
    args = (k_pages.data_ptr(), v_pages.data_ptr(), weight.data_ptr(), pages, Hkv, page, d,
            table.data_ptr(), max_pages, length.data_ptr(), B, keep, recent, table_out.data_ptr(),
            max_out, length_out.data_ptr(), kept.data_ptr(), _b._raw_stream(stream, dev))
    return _b._invoke("kv_cache_evict", args, (k_pages, v_pages, weight, table, length, table_out,
                                               length_out, kept), prepare, (length_out, kept), dev)
