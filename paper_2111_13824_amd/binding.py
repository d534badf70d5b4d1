"""ctypes binding of libfqvit (include/fqvit.h).

Argument marshalling only: each function checks dtypes, devices, shapes and
contiguity of torch tensors, passes their device pointers and the current HIP
stream to the C ABI entry point of the same name, and raises ``FqError`` on a
non-zero status.  Every step of the computation runs in the HIP kernels; there
is no fallback.  If libfqvit.so is not built the first call raises.
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libfqvit.so")

(FQ_OK, FQ_ERR_NULL, FQ_ERR_SHAPE, FQ_ERR_PARAM, FQ_ERR_HEADROOM, FQ_ERR_HIP,
 FQ_ERR_SCRATCH) = range(7)
# Bytes of the library's fixed device scratch (FQ_NOALLOC_SCRATCH_BYTES).
NOALLOC_SCRATCH_BYTES = 8 << 20

# Entry points declared in include/fqvit.h and their C argument types.
_P = ctypes.c_void_p
_I32, _I64, _F32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
SIGNATURES = {
    "ptf_layernorm_int8": [_P, _I64, _I32, _I32, _P, _I32, _P, _P, _F32, _I32, _I32, _P, _P],
    "lis_softmax_log4": [_P, _I64, _I32, _I32, _P, _I32, _F32, _I32, _I32, _P, _I32, _P],
    "lis_attn_v_shift": [_P, _I32, _P, _I32, _I64, _I32, _I32, _I32, _I32, _P, _P],
    "lis_attn_v_shift_wide": [_P, _I32, _P, _I32, _I64, _I32, _I32, _I32, _I32, _P, _P],
    "lis_attention_head": [_P, _P, _I32, _I64, _I32, _I32, _F32, _I32, _I32, _P, _I32, _I32, _P,
                           _P, _I32, _P],
    "lis_attention_qk": [_P, _P, _I32, _I32, _I32, _P, _I32, _I64, _I32, _I32, _F32, _I32, _I32,
                         _P, _I32, _I32, _P, _P],
    "ptf_calibrate": [_P, _I64, _I32, _I32, _I32, _P, _P, _P, _P, ctypes.c_size_t, _P],
    "ptf_calibrate_noalloc": [_P, _I64, _I32, _I32, _I32, _P, _P, _P, _P],
    "ptf_quantize_int8": [_P, _I64, _I32, _P, _P, _P, _I32, _P, _P],
    "requant_dyadic_int8": [_P, _I64, _F32, _F32, _I32, _I32, _P, _P],
    "linear_fold_int8": [_P, _I32, _I32, _P, _P, _I32, _F32, _F32, _P, _P, _P],
    "linear_int8": [_P, _I64, _P, _I32, _I32, _P, _P, _I32, _P, _I32, _I32, _P, _I32, _F32, _I32,
                    _I32, _P, _P],
    "linear_int32": [_P, _I64, _P, _I32, _I32, _P, _P, _P],
    "rope_table_int16": [_P, _I32, _I64, _P, _P, _I32, _P, _P],
    "rope_qkv_int8": [_P, _I64, _I32, _I32, _I32, _I32, _F32, _I32, _P, _I64, _I32, _I32, _F32,
                      _I32, _F32, _I32, _I32, _P, _P, _P, _P],
    "requant_heads_int8": [_P, _I64, _I32, _I32, _I32, _F32, _F32, _I32, _I32, _P, _P],
    "fq_activation_table": [_I32, _F32, _I32, _I32, _F32, _P],
}


def _int32s(types):
    """Takes a call's 32-bit integers out of its arguments, and packs them, which
    refuses what 32 bits do not hold."""
    at = [i for i, t in enumerate(types) if t is _I32]
    return operator.itemgetter(*at), struct.Struct(f"={len(at)}i").pack


_INT32S = {name: _int32s(types) for name, types in SIGNATURES.items()}

# Activations of linear_int8 and functions of fq_activation_table.
ACT_NONE, ACT_RELU, ACT_TABLE = range(3)
_FUNCTIONS = {"gelu": 0, "gelu_tanh": 1, "silu": 2}


class FqError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn}: {status_str(status)}")


_lib: Optional[ctypes.CDLL] = None


def load(path: str) -> ctypes.CDLL:
    """Open a build of libfqvit at `path` and declare its entry points' C types."""
    L = ctypes.CDLL(path)
    for name, args in SIGNATURES.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int32
    L.fq_status_str.argtypes = [ctypes.c_int]
    L.fq_status_str.restype = ctypes.c_char_p
    L.fq_version.argtypes = []
    L.fq_version.restype = ctypes.c_int32
    L.fq_time_next_call.argtypes = [_P, _P]
    L.fq_time_next_call.restype = ctypes.c_int32
    L.fq_ptf_calibrate_workspace_bytes.argtypes = [_I64, _I32, _I32]
    L.fq_ptf_calibrate_workspace_bytes.restype = ctypes.c_size_t
    return L


def lib() -> ctypes.CDLL:
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -c "
                               f"'import __graft_entry__ as g; g.build()'` (no fallback exists)")
        _lib = load(LIB_PATH)
    return _lib


def status_str(status: int) -> str:
    return lib().fq_status_str(int(status)).decode()


def version() -> int:
    return lib().fq_version()


def time_next_call(start_event: int, stop_event: int) -> None:
    """Attach two hipEvent_t handles (ints) to the kernel of the next call on
    this thread: they record that kernel's own start and end."""
    lib().fq_time_next_call(start_event or None, stop_event or None)


def _stream(stream, like) -> int:
    """Raw hipStream_t: the given torch stream, else torch's current stream on
    the device of tensor `like` (read without creating a Stream object)."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(like.device.index)


def _dev_ptr(t, dtype, name: str, ndim: Optional[int] = None):
    if t is None:
        return None
    try:
        ok = (t.dtype is dtype and t.is_cuda and (ndim is None or t.dim() == ndim)
              and t.is_contiguous())
    except AttributeError:
        raise TypeError(f"{name} must be a torch.Tensor") from None
    if not ok:
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        raise ValueError(f"{name} must have {ndim} dimensions, got {t.dim()}")
    return t.data_ptr()


def _check(fn: str, status: int) -> None:
    if status != FQ_OK:
        raise FqError(fn, status)


def _narrow(name: str, args) -> None:
    """Raises where ctypes would silently drop the high bits of an integer (a
    row of 2^32 + 16 values would be taken for one of 16)."""
    ints, pack = _INT32S[name]
    try:
        pack(*ints(args))
    except struct.error:
        for a in ints(args):
            if isinstance(a, int) and not -0x80000000 <= a <= 0x7fffffff:
                raise ValueError(f"{name}: {a} does not fit a 32-bit integer") from None
        # not integers: left to ctypes, which names the argument


class Prepared:
    """A validated call with its arguments already converted to C types:
    calling it only enters the library (for launch loops where Python
    marshalling would otherwise dominate).  The stream is the one current when
    the call was prepared; the tensors are kept alive by the object.  With
    `device`, the call runs with that device current (a default stream is the
    current device's)."""

    __slots__ = ("_name", "_fn", "_args", "_keep", "_device")

    def __init__(self, name: str, args, keep, device: Optional[int] = None):
        _narrow(name, args)
        self._name = name
        self._fn = getattr(lib(), name)
        self._args = tuple(t(a) if a is not None else None
                           for t, a in zip(SIGNATURES[name], args))
        self._keep = keep
        self._device = device

    def __call__(self) -> None:
        st = _enter(self._fn, self._args, self._device)
        if st != FQ_OK:
            raise FqError(self._name, st)


def _enter(fn, args, device: Optional[int]) -> int:
    """fn(*args), with `device` current where one is given."""
    if device is None:
        return fn(*args)
    import torch
    if torch._C._cuda_getDevice() == device:
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def _invoke(name: str, args, keep, prepare: bool, result, device: Optional[int] = None):
    """Run the entry point now, or return it prepared for repeated calls."""
    if prepare:
        return Prepared(name, args, keep, device)
    try:                       # as _narrow, without a call more on the way of each call
        ints, pack = _INT32S[name]
        pack(*ints(args))
    except struct.error:
        _narrow(name, args)
    st = _enter(getattr(_lib or lib(), name), args, device)
    if st != FQ_OK:
        raise FqError(name, st)
    return result


def _refuse(device: int, *specs):
    """Raises for the first of (name, tensor, dtype, shape) that does not fit: a
    contiguous tensor of that dtype and shape (None where the argument may be
    left out: the spec is then not given), all on one device.  The functions
    below ask this only where one expression over all their tensors has failed:
    a call of a helper for each tensor would take a seventh of a short call."""
    for name, t, dtype, shape in specs:
        if not hasattr(t, "is_contiguous"):
            raise TypeError(f"{name} must be a torch.Tensor")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    for name, t, _, _ in specs:
        if t.get_device() < 0:
            raise ValueError(f"{name} must be a device tensor")
        if t.get_device() != device:
            raise ValueError(f"{name} must be on device {device}, got {t.device}")
    raise ValueError("arguments do not fit together")


def _dims(t, n: int, name: str):
    """The shape of tensor `t`, which has to have n dimensions."""
    shape = t.shape
    if len(shape) != n:
        raise ValueError(f"{name} must have {n} dimensions, got {len(shape)}")
    return shape


def _raw_stream(stream, device: int) -> int:
    """Raw hipStream_t: the given torch stream, else the device's current one."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(device)


def _empty(like, stream, shape, dtype):
    """An output or workspace that the caller did not give, on the device of `like`
    and from the memory of the stream that the call runs on: torch's allocator
    then hands it on only behind that stream's work (memory of the current stream
    could still be in use there when another stream writes it, or be handed on
    while that stream still does)."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    import torch
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def ptf_layernorm_int8(x_q, zp_in: int, alpha, K: int, gamma, beta, s_out: float, zp_out: int,
                       bits: int = 8, y_q=None, stream=None, prepare: bool = False):
    """PTF LayerNorm of an int8 [T, C] tensor; returns (or fills) int8 [T, C].
    With prepare=True returns a Prepared call instead of running it."""
    import torch
    T, C = x_q.shape
    if y_q is None:
        y_q = torch.empty_like(x_q) if stream is None else _empty(x_q, stream, x_q.shape, torch.int8)
    if alpha.shape != (C,) or gamma.shape != (C,) or beta.shape != (C,) or y_q.shape != (T, C):
        raise ValueError("alpha, gamma, beta must be [C] and y_q [T, C]")
    args = (_dev_ptr(x_q, torch.int8, "x_q", 2), T, C, zp_in,
            _dev_ptr(alpha, torch.uint8, "alpha", 1), K,
            _dev_ptr(gamma, torch.float32, "gamma", 1),
            _dev_ptr(beta, torch.float32, "beta", 1), s_out, zp_out, bits,
            _dev_ptr(y_q, torch.int8, "y_q", 2), _stream(stream, x_q))
    return _invoke("ptf_layernorm_int8", args, (x_q, alpha, gamma, beta, y_q), prepare, y_q)


def codes_ld(Lk: int, bits: int = 4) -> int:
    """Bytes per row of stored codes: two per byte up to 4 bits, else one."""
    return (Lk + 1) // 2 if bits <= 4 else Lk


def lis_softmax_log4(logits, s_logit: float, bits: int = 4, exp_n: int = 20, bias=None,
                     codes=None, stream=None, prepare: bool = False):
    """Log-Int-Softmax codes [G, Lq, ld] of int32 logits [G, Lq, Lk]: packed two
    per byte for bits <= 4, one per byte for bits in [5, 8]."""
    import torch
    G, Lq, Lk = logits.shape
    if codes is None:
        # rows without padding: the kernel writes every byte (an odd row's last
        # high nibble 0)
        codes = _empty(logits, stream, (G, Lq, codes_ld(Lk, bits)), torch.uint8)
    if codes.dim() != 3 or codes.shape[:2] != (G, Lq):
        raise ValueError("codes must be [G, Lq, ld_codes]")
    Hb = 0
    if bias is not None:
        if bias.dim() != 3 or bias.shape[1:] != (Lq, Lk):
            raise ValueError("bias must be [Hb, Lq, Lk]")
        Hb = bias.shape[0]
    args = (_dev_ptr(logits, torch.int32, "logits", 3), G, Lq, Lk,
            _dev_ptr(bias, torch.int32, "bias", 3), Hb, s_logit, bits, exp_n,
            _dev_ptr(codes, torch.uint8, "codes", 3), codes.shape[2], _stream(stream, logits))
    return _invoke("lis_softmax_log4", args, (logits, bias, codes), prepare, codes)


def lis_attn_v_shift(codes, v, Lk: int, zp_v: int = 0, bits: int = 4, out=None, stream=None,
                     prepare: bool = False):
    """BitShift Attn x V: int32 [G, Lq, d] from packed codes [G, Lq, ld] and int8 V [G, Lk, d]."""
    import torch
    G, Lq, ld = codes.shape
    d = v.shape[2]
    if v.dim() != 3 or v.shape[:2] != (G, Lk):
        raise ValueError("v must be [G, Lk, d]")
    if out is None:
        out = _empty(v, stream, (G, Lq, d), torch.int32)
    if out.shape != (G, Lq, d):
        raise ValueError("out must be [G, Lq, d]")
    args = (_dev_ptr(codes, torch.uint8, "codes", 3), ld, _dev_ptr(v, torch.int8, "v", 3), zp_v,
            G, Lq, Lk, d, bits, _dev_ptr(out, torch.int32, "out", 3), _stream(stream, v))
    return _invoke("lis_attn_v_shift", args, (codes, v, out), prepare, out)


def lis_attn_v_shift_wide(codes, v, Lk: int, zp_v: int = 0, bits: int = 8, out=None, stream=None,
                          prepare: bool = False):
    """BitShift Attn x V for codes of any width b in [1, 8] (nibbles for b <= 4,
    bytes above): int64 [G, Lq, d] at scale s_V / 2^min(2^b - 1, 44)."""
    import torch
    G, Lq, ld = codes.shape
    d = v.shape[2]
    if v.dim() != 3 or v.shape[:2] != (G, Lk):
        raise ValueError("v must be [G, Lk, d]")
    if out is None:
        out = _empty(v, stream, (G, Lq, d), torch.int64)
    if out.shape != (G, Lq, d):
        raise ValueError("out must be [G, Lq, d]")
    args = (_dev_ptr(codes, torch.uint8, "codes", 3), ld, _dev_ptr(v, torch.int8, "v", 3), zp_v,
            G, Lq, Lk, d, bits, _dev_ptr(out, torch.int64, "out", 3), _stream(stream, v))
    return _invoke("lis_attn_v_shift_wide", args, (codes, v, out), prepare, out)


def lis_attention_head(logits, v, s_logit: float, bits: int = 4, exp_n: int = 20, zp_v: int = 0,
                       bias=None, out=None, codes_out=None, stream=None, prepare: bool = False):
    """Fused Log-Int-Softmax + BitShift Attn x V; returns int32 [G, Lq, d]."""
    import torch
    G, Lq, Lk = logits.shape
    d = v.shape[2]
    if v.dim() != 3 or v.shape[:2] != (G, Lk):
        raise ValueError("v must be [G, Lk, d]")
    if out is None:
        out = _empty(logits, stream, (G, Lq, d), torch.int32)
    if out.shape != (G, Lq, d):
        raise ValueError("out must be [G, Lq, d]")
    Hb = 0
    if bias is not None:
        if bias.dim() != 3 or bias.shape[1:] != (Lq, Lk):
            raise ValueError("bias must be [Hb, Lq, Lk]")
        Hb = bias.shape[0]
    ld = 0
    if codes_out is not None:
        if codes_out.dim() != 3 or codes_out.shape[:2] != (G, Lq):
            raise ValueError("codes_out must be [G, Lq, ld_codes]")
        ld = codes_out.shape[2]
    args = (_dev_ptr(logits, torch.int32, "logits", 3), _dev_ptr(bias, torch.int32, "bias", 3), Hb,
            G, Lq, Lk, s_logit, bits, exp_n, _dev_ptr(v, torch.int8, "v", 3), zp_v, d,
            _dev_ptr(out, torch.int32, "out", 3),
            _dev_ptr(codes_out, torch.uint8, "codes_out", 3), ld, _stream(stream, logits))
    return _invoke("lis_attention_head", args, (logits, bias, v, out, codes_out), prepare, out)


def ptf_calibrate_workspace_bytes(T: int, C: int, K: int = 3) -> int:
    """Bytes of device scratch that ptf_calibrate needs (0 for invalid sizes)."""
    return int(lib().fq_ptf_calibrate_workspace_bytes(T, C, K))


def ptf_calibrate(x, bits: int = 8, K: int = 3, s=None, zp=None, alpha=None, workspace=None,
                  stream=None, prepare: bool = False):
    """PTF calibration of a float [T, C] tensor: returns (s, zp, alpha) as device
    tensors (float64 [1], int32 [1] in container form, uint8 [C]).  The
    workspace is allocated here with torch when not given."""
    import torch
    T, C = x.shape
    s = _empty(x, stream, 1, torch.float64) if s is None else s
    zp = _empty(x, stream, 1, torch.int32) if zp is None else zp
    alpha = _empty(x, stream, C, torch.uint8) if alpha is None else alpha
    need = ptf_calibrate_workspace_bytes(T, C, K) if T > 0 else 0
    if workspace is None:
        workspace = _empty(x, stream, max(need, 1), torch.uint8)
    args = (_dev_ptr(x, torch.float32, "x", 2), T, C, bits, K,
            _dev_ptr(s, torch.float64, "s", 1), _dev_ptr(zp, torch.int32, "zp", 1),
            _dev_ptr(alpha, torch.uint8, "alpha", 1), _dev_ptr(workspace, torch.uint8, "workspace", 1),
            workspace.numel(), _stream(stream, x))
    return _invoke("ptf_calibrate", args, (x, s, zp, alpha, workspace), prepare, (s, zp, alpha))


def ptf_calibrate_noalloc(x, bits: int = 8, K: int = 3, s=None, zp=None, alpha=None,
                          stream=None, prepare: bool = False):
    """ptf_calibrate with the workspace in the library's fixed device scratch:
    the entry point allocates nothing (outputs not given are allocated here,
    by torch, before the call)."""
    import torch
    T, C = x.shape
    s = _empty(x, stream, 1, torch.float64) if s is None else s
    zp = _empty(x, stream, 1, torch.int32) if zp is None else zp
    alpha = _empty(x, stream, C, torch.uint8) if alpha is None else alpha
    args = (_dev_ptr(x, torch.float32, "x", 2), T, C, bits, K,
            _dev_ptr(s, torch.float64, "s", 1), _dev_ptr(zp, torch.int32, "zp", 1),
            _dev_ptr(alpha, torch.uint8, "alpha", 1), _stream(stream, x))
    return _invoke("ptf_calibrate_noalloc", args, (x, s, zp, alpha), prepare, (s, zp, alpha))


def ptf_quantize_int8(x, s, zp, alpha, bits: int = 8, x_q=None, stream=None,
                      prepare: bool = False):
    """PTF quantization of a float [T, C] tensor with device scalars s, zp (as
    returned by ptf_calibrate) and alpha [C]; returns (or fills) int8 [T, C]."""
    import torch
    T, C = x.shape
    if x_q is None:
        x_q = _empty(x, stream, (T, C), torch.int8)
    if alpha.shape != (C,) or x_q.shape != (T, C):
        raise ValueError("alpha must be [C] and x_q [T, C]")
    args = (_dev_ptr(x, torch.float32, "x", 2), T, C, _dev_ptr(s, torch.float64, "s", 1),
            _dev_ptr(zp, torch.int32, "zp", 1), _dev_ptr(alpha, torch.uint8, "alpha", 1), bits,
            _dev_ptr(x_q, torch.int8, "x_q", 2), _stream(stream, x))
    return _invoke("ptf_quantize_int8", args, (x, s, zp, alpha, x_q), prepare, x_q)


def requant_dyadic_int8(q, s_in: float, s_out: float, zp_out: int, bits: int = 8, y=None,
                        stream=None, prepare: bool = False):
    """Dyadic requantization of an int32 tensor (any shape, contiguous) to the
    int8 container; returns (or fills) int8 of the same shape."""
    import torch
    if y is None:
        y = _empty(q, stream, q.shape, torch.int8)
    if y.shape != q.shape:
        raise ValueError("y must have the shape of q")
    args = (_dev_ptr(q, torch.int32, "q"), q.numel(), s_in, s_out, zp_out, bits,
            _dev_ptr(y, torch.int8, "y"), _stream(stream, q))
    return _invoke("requant_dyadic_int8", args, (q, y), prepare, y)


def lis_attention_qk(q, k, v, s_logit: float, zp_q: int = 0, zp_k: int = 0, bits: int = 4,
                     exp_n: int = 20, zp_v: int = 0, bias=None, out=None, stream=None,
                     prepare: bool = False):
    """Integer-only attention from int8 q [G, Lq, dk], k [G, Lk, dk] and
    v [G, Lk, d]; returns (or fills) int32 [G, Lq, d]."""
    import torch
    G, Lq, dk = q.shape
    Lk = k.shape[1]
    d = v.shape[2]
    if k.shape != (G, Lk, dk) or v.shape[:2] != (G, Lk):
        raise ValueError("k must be [G, Lk, dk] and v [G, Lk, d]")
    if out is None:
        out = _empty(q, stream, (G, Lq, d), torch.int32)
    Hb = bias.shape[0] if bias is not None else 0
    args = (_dev_ptr(q, torch.int8, "q", 3), _dev_ptr(k, torch.int8, "k", 3), zp_q, zp_k, dk,
            _dev_ptr(bias, torch.int32, "bias", 3), Hb, G, Lq, Lk, s_logit, bits, exp_n,
            _dev_ptr(v, torch.int8, "v", 3), zp_v, d, _dev_ptr(out, torch.int32, "out", 3),
            _stream(stream, q))
    return _invoke("lis_attention_qk", args, (q, k, v, bias, out), prepare, out)


def linear_fold_int8(w, s_w, s_x: float, s_y: float = 1.0, zp_x: int = 0, bias=None, fold=None,
                     mul=None, stream=None, prepare: bool = False):
    """What a linear layer's products take besides its int8 weights w [N, K]:
    (fold, mul), the folded bias (int32 [N]) and the channels' multipliers
    (float [N]), from the weight scales s_w [N], the input's scale and zero
    point, the float bias [N] and the output's step s_y (the table's step where
    an activation table follows).  Once for a layer."""
    import torch
    N, K = _dims(w, 2, "w")
    dev = w.get_device()
    if fold is None:
        fold = _empty(w, stream, N, torch.int32)
    if mul is None:
        mul = _empty(w, stream, N, torch.float32)
    specs = [("w", w, torch.int8, (N, K)), ("s_w", s_w, torch.float32, (N,)),
             ("fold", fold, torch.int32, (N,)), ("mul", mul, torch.float32, (N,))]
    if bias is not None:
        specs.append(("bias", bias, torch.float32, (N,)))
    for _, t, dtype, shape in specs:
        if not (hasattr(t, "is_contiguous") and t.dtype is dtype and t.shape == shape
                and t.is_contiguous() and t.get_device() == dev >= 0):
            _refuse(dev, *specs)
    args = (w.data_ptr(), N, K, s_w.data_ptr(), None if bias is None else bias.data_ptr(), zp_x, s_x,
            s_y, fold.data_ptr(), mul.data_ptr(), _raw_stream(stream, dev))
    return _invoke("linear_fold_int8", args, (w, s_w, bias, fold, mul), prepare, (fold, mul), dev)


def linear_int8(x, w, fold, mul, zp_y: int = 0, bits: int = 8, relu: bool = False, table=None,
                zp_t: Optional[int] = None, residual=None, zp_r: int = 0, mul_r: float = 1.0,
                y=None, stream=None, prepare: bool = False):
    """Linear layer with its epilogue: int8 [T, N] from int8 x [T, K] and w [N, K]
    with fold and mul of linear_fold_int8.  relu, or an activation table
    (activation_table; zp_t defaults to its middle); residual int8 [T, N] with
    zero point zp_r and mul_r = s_r / s_y is added after the activation.  y may
    be the residual."""
    import torch
    i8, i32, f32 = torch.int8, torch.int32, torch.float32
    T, K = _dims(x, 2, "x")
    N = w.shape[0]
    dev = x.get_device()
    act, bits_t, size = ACT_NONE, 0, 0
    if table is not None:
        if relu:
            raise ValueError("give relu or a table, not both")
        act, size = ACT_TABLE, table.numel()
        bits_t = size.bit_length() - 1
        if size != 1 << bits_t:
            raise ValueError("table must hold a power of two of values")
        if zp_t is None:
            zp_t = size >> 1
    elif relu:
        act = ACT_RELU
    if y is None:
        y = x.new_empty((T, N)) if stream is None else _empty(x, stream, (T, N), i8)
    try:
        fits = (x.dtype is i8 and x.is_contiguous() and dev >= 0
                and w.dtype is i8 and w.shape == (N, K) and w.is_contiguous()
                and w.get_device() == dev
                and mul.dtype is f32 and mul.shape == (N,) and mul.is_contiguous()
                and mul.get_device() == dev
                and y.dtype is i8 and y.shape == (T, N) and y.is_contiguous()
                and y.get_device() == dev
                and (fold is None or fold.dtype is i32 and fold.shape == (N,)
                     and fold.is_contiguous() and fold.get_device() == dev)
                and (table is None or table.dtype is f32 and table.shape == (size,)
                     and table.is_contiguous() and table.get_device() == dev)
                and (residual is None or residual.dtype is i8 and residual.shape == (T, N)
                     and residual.is_contiguous() and residual.get_device() == dev))
    except AttributeError:
        fits = False
    if not fits:
        _refuse(dev, ("x", x, i8, (T, K)), ("w", w, i8, (N, K)), ("mul", mul, f32, (N,)),
                *[s for s in (("fold", fold, i32, (N,)), ("table", table, f32, (size,)),
                              ("residual", residual, i8, (T, N))) if s[1] is not None],
                ("y", y, i8, (T, N)))
    args = (x.data_ptr(), T, w.data_ptr(), N, K, None if fold is None else fold.data_ptr(),
            mul.data_ptr(), act, None if table is None else table.data_ptr(), bits_t, zp_t or 0,
            None if residual is None else residual.data_ptr(), zp_r, mul_r, zp_y, bits, y.data_ptr(),
            _raw_stream(stream, dev))
    return _invoke("linear_int8", args, (x, w, fold, mul, table, residual, y), prepare, y, dev)


def linear_int32(x, w, fold=None, out=None, stream=None, prepare: bool = False):
    """The linear layer's accumulators: int32 [T, N] = x w^T + fold."""
    import torch
    i8, i32 = torch.int8, torch.int32
    T, K = _dims(x, 2, "x")
    N = w.shape[0]
    dev = x.get_device()
    if out is None:
        out = _empty(x, stream, (T, N), i32)
    try:
        fits = (x.dtype is i8 and x.is_contiguous() and dev >= 0
                and w.dtype is i8 and w.shape == (N, K) and w.is_contiguous()
                and w.get_device() == dev
                and out.dtype is i32 and out.shape == (T, N) and out.is_contiguous()
                and out.get_device() == dev
                and (fold is None or fold.dtype is i32 and fold.shape == (N,)
                     and fold.is_contiguous() and fold.get_device() == dev))
    except AttributeError:
        fits = False
    if not fits:
        _refuse(dev, ("x", x, i8, (T, K)), ("w", w, i8, (N, K)),
                *([] if fold is None else [("fold", fold, i32, (N,))]), ("out", out, i32, (T, N)))
    args = (x.data_ptr(), T, w.data_ptr(), N, K, None if fold is None else fold.data_ptr(),
            out.data_ptr(), _raw_stream(stream, dev))
    return _invoke("linear_int32", args, (x, w, fold, out), prepare, out, dev)


def activation_table(kind: str, s_t: float, s_y: float, zp_t: Optional[int] = None,
                     table_bits: int = 10, device="cuda"):
    """An activation ("gelu", "gelu_tanh" or "silu") as a table for linear_int8:
    its values in steps s_y of the output over the grid s_t (u - zp_t) of
    2^table_bits inputs (zp_t defaults to the middle)."""
    import torch
    if kind not in _FUNCTIONS:
        raise ValueError(f"kind must be one of {', '.join(_FUNCTIONS)}")
    if not 4 <= table_bits <= 12:
        raise ValueError("table_bits must be in [4, 12]")
    host = torch.empty(1 << table_bits, dtype=torch.float32)
    zp_t = (1 << table_bits) >> 1 if zp_t is None else zp_t
    args = (_FUNCTIONS[kind], s_t, zp_t, table_bits, s_y, host.data_ptr())
    _narrow("fq_activation_table", args)
    _check("fq_activation_table", lib().fq_activation_table(*args))
    return host.to(device)


def rope_table_int16(positions, freq, axis, table=None, stream=None, prepare: bool = False):
    """cos and sin of positions int32 [axes, T] times freq float64 [P], pair p
    along axis[p] (uint8 [P]), in steps of 2^-14: int16 [T, P, 2]."""
    import torch
    i32, f64, u8, i16 = torch.int32, torch.float64, torch.uint8, torch.int16
    axes, T = _dims(positions, 2, "positions")
    P, = _dims(freq, 1, "freq")
    dev = positions.get_device()
    if table is None:
        table = _empty(positions, stream, (T, P, 2), i16)
    try:
        fits = (positions.dtype is i32 and positions.is_contiguous() and dev >= 0
                and freq.dtype is f64 and freq.is_contiguous() and freq.get_device() == dev
                and axis.dtype is u8 and axis.shape == (P,) and axis.is_contiguous()
                and axis.get_device() == dev
                and table.dtype is i16 and table.shape == (T, P, 2) and table.is_contiguous()
                and table.get_device() == dev)
    except AttributeError:
        fits = False
    if not fits:
        _refuse(dev, ("positions", positions, i32, (axes, T)), ("freq", freq, f64, (P,)),
                ("axis", axis, u8, (P,)), ("table", table, i16, (T, P, 2)))
    args = (positions.data_ptr(), axes, T, freq.data_ptr(), axis.data_ptr(), P, table.data_ptr(),
            _raw_stream(stream, dev))
    return _invoke("rope_table_int16", args, (positions, freq, axis, table), prepare, table, dev)


def rope_qkv_int8(qkv, table, Hq: int, Hkv: int, s_x: float, s_q: float, s_k: float, zp_x: int = 0,
                  zp_q: int = 0, zp_k: int = 0, bits: int = 8, interleaved: bool = False, q=None,
                  k=None, v=None, stream=None, prepare: bool = False):
    """The query-key-value layer's int8 rows [B, L, (Hq + 2 Hkv) d] split into
    heads, queries and keys rotated by the table (int16 [L or B L, P, 2]; None:
    no rotation) and requantized: (q [B, Hq, L, d], k and v [B, Hkv, L, d])."""
    import torch
    i8, i16 = torch.int8, torch.int16
    B, L, row = _dims(qkv, 3, "qkv")
    heads = Hq + 2 * Hkv
    if Hq < 1 or Hkv < 1 or row % heads:
        raise ValueError("qkv must be [B, L, (Hq + 2 Hkv) d]")
    d = row // heads
    dev = qkv.get_device()
    rows, P = (0, 0) if table is None else _dims(table, 3, "table")[:2]
    sq, sk = (B, Hq, L, d), (B, Hkv, L, d)
    new = qkv.new_empty if stream is None else lambda shape: _empty(qkv, stream, shape, i8)
    if q is None:
        q = new(sq)
    if k is None:
        k = new(sk)
    if v is None:
        v = new(sk)
    try:
        fits = (qkv.dtype is i8 and qkv.is_contiguous() and dev >= 0
                and (table is None or table.dtype is i16 and table.shape == (rows, P, 2)
                     and table.is_contiguous() and table.get_device() == dev)
                and q.dtype is i8 and q.shape == sq and q.is_contiguous() and q.get_device() == dev
                and k.dtype is i8 and k.shape == sk and k.is_contiguous() and k.get_device() == dev
                and v.dtype is i8 and v.shape == sk and v.is_contiguous() and v.get_device() == dev)
    except AttributeError:
        fits = False
    if not fits:
        _refuse(dev, ("qkv", qkv, i8, (B, L, row)),
                *([] if table is None else [("table", table, i16, (rows, P, 2))]),
                ("q", q, i8, sq), ("k", k, i8, sk), ("v", v, i8, sk))
    args = (qkv.data_ptr(), B, L, Hq, Hkv, d, s_x, zp_x, None if table is None else table.data_ptr(),
            rows, P, 1 if interleaved else 0, s_q, zp_q, s_k, zp_k, bits, q.data_ptr(), k.data_ptr(),
            v.data_ptr(), _raw_stream(stream, dev))
    return _invoke("rope_qkv_int8", args, (qkv, table, q, k, v), prepare, (q, k, v), dev)


def requant_heads_int8(q, s_in: float, s_out: float, zp_out: int, bits: int = 8, y=None,
                       stream=None, prepare: bool = False):
    """Dyadic requantization of an attention result int32 [B, H, L, d] with its
    heads brought back to rows: int8 [B, L, H d]."""
    import torch
    i8, i32 = torch.int8, torch.int32
    B, H, L, d = _dims(q, 4, "q")
    dev = q.get_device()
    if y is None:
        y = _empty(q, stream, (B, L, H * d), i8)
    try:
        fits = (q.dtype is i32 and q.is_contiguous() and dev >= 0
                and y.dtype is i8 and y.shape == (B, L, H * d) and y.is_contiguous()
                and y.get_device() == dev)
    except AttributeError:
        fits = False
    if not fits:
        _refuse(dev, ("q", q, i32, (B, H, L, d)), ("y", y, i8, (B, L, H * d)))
    args = (q.data_ptr(), B, H, L, d, s_in, s_out, zp_out, bits, y.data_ptr(),
            _raw_stream(stream, dev))
    return _invoke("requant_heads_int8", args, (q, y), prepare, y, dev)
