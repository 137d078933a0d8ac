"""Thin Python binding over the operators of quantised transformer blocks in
libmiconv.so (``include/miquant.h``): the norm with an 8-bit output, the 8-bit
matrix product, the paged 4-bit cache of keys and values, and attention over it.

Argument marshalling only, as in ``miconv``: dtype / device / shape checks, raw
device pointers, torch's current HIP stream, and outputs and a workspace
allocated here when the caller passes none (the C entry points never allocate).
With ``stream=`` these are allocated on that stream, so that its work may use
them at once.  All arithmetic runs in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import miconv
from .miconv import _check, _ptr, _stream

HEAD_DIMS = (32, 64, 96, 128, 192, 256)
_CODE = {torch.float32: 0, torch.bfloat16: 1}


class _Kv4(ctypes.Structure):
    """quant_kv4"""
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_exps", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("v_exps", ctypes.c_void_p), ("pages", ctypes.c_long), ("heads", ctypes.c_int),
                ("page_size", ctypes.c_int), ("head_dim", ctypes.c_int)]


_bound: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """libmiconv.so with the argument types of the quant entry points set."""
    global _bound
    if _bound is None:
        L = miconv.lib()
        i, p, l, f, sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_long, ctypes.c_float, ctypes.c_size_t
        c = ctypes.POINTER(_Kv4)
        L.quant_rmsnorm_i8.argtypes = [l, l, i, p, l, p, l, p, f, p, l, p, l, p, p]
        L.quant_rows_i8.argtypes = [l, l, i, p, l, p, l, p, p]
        L.quant_matmul_workspace_bytes.argtypes = [l, l, l, p, l, p, l]
        L.quant_matmul_i8.argtypes = [l, l, l, p, l, p, p, l, p, p, p, l, i, p, l, i, p, sz, p]
        L.quant_kv4_write.argtypes = [c, l, i, p, l, p, l, p, p]
        L.quant_kv4_read.argtypes = [c, l, p, i, p, l, p, l, p]
        L.quant_attention_workspace_bytes.argtypes = [c, i, i, i, i, i, i]
        L.quant_attention_kv4.argtypes = [c, i, i, l, p, l, p, p, p, i, i, i, f, i, i, p, l, p, sz, p]
        L.quant_matmul_describe.argtypes = [l, l, l, p, l, p, l, i, ctypes.c_char_p, i, ctypes.POINTER(i)]
        L.quant_attention_describe.argtypes = [c, i, i, i, i, i, i, ctypes.c_char_p, i, ctypes.POINTER(i)]
        L.quant_matmul_workspace_bytes.restype = L.quant_attention_workspace_bytes.restype = l
        for name in ("rmsnorm_i8", "rows_i8", "matmul_i8", "kv4_write", "kv4_read", "attention_kv4", "matmul_describe",
                     "attention_describe"):
            getattr(L, "quant_" + name).restype = i
        _bound = L
    return _bound


# ------------------------------------------------------------------ checks
#
# A call's own time on the host matters where one token is in flight, so each
# check is one test in the good case.

_Tensor = torch.Tensor
_getdevice = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_rawstream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _here(t, name: str) -> int:
    """The device of a call's first operand, which has to be the current one, where the call runs."""
    if isinstance(t, _Tensor):
        i = t.get_device()
        if i >= 0 and i == _getdevice():
            return i
        if i < 0:
            raise ValueError(f"{name} must be a device tensor")
        raise ValueError(f"{name} is on device {i}, the current device is {_getdevice()}")
    raise TypeError(f"{name} must be a torch.Tensor")


def _tensor(t, name: str, dev: int, *dtypes) -> None:
    """t has to be a tensor of one of dtypes on device dev."""
    if isinstance(t, _Tensor) and t.get_device() == dev and t.dtype in dtypes:
        return
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(map(str, dtypes))}, got {t.dtype}")
    raise ValueError(f"{name} is on device {t.get_device()}, others are on device {dev}")


def _matrix(t, name: str, dev: int, rows, cols, *dtypes) -> int:
    """A tensor [rows][cols] (None: any) on device dev with dense rows; returns its row stride."""
    _tensor(t, name, dev, *dtypes)
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape != (rows, cols)):
        raise ValueError(f"{name} must be {'[rows][cols]' if rows is None else [rows, cols]}, got {list(shape)}")
    s0, s1 = t.stride()
    n, width = shape
    if (width > 1 and s1 != 1) or (n > 1 and s0 < width):
        raise ValueError(f"{name} must have dense rows that do not overlap")
    return s0 if n > 1 else width


def _heads(t, name: str, dev: int, *dtypes) -> int:
    """A tensor [tokens][heads][channels] on device dev whose tokens are dense; returns the token stride."""
    _tensor(t, name, dev, *dtypes)
    if t.dim() != 3:
        raise ValueError(f"{name} must be [tokens][heads][channels]")
    n, h, d = t.shape
    s0, s1, s2 = t.stride()
    if s2 != 1 or (h > 1 and s1 != d) or (n > 1 and s0 < h * d):
        raise ValueError(f"{name} must be dense within each token, and tokens must not overlap")
    return s0 if n > 1 else h * d


def _vector(t, name: str, dev: int, n: int, dtype) -> None:
    _tensor(t, name, dev, dtype)
    if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a dense vector of {n}")


def _int32(**values) -> None:
    """Numbers that the library takes in 32 bits: ctypes would pass the low ones of a larger number on."""
    if max(values.values()) >= 1 << 31 or min(values.values()) < -1 << 31:
        raise ValueError("must fit 32 bits: " + ", ".join(f"{k} = {v}" for k, v in values.items()))


def _where(dev: int, stream):
    """The stream for work on device dev, the current one: its current stream when None."""
    if stream is not None:
        return _stream(stream)
    return _rawstream(dev) if _rawstream else _stream(None)


def _empty(like, shape, dtype, stream):
    """A tensor on like's device for work of `stream` (None: the current one), so that its memory is free there."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream))
    with torch.cuda.stream(s):
        return like.new_empty(shape, dtype=dtype)


def _workspace(nbytes: int, what: str, ws, like, dev: int, stream):
    if nbytes == 0:
        return None, 0
    if nbytes < 0:
        _check(int(nbytes), what)
    if ws is None:
        ws = _empty(like, nbytes, torch.uint8, stream)
    size = ws.numel() * ws.element_size()
    if ws.get_device() != dev or not ws.is_contiguous() or size < nbytes or ws.data_ptr() % 256:
        raise ValueError(f"workspace must be a 256-byte aligned tensor of at least {nbytes} bytes on the operands' device")
    return ws.data_ptr(), size


# ------------------------------------------------------------------ rows in 8 bits

def _out_i8(x, dev, rows, cols, q, scale, stream):
    if q is None:
        q, qs = _empty(x, (rows, cols), torch.int8, stream), cols
    else:
        qs = _matrix(q, "q", dev, rows, cols, torch.int8)
    if scale is None:
        scale = _empty(x, rows, torch.float32, stream)
    else:
        _vector(scale, "scale", dev, rows, torch.float32)
    return q, qs, scale


def rmsnorm_i8(x, weight=None, residual=None, eps: float = 1e-6, h=None, q=None, scale=None, stream=None):
    """RMS norm of each row of x [rows][cols] (fp32 or bf16), after the residual's addition, as 8-bit integers:
    (q int8 [rows][cols], scale fp32 [rows], h) with q * scale the normed row and h = x + residual in x's type,
    or None without a residual.  h may be residual or x: the addition is then in place."""
    dev = _here(x, "x")
    xs = _matrix(x, "x", dev, None, None, torch.bfloat16, torch.float32)
    rows, cols = x.shape
    t = x.dtype
    if weight is not None:
        _vector(weight, "weight", dev, cols, torch.float32)
    rp = hp = None
    rs = hs = 0
    if residual is not None:
        rs = _matrix(residual, "residual", dev, rows, cols, t)
        if h is None:
            h, hs = _empty(x, (rows, cols), t, stream), cols
        else:
            hs = _matrix(h, "h", dev, rows, cols, t)
        rp, hp = residual.data_ptr(), h.data_ptr()
    elif h is not None:
        raise ValueError("h is the sum with a residual: there is none")
    q, qs, scale = _out_i8(x, dev, rows, cols, q, scale, stream)
    rc = lib().quant_rmsnorm_i8(rows, cols, _CODE[t], x.data_ptr(), xs, rp, rs, _ptr(weight), eps, hp, hs, q.data_ptr(),
                                qs, scale.data_ptr(), _where(dev, stream))
    if rc:
        _check(rc, "quant_rmsnorm_i8")
    return q, scale, h


def rows_i8(x, q=None, scale=None, stream=None):
    """Each row of x [rows][cols] (fp32 or bf16) as 8-bit integers: (q int8, scale fp32 [rows]), q * scale ~ x."""
    dev = _here(x, "x")
    xs = _matrix(x, "x", dev, None, None, torch.bfloat16, torch.float32)
    rows, cols = x.shape
    q, qs, scale = _out_i8(x, dev, rows, cols, q, scale, stream)
    rc = lib().quant_rows_i8(rows, cols, _CODE[x.dtype], x.data_ptr(), xs, q.data_ptr(), qs, scale.data_ptr(),
                             _where(dev, stream))
    if rc:
        _check(rc, "quant_rows_i8")
    return q, scale


# ------------------------------------------------------------------ product of 8-bit integers

def matmul_workspace_bytes(a, w) -> int:
    """Bytes of workspace that matmul_i8 needs for these operands: 0 unless rows are not 16-byte aligned, or 2^23 or
    more bytes apart."""
    dev = _here(a, "a")
    sa, sw = _matrix(a, "a", dev, None, None, torch.int8), _matrix(w, "w", dev, None, None, torch.int8)
    n = lib().quant_matmul_workspace_bytes(a.shape[0], w.shape[0], a.shape[1], a.data_ptr(), sa, w.data_ptr(), sw)
    if n < 0:
        _check(int(n), "quant_matmul_workspace_bytes")
    return int(n)


def _describe(f, what: str, *args):
    buf, n = ctypes.create_string_buffer(256), ctypes.c_int()
    _check(f(*args, buf, 256, ctypes.byref(n)), what)
    return buf.value.decode(), n.value


def matmul_describe(M: int, N: int, K: int, out_dtype=torch.bfloat16, a_stride: Optional[int] = None,
                    w_stride: Optional[int] = None):
    """(kernel names, launch count) of matmul_i8 for operands at 16-byte aligned addresses (strides: dense rows)."""
    return _describe(lib().quant_matmul_describe, "quant_matmul_describe", M, N, K, None, K if a_stride is None else a_stride,
                     None, K if w_stride is None else w_stride, _CODE[out_dtype])


def matmul_i8(a, a_scale, w, w_scale, bias=None, residual=None, relu: bool = False, out=None,
              out_dtype=torch.bfloat16, ws=None, stream=None):
    """act(a_scale[m] * w_scale[n] * (a w^T)[m][n] + bias[n] + residual[m][n]) of a int8 [M][K] and w int8 [N][K];
    fp32 scales [M], [N] and bias [N]; residual [M][N] of the output's type (it may be out).  out_dtype: bf16 or
    fp32, out's where out is given."""
    dev = _here(a, "a")
    sa = _matrix(a, "a", dev, None, None, torch.int8)
    sw = _matrix(w, "w", dev, None, None, torch.int8)
    M, K = a.shape
    N, wk = w.shape
    if wk != K:
        raise ValueError(f"w must be [N][{K}], got {list(w.shape)}")
    _vector(a_scale, "a_scale", dev, M, torch.float32)
    _vector(w_scale, "w_scale", dev, N, torch.float32)
    if bias is not None:
        _vector(bias, "bias", dev, N, torch.float32)
    if out is None:
        if out_dtype not in _CODE:
            raise TypeError("out_dtype must be torch.bfloat16 or torch.float32")
        out, so = _empty(a, (M, N), out_dtype, stream), N
    else:
        so = _matrix(out, "out", dev, M, N, torch.bfloat16, torch.float32)
        out_dtype = out.dtype
    rp, sr = None, 0
    if residual is not None:
        rp, sr = residual.data_ptr(), _matrix(residual, "residual", dev, M, N, out_dtype)
    L = lib()
    ap, wp = a.data_ptr(), w.data_ptr()
    sp, sn = None, 0
    if (K | sa | sw | ap | wp) % 16 or sa >= 1 << 23 or sw >= 1 << 23:   # else no workspace is needed
        sp, sn = _workspace(L.quant_matmul_workspace_bytes(M, N, K, ap, sa, wp, sw), "quant_matmul_i8", ws, a, dev, stream)
    rc = L.quant_matmul_i8(M, N, K, ap, sa, a_scale.data_ptr(), wp, sw, w_scale.data_ptr(), _ptr(bias), rp, sr,
                           _CODE[out_dtype], out.data_ptr(), so, relu, sp, sn, _where(dev, stream))
    if rc:
        _check(rc, "quant_matmul_i8")
    return out


# ------------------------------------------------------------------ the 4-bit cache

class KV4Cache:
    """A paged cache of keys and values in 4 bits: codes uint8 [pages][heads][page_size][head_dim / 2] and exponent
    bytes uint8 [pages][heads][page_size][head_dim / 32] of each (the format: ``include/miquant.h``)."""

    __slots__ = ("k_codes", "k_exps", "v_codes", "v_exps", "pages", "heads", "page_size", "head_dim", "device",
                 "_desc")

    def __init__(self, k_codes, k_exps, v_codes, v_exps):
        dev = k_codes.get_device() if isinstance(k_codes, _Tensor) and k_codes.is_cuda else -2   # not the current one's alone
        _tensor(k_codes, "k_codes", dev, torch.uint8)
        codes = k_codes.shape
        if len(codes) != 4 or 2 * codes[3] not in HEAD_DIMS:
            raise ValueError(f"codes must be [pages][heads][page_size][head_dim / 2], head_dim one of {HEAD_DIMS}")
        pages, heads, page_size, half = codes
        exps = (pages, heads, page_size, half // 16)
        _tensor(k_exps, "k_exps", dev, torch.uint8)
        _tensor(v_codes, "v_codes", dev, torch.uint8)
        _tensor(v_exps, "v_exps", dev, torch.uint8)
        if v_codes.shape != codes or k_exps.shape != exps or v_exps.shape != exps:
            raise ValueError(f"with k_codes {list(codes)} v_codes must be the same and k_exps and v_exps {list(exps)}")
        if not (k_codes.is_contiguous() and k_exps.is_contiguous() and v_codes.is_contiguous() and v_exps.is_contiguous()):
            raise ValueError("codes and exponents must be contiguous")
        if (heads | page_size) >> 31:
            _int32(heads=heads, page_size=page_size)
        self.k_codes, self.k_exps, self.v_codes, self.v_exps = k_codes, k_exps, v_codes, v_exps
        self.pages, self.heads, self.page_size, self.head_dim, self.device = pages, heads, page_size, 2 * half, dev
        self._desc = _Kv4(k_codes.data_ptr(), k_exps.data_ptr(), v_codes.data_ptr(), v_exps.data_ptr(), pages, heads,
                          page_size, 2 * half)

    @classmethod
    def allocate(cls, pages: int, heads: int, page_size: int, head_dim: int, device="cuda") -> "KV4Cache":
        """An empty cache: every value reads as 0."""
        if head_dim not in HEAD_DIMS:
            raise ValueError(f"head_dim must be one of {HEAD_DIMS}")
        new = lambda n: torch.zeros((pages, heads, page_size, n), dtype=torch.uint8, device=device)  # noqa: E731
        return cls(new(head_dim // 2), new(head_dim // 32), new(head_dim // 2), new(head_dim // 32))

    def nbytes(self) -> int:
        return sum(t.numel() for t in (self.k_codes, self.k_exps, self.v_codes, self.v_exps))


def _cache(cache, dev: Optional[int] = None) -> KV4Cache:
    """A cache on device dev (None: any)."""
    if not isinstance(cache, KV4Cache):
        raise TypeError("cache must be a KV4Cache")
    if dev is not None and cache.device != dev:
        raise ValueError(f"the cache is on device {cache.device}, the operands are on device {dev}")
    return cache


def _tokens(t, name, dev, n, cache, *dtypes) -> int:
    s = _heads(t, name, dev, *dtypes)
    if t.shape != (n, cache.heads, cache.head_dim):
        raise ValueError(f"{name} must be {[n, cache.heads, cache.head_dim]}, got {list(t.shape)}")
    return s


def kv4_write(k, v, slots, cache: KV4Cache, stream=None) -> None:
    """Quantises k and v [tokens][heads][head_dim] (fp32 or bf16; tokens may be strided) into the cache at
    slots int32 [tokens] (page * page_size + place; outside the cache: skipped)."""
    dev = _here(k, "k")
    c = _cache(cache, dev)
    n = k.shape[0] if k.dim() == 3 else -1
    ks = _tokens(k, "k", dev, n, c, torch.bfloat16, torch.float32)
    vs = _tokens(v, "v", dev, n, c, k.dtype)
    _vector(slots, "slots", dev, n, torch.int32)
    rc = lib().quant_kv4_write(c._desc, n, _CODE[k.dtype], k.data_ptr(), ks, v.data_ptr(), vs, slots.data_ptr(),
                               _where(dev, stream))
    if rc:
        _check(rc, "quant_kv4_write")


def kv4_read(slots, cache: KV4Cache, k=None, v=None, dtype=torch.bfloat16, stream=None):
    """The keys and values at slots int32 [tokens] as (k, v) [tokens][heads][head_dim] of dtype (bf16 or fp32; both
    hold every value exactly), k's where k is given; zeros for slots outside the cache."""
    c = _cache(cache)
    dev = _here(slots, "slots")
    _cache(c, dev)
    n = slots.shape[0] if slots.dim() == 1 else -1
    _vector(slots, "slots", dev, n, torch.int32)
    if k is not None:
        dtype = k.dtype
    if dtype not in _CODE:
        raise TypeError("dtype must be torch.bfloat16 or torch.float32")
    shape = (n, c.heads, c.head_dim)
    ks = vs = c.heads * c.head_dim
    if k is None:
        k = _empty(slots, shape, dtype, stream)
    else:
        ks = _tokens(k, "k", dev, n, c, dtype)
    if v is None:
        v = _empty(slots, shape, dtype, stream)
    else:
        vs = _tokens(v, "v", dev, n, c, dtype)
    rc = lib().quant_kv4_read(c._desc, n, slots.data_ptr(), _CODE[dtype], k.data_ptr(), ks, v.data_ptr(), vs,
                              _where(dev, stream))
    if rc:
        _check(rc, "quant_kv4_read")
    return k, v


def attention_workspace_bytes(cache: KV4Cache, seqs: int, heads: int, max_new: int, max_len: int, causal: bool = True,
                              window: int = 0) -> int:
    _int32(seqs=seqs, heads=heads, max_new=max_new, max_len=max_len, window=window)
    n = lib().quant_attention_workspace_bytes(_cache(cache)._desc, seqs, heads, max_new, max_len, causal, window)
    if n < 0:
        _check(int(n), "quant_attention_workspace_bytes")
    return int(n)


def attention_describe(cache: KV4Cache, seqs: int, heads: int, max_new: int, max_len: int, causal: bool = True,
                       window: int = 0):
    """(kernel names, launch count) of attention_kv4 with these bounds."""
    _int32(seqs=seqs, heads=heads, max_new=max_new, max_len=max_len, window=window)
    return _describe(lib().quant_attention_describe, "quant_attention_describe", _cache(cache)._desc, seqs, heads, max_new,
                     max_len, causal, window)


def attention_kv4(q, cache: KV4Cache, table, lens, starts=None, max_new: Optional[int] = None,
                  max_len: Optional[int] = None, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                  out=None, ws=None, stream=None):
    """Attention of queries q bf16 [tokens][heads][head_dim] (tokens may be strided) over the cache, which holds
    their own keys and values already.

    table int32 [seqs][pages], contiguous: the pages of each sequence in order; lens int32 [seqs]: its cached tokens;
    starts int32 [seqs + 1]: where its queries begin in q (None: one query each).  max_new and max_len bound the
    queries and the length of any sequence (None: the bounds that the shapes give); work is laid out for these, so
    tight bounds are faster.  scale: head_dim ** -0.5 unless given.  window > 0: only the last `window` places, the
    query's own among them."""
    dev = _here(q, "q")
    c = _cache(cache, dev)
    qs = _heads(q, "q", dev, torch.bfloat16)
    n, heads, d = q.shape
    if d != c.head_dim:
        raise ValueError(f"q has {d} channels a head, the cache {c.head_dim}")
    _tensor(table, "table", dev, torch.int32)
    if table.dim() != 2 or not table.is_contiguous():
        raise ValueError("table must be [seqs][pages], contiguous")
    seqs, width = table.shape
    _vector(lens, "lens", dev, seqs, torch.int32)
    sp = None
    if starts is not None:
        _vector(starts, "starts", dev, seqs + 1, torch.int32)
        sp = starts.data_ptr()
    elif n != seqs:
        raise ValueError(f"without starts q holds one token for each of the {seqs} sequences, got {n}")
    if max_new is None:
        max_new = 1 if starts is None else max(n, 1)
    if max_len is None:
        max_len = width * c.page_size
    if (seqs | heads | width | max_new | max_len | window) >> 31:   # one of them negative or too large
        _int32(seqs=seqs, heads=heads, width=width, max_new=max_new, max_len=max_len, window=window)
    if out is None:
        out, outs = _empty(q, (n, heads, d), torch.bfloat16, stream), heads * d
    else:
        outs = _heads(out, "out", dev, torch.bfloat16)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    L = lib()
    wp, wn = _workspace(L.quant_attention_workspace_bytes(c._desc, seqs, heads, max_new, max_len, causal, window),
                        "quant_attention_kv4", ws, q, dev, stream)
    rc = L.quant_attention_kv4(c._desc, seqs, heads, n, q.data_ptr(), qs, sp, lens.data_ptr(), table.data_ptr(), width,
                               max_new, max_len, d ** -0.5 if scale is None else scale, causal, window, out.data_ptr(),
                               outs, wp, wn, _where(dev, stream))
    if rc:
        _check(rc, "quant_attention_kv4")
    return out
