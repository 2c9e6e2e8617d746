"""Python binding of libc3c's token operators (ctypes): argument marshalling only.

The operators of one layer of a causal transformer over the stream whose
chunks the cached Conv3D layers decode (``include/c3c_tokens.h`` states each):

    linear_i8        matrix product in 8-bit integers, scales per token and channel
    quantize_rows    8-bit rows with a scale each (weights, activations)
    kv_append        rotated queries; keys and values into a paged 8-bit cache
    paged_attention  attention over that cache
    norm_gate        norm after a block, gate, scaled residual, norm before the next

As in :mod:`.c3c`, every step runs in the HIP library on torch's current
stream (or ``stream``), errors are :class:`.c3c.C3CError`, outputs are
allocated with torch where they are not given, and a call uses the workspace
attached to its :class:`.c3c.Context`.  Tensors are contiguous unless a
function says otherwise.

Token tensors of a ``Batch`` are packed: rows ``cu[b] .. cu[b + 1]`` belong to
sequence ``b`` and are the last tokens of its ``len[b]``.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import c3c
from .c3c import _raise, lib

BLOCK = 16  # C3C_KV_BLOCK: tokens that share a scale
DTYPES = dict(c3c.DTYPES, i8=16)
_NAMES = {torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}
_TORCH = {n: d for d, n in _NAMES.items()}
PAIRS = {"half": 0, "next": 1}

_vp, _i64, _int, _f32, _P = C.c_void_p, C.c_int64, C.c_int, C.c_float, C.POINTER


class LinearDesc(C.Structure):
    _fields_ = [(n, _i64) for n in ("M", "N", "K", "ld_x")] + [("x_dtype", C.c_int32), ("y_dtype", C.c_int32)]


class NormDesc(C.Structure):
    _fields_ = [(n, _i64) for n in ("T", "C", "rows_per_gate")] + \
               [("alpha", _f32), ("eps", _f32), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class _CacheDesc(C.Structure):
    _fields_ = [(n, _vp) for n in ("k", "v", "k_scale", "v_scale")] + \
               [(n, _i64) for n in ("pages", "heads", "page", "dim")]


class _BatchDesc(C.Structure):
    _fields_ = [(n, _vp) for n in ("table", "cu", "len")] + \
               [(n, _i64) for n in ("B", "cols", "T", "max_new", "max_len")]


class _RopeDesc(C.Structure):
    _fields_ = [(n, _vp) for n in ("cos", "sin", "pos")] + [("rows", _i64), ("rot", _i64)] + \
               [("pairs", C.c_int32), ("reserved", C.c_int32)]


lib.c3c_quantize_rows.argtypes = [_vp, _i64, _i64, _i64, _int, _vp, _vp, _vp, _vp]
lib.c3c_linear_i8_workspace_bytes.argtypes = [_P(LinearDesc), _P(C.c_size_t)]
lib.c3c_linear_i8.argtypes = [_vp, _P(LinearDesc)] + [_vp] * 7
lib.c3c_norm_gate.argtypes = [_vp, _P(NormDesc)] + [_vp] * 10
lib.c3c_kv_append.argtypes = [_vp, _P(_CacheDesc), _P(_BatchDesc), _P(_RopeDesc), _int, _i64, _vp, _i64, _vp, _i64, _vp,
                              _i64, _vp, _vp]
lib.c3c_paged_attention_workspace_bytes.argtypes = [_P(_CacheDesc), _P(_BatchDesc), _int, _i64, _int, _i64,
                                                    _P(C.c_size_t)]
lib.c3c_paged_attention.argtypes = [_vp, _P(_CacheDesc), _P(_BatchDesc), _int, _i64, _vp, _i64, _f32, _int, _i64, _vp,
                                    _vp, _vp]


# A call of a single token takes a few microseconds on the device: what the
# host does for it is kept short.  torch.cuda.current_stream() alone takes 2.8
# us, the raw handle 0.1.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream, t):
    """The HIP stream of a call: the given one, or the current one of t's device."""
    return _raw_stream(t.get_device()) if stream is None else getattr(stream, "cuda_stream", stream)


def _addr(t, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    return t.data_ptr() or None


def _check(t, name, dtype, shape):
    """The device address of a contiguous tensor of this dtype and shape."""
    if t.dtype is not dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    return t.data_ptr() or None


def _float_dtype(t, name):
    n = _NAMES.get(t.dtype)
    if n is None:
        raise ValueError(f"{name} has dtype {t.dtype}, expected bf16, f16 or f32")
    return n


def _rows(t, name):
    """Stride between the rows of a 2-d tensor whose rows are contiguous."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be 2-d with contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


# ---------------------------------------------------------------- linear

def quantize_rows(ctx, x, q=None, scale=None, stream=None):
    """(q, scale) of x (T, C): q int8 with x ~ q * scale[:, None], scale[t] =
    max|x[t]| / 127.  Rows of x may be strided."""
    dtype, ld = _float_dtype(x, "x"), _rows(x, "x")
    T, n = x.shape
    q = x.new_empty((T, n), dtype=torch.int8) if q is None else q
    scale = x.new_empty(T, dtype=torch.float32) if scale is None else scale
    _raise(lib.c3c_quantize_rows(ctx._h, T, n, ld, DTYPES[dtype], _addr(x, "x"), _check(q, "q", torch.int8, (T, n)),
                                 _check(scale, "scale", torch.float32, (T,)), _stream(stream, x)), ctx, "c3c_quantize_rows")
    return q, scale


def linear_i8_workspace_bytes(M: int, N: int, K: int, x_dtype: str = "bf16", y_dtype: str = "bf16", ld_x=None) -> int:
    """Workspace bytes of a linear_i8 call: the quantised rows of float
    activations, copies of rows that are no multiple of 16 bytes and the
    partial sums of a call that splits K.  ``ld_x``: x's row stride (default K)."""
    n = C.c_size_t()
    d = LinearDesc(M, N, K, K if ld_x is None else ld_x, DTYPES[x_dtype], DTYPES[y_dtype])
    _raise(lib.c3c_linear_i8_workspace_bytes(C.byref(d), C.byref(n)), what="c3c_linear_i8_workspace_bytes")
    return n.value


def linear_i8(ctx, x, w, w_scale, bias=None, x_scale=None, out=None, out_dtype=None, stream=None):
    """y (M, N) = x (M, K) times w (N, K) int8 with w_scale (N,) and bias (N,)
    in fp32.  x is bf16, f16 or f32 (quantised in the call; the context needs
    linear_i8_workspace_bytes), or int8 with x_scale (M,).  Rows of x may be
    strided.  ``out_dtype`` ("bf16", "f16", "f32") defaults to x's, or bf16."""
    i8 = x.dtype == torch.int8
    xd = "i8" if i8 else _float_dtype(x, "x")
    ld = _rows(x, "x")
    M, K = x.shape
    N = w.shape[0]
    yd = out_dtype or (_float_dtype(out, "out") if out is not None else "bf16" if i8 else xd)
    ydt = _TORCH[yd]
    if out is None:
        out = x.new_empty((M, N), dtype=ydt)
    d = LinearDesc(M, N, K, ld, DTYPES[xd], DTYPES[yd])
    st = lib.c3c_linear_i8(
        ctx._h, C.byref(d), _addr(x, "x"), None if x_scale is None else _check(x_scale, "x_scale", torch.float32, (M,)),
        _check(w, "w", torch.int8, (N, K)), _check(w_scale, "w_scale", torch.float32, (N,)),
        None if bias is None else _check(bias, "bias", torch.float32, (N,)), _check(out, "out", ydt, (M, N)),
        _stream(stream, x))
    if st:
        _raise(st, ctx, "c3c_linear_i8")
    return out


# ---------------------------------------------------------------- norms and gate

def norm_gate(ctx, h, y=None, gate=None, *, post=None, pre=None, alpha=1.0, eps=1e-6, rows_per_gate=1, h_out=None,
              u=None, u_q=None, u_scale=None, quantize=False, stream=None):
    """h' = alpha h + gate * (post * n(y)) and u = pre * n(h'), n the RMS norm
    over channels (the header states every omission).  h, y (T, C); gate
    (groups, C), one row for ``rows_per_gate`` tokens; post, pre fp32 (C,).

    Returns (h', u), u None without ``pre``.  ``h_out`` may be h itself.  With
    ``quantize`` u comes as 8-bit rows, and (h', u_q, u_scale) is returned."""
    dtype = _float_dtype(h, "h")
    if h.dim() != 2:
        raise ValueError("h must be 2-d")
    T, n = h.shape
    dt, shape = h.dtype, h.shape
    if h_out is None:
        h_out = torch.empty_like(h)
    if quantize:
        u_q = torch.empty_like(h, dtype=torch.int8) if u_q is None else u_q
        u_scale = h.new_empty(T, dtype=torch.float32) if u_scale is None else u_scale
    elif pre is not None and u is None:
        u = torch.empty_like(h)
    groups = -(-T // rows_per_gate) if rows_per_gate > 0 else 0
    d = NormDesc(T, n, rows_per_gate, alpha, eps, DTYPES[dtype], 0)
    st = lib.c3c_norm_gate(
        ctx._h, C.byref(d), _check(h, "h", dt, shape), None if y is None else _check(y, "y", dt, shape),
        None if gate is None else _check(gate, "gate", dt, (groups, n)),
        None if post is None else _check(post, "post", torch.float32, (n,)),
        None if pre is None else _check(pre, "pre", torch.float32, (n,)), _check(h_out, "h_out", dt, shape),
        None if u is None else _check(u, "u", dt, shape), None if u_q is None else _check(u_q, "u_q", torch.int8, shape),
        None if u_scale is None else _check(u_scale, "u_scale", torch.float32, (T,)), _stream(stream, h))
    if st:
        _raise(st, ctx, "c3c_norm_gate")
    return (h_out, u_q, u_scale) if quantize else (h_out, u)


# ---------------------------------------------------------------- the paged cache

class KVCache:
    """A paged 8-bit cache of keys and values: float8_e4m3fn codes k (pages,
    heads, page, dim) and v (pages, heads, page / 16, dim, 16), fp32 scales
    (pages, heads, page / 16).  Holds its tensors."""

    def __init__(self, k, v, k_scale, v_scale):
        if k.dim() != 4:
            raise ValueError("k must be (pages, heads, page, dim)")
        pages, heads, page, dim = k.shape
        f8, f32, nb = torch.float8_e4m3fn, torch.float32, page // BLOCK
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.heads, self.page, self.dim = heads, page, dim
        self._d = _CacheDesc(_check(k, "k", f8, (pages, heads, page, dim)),
                             _check(v, "v", f8, (pages, heads, nb, dim, BLOCK)),
                             _check(k_scale, "k_scale", f32, (pages, heads, nb)),
                             _check(v_scale, "v_scale", f32, (pages, heads, nb)), pages, heads, page, dim)

    @classmethod
    def empty(cls, pages: int, heads: int, page: int, dim: int, device="cuda"):
        if page % BLOCK:
            raise ValueError(f"page must be a multiple of {BLOCK}")
        nb = page // BLOCK
        codes = [torch.zeros(s, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
                 for s in ((pages, heads, page, dim), (pages, heads, nb, dim, BLOCK))]
        scales = [torch.ones((pages, heads, nb), dtype=torch.float32, device=device) for _ in range(2)]
        return cls(*codes, *scales)


class Batch:
    """The sequences of a step: page table (B, cols), row bounds cu (B + 1,)
    and lengths len (B,), int32 on the device, with host bounds on the new
    tokens and on the length of any sequence.  Holds its tensors: the same
    object serves every layer, and a captured graph, while they are updated in
    place."""

    def __init__(self, table, cu, lens, *, max_new: int, max_len: int):
        if table.dim() != 2:
            raise ValueError("table must be (B, cols)")
        B, cols = table.shape
        self.table, self.cu, self.lens, self.max_new, self.max_len = table, cu, lens, max_new, max_len
        i32 = torch.int32
        self._d = _BatchDesc(_check(table, "table", i32, (B, cols)), _check(cu, "cu", i32, (B + 1,)),
                             _check(lens, "lens", i32, (B,)), B, cols, 0, max_new, max_len)

    def _of(self, T):
        # a descriptor is never changed once a call may have it: threads with
        # contexts of their own share a batch
        d = self._d
        if d.T != T:
            d = _BatchDesc.from_buffer_copy(d)
            d.T = T
            self._d = d
        return C.byref(d)


def _heads(t, name, dtype, T, heads, dim):
    """(address, token stride) of a (T, heads, dim) tensor whose tokens are
    contiguous; they may be strided, as slices of one projection are."""
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.shape != (T, heads, dim):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(T, heads, dim)}")
    by_token, by_head, by_channel = t.stride()
    if by_channel != 1 or (heads > 1 and by_head != dim):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    return _addr(t, name), by_token if T > 1 else heads * dim


def kv_append(ctx, cache: KVCache, batch: Batch, k, v, *, q=None, cos=None, sin=None, pos=None, pairs="half",
              q_out=None, stream=None):
    """Rotates the new tokens' k (and q) by the angle table cos, sin (rows,
    rot / 2) at row pos[t] (default: the token's place in its sequence) and
    stores k and v in the cache.  q (T, q_heads, dim), k, v (T, heads, dim);
    tokens may be strided.  Returns the rotated queries (None without q);
    ``q_out`` may be q itself where that is contiguous."""
    dtype = _float_dtype(k, "k")
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin go together")
    T, dt = k.shape[0], k.dtype
    pk, ldk = _heads(k, "k", dt, T, cache.heads, cache.dim)
    pv, ldv = _heads(v, "v", dt, T, cache.heads, cache.dim)
    pq = ldq = po = qh = 0
    if q is not None:
        qh = q.shape[1]
        pq, ldq = _heads(q, "q", dt, T, qh, cache.dim)
        if q_out is None:
            q_out = k.new_empty((T, qh, cache.dim))
        po = _check(q_out, "q_out", dt, (T, qh, cache.dim))
    elif q_out is not None:
        raise ValueError("q_out goes with q")
    rope = None
    if cos is not None:
        rows, half = cos.shape
        f32 = torch.float32
        rope = C.byref(_RopeDesc(_check(cos, "cos", f32, (rows, half)), _check(sin, "sin", f32, (rows, half)),
                                 None if pos is None else _check(pos, "pos", torch.int32, (T,)), rows, 2 * half,
                                 PAIRS[pairs], 0))
    st = lib.c3c_kv_append(ctx._h, C.byref(cache._d), batch._of(T), rope, DTYPES[dtype], qh, pq or None, ldq, pk, ldk,
                           pv, ldv, po or None, _stream(stream, k))
    if st:
        _raise(st, ctx, "c3c_kv_append")
    return q_out


def paged_attention_workspace_bytes(cache: KVCache, q, batch: Batch, causal: bool = True, window: int = 0) -> int:
    """Workspace bytes with which a call on these queries may split its
    sequences."""
    n = C.c_size_t()
    _raise(lib.c3c_paged_attention_workspace_bytes(C.byref(cache._d), batch._of(q.shape[0]), DTYPES[_float_dtype(q, "q")],
                                                   q.shape[1], int(causal), window, C.byref(n)),
           what="c3c_paged_attention_workspace_bytes")
    return n.value


def paged_attention(ctx, cache: KVCache, batch: Batch, q, *, scale=None, causal: bool = True, window: int = 0, out=None,
                    lse=None, stream=None):
    """Attention of the new tokens' queries q (T, q_heads, dim; tokens may be
    strided) over the cache, which holds the new tokens already: query heads
    share key/value heads in groups, ``causal`` hides later tokens, ``window``
    all but the last ``window``.  scale defaults to dim ** -0.5.  Returns out
    (T, q_heads, dim); ``lse`` (T, q_heads) fp32 receives the log of the sum."""
    dtype = _float_dtype(q, "q")
    T, qh, dim = q.shape
    pq, ldq = _heads(q, "q", q.dtype, T, qh, cache.dim)
    if out is None:
        out = q.new_empty((T, qh, dim))
    st = lib.c3c_paged_attention(
        ctx._h, C.byref(cache._d), batch._of(T), DTYPES[dtype], qh, pq, ldq, dim ** -0.5 if scale is None else scale,
        int(causal), window, _check(out, "out", q.dtype, (T, qh, dim)),
        None if lse is None else _check(lse, "lse", torch.float32, (T, qh)), _stream(stream, q))
    if st:
        _raise(st, ctx, "c3c_paged_attention")
    return out
