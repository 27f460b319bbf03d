"""Binding of libcelty's operators around the products of a decoding step
(include/celty_decode.h): block norm, the 4-bit key/value cache with its
attention, and sampling.  As in the package's other bindings the functions
carry the C names and only marshal arguments; everything is re-exported by the
package.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

from . import _check, _f32, _i32, _i64, _p, _sig, _stream_handle, _sz, _torch

NORM_RMS, NORM_LAYER = 0, 1
_NORM_KINDS = {"rms": NORM_RMS, "layer": NORM_LAYER}


class celty_norm(ctypes.Structure):
    _fields_ = [("kind", _i32), ("post", _i32), ("eps", _f32), ("alpha", _f32), ("w_pre", _p), ("b_pre", _p),
                ("w_post", _p), ("b_post", _p), ("gate", _p), ("ld_gate", _i64)]


class celty_kv4_cache(ctypes.Structure):
    _fields_ = [("head_dim", _i32), ("kv_heads", _i32), ("page_tokens", _i32), ("n_pages", _i32), ("k_codes", _p),
                ("v_codes", _p), ("k_params", _p), ("v_params", _p)]


class celty_kv4_seqs(ctypes.Structure):
    _fields_ = [("n_seqs", _i32), ("n_tokens", _i32), ("max_pages", _i32), ("table_stride", _i32), ("block_table", _p),
                ("kv_len", _p), ("q_start", _p)]


class celty_heads(ctypes.Structure):
    _fields_ = [("data", _p), ("token_stride", _i64), ("head_stride", _i64)]


class celty_filters(ctypes.Structure):
    _fields_ = [("temperature", _p), ("top_k", _p), ("top_p", _p), ("min_p", _p)]


_ptr = ctypes.POINTER
_norm = _sig("celty_block_norm", ctypes.c_int, _i32, _i32, _ptr(celty_norm), _i32, _i32, _p, _i64, _p, _i64, _p, _i64, _p,
             _i64, _p)
_append = _sig("celty_kv4_append", ctypes.c_int, _ptr(celty_kv4_cache), _ptr(celty_kv4_seqs), _i32, _ptr(celty_heads),
               _ptr(celty_heads), _p)
_gather = _sig("celty_kv4_gather", ctypes.c_int, _ptr(celty_kv4_cache), _ptr(celty_kv4_seqs), _i32, _ptr(celty_heads),
               _ptr(celty_heads), _p)
_attention = _sig("celty_kv4_attention", ctypes.c_int, _ptr(celty_kv4_cache), _ptr(celty_kv4_seqs), _i32, _i32,
                  _ptr(celty_heads), _ptr(celty_heads), _f32, _i32, _p, _sz, _p)
_attention_ws = _sig("celty_kv4_attention_workspace_bytes", _sz, _ptr(celty_kv4_cache), _ptr(celty_kv4_seqs), _i32)
_sample = _sig("celty_sample", ctypes.c_int, _i32, _i32, _i32, _p, _i64, _p, _i64, _ptr(celty_filters), _p, _p, _sz, _p)
_sample_ws = _sig("celty_sample_workspace_bytes", _sz, _i32, _i32)

_HALVES = ("float16", "bfloat16")
_FLOATS = ("float16", "bfloat16", "float32")
_dtype_codes = {}


def _dtype_code(dtype, name: str, allowed=_HALVES) -> int:
    if not _dtype_codes:
        torch = _torch()
        _dtype_codes.update({torch.float16: 0, torch.bfloat16: 1, torch.float32: 2})
    code = _dtype_codes.get(dtype, 3)
    if code >= len(allowed):
        raise ValueError(f"{name} has dtype {dtype}; expected one of {', '.join(allowed)}")
    return code


def _on(t, dev: int, name: str):
    """t must be on the GPU of index dev."""
    if t.get_device() != dev:
        if not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
        raise ValueError(f"{name} is on {t.device}, the call's other tensors on cuda:{dev}")


def _vector(t, n: int, dtype, dev: int, name: str) -> Optional[int]:
    """Address of a contiguous vector of at least n elements, or None."""
    if t is None:
        return None
    if t.get_device() != dev:
        _on(t, dev, name)
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements")
    return t.data_ptr()


def _rows(t, rows: int, n: int, dtype, dev: int, name: str):
    """(address, row stride) of a rows x n matrix with contiguous rows."""
    if t.get_device() != dev:
        _on(t, dev, name)
    if t.dtype is not dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.dim() != 2 or t.size(0) != rows or t.size(1) != n:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected ({rows}, {n})")
    ld, step = t.stride()
    if step != 1 and n > 1:
        raise ValueError(f"{name} must have contiguous rows")
    return t.data_ptr(), ld if rows > 1 else n


def _gpu(t, name: str) -> int:
    """Index of the GPU that t is on."""
    dev = t.get_device()
    if dev < 0 or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return dev


def _stream_on(stream, dev: int) -> int:
    """The stream's handle.  A launch goes to the current GPU, so that must be
    the tensors', and a given stream's as well."""
    c = _torch()._C
    current = c._cuda_getDevice()
    if current != dev:
        raise ValueError(f"the call's tensors are on cuda:{dev}, the current device is cuda:{current}")
    if stream is None:
        return c._cuda_getCurrentRawStream(dev)   # without a stream object, as _stream_handle
    given = getattr(stream, "device", None)
    if given is not None and given.index is not None and given.index != dev:
        raise ValueError(f"the call's tensors are on cuda:{dev}, its stream on {given}")
    return _stream_handle(stream)


def celty_block_norm(h, b, h_out=None, x=None, *, kind: str = "rms", w_pre=None, b_pre=None, w_post=None, b_post=None,
                     gate=None, alpha: float = 1.0, eps: float = 1e-5, post: Optional[bool] = None, stream=None) -> None:
    """h_out = h + alpha * gate * u and x = norm(h_out) * w_pre + b_pre, with
    u = norm(b) * w_post + b_post where `post` (by default: where w_post is
    given), else b.  h and b are rows x n; b may be None (no update), so may
    h_out or x (not written).  gate holds n elements or rows x n."""
    if h.dim() != 2:
        raise ValueError("h must be 2-D (rows x n)")
    rows, n = h.shape
    dev = _gpu(h, "h")
    if x is None and h_out is None:
        raise ValueError("nothing to write: give h_out or x")
    t = x if b is None else b
    torch = _torch()
    res_dtype = h.dtype
    # h alone: the block's type is of no matter
    dtype = t.dtype if t is not None else torch.float16 if res_dtype is torch.float32 else res_dtype
    code = _dtype_code(dtype, "b" if b is not None else "x")
    if res_dtype is not dtype and res_dtype is not torch.float32:
        raise ValueError(f"h has dtype {res_dtype}; expected {dtype} or torch.float32")
    res = _dtype_code(res_dtype, "h", _FLOATS)
    hp, ldh = _rows(h, rows, n, res_dtype, dev, "h")
    bp, ldb = _rows(b, rows, n, dtype, dev, "b") if b is not None else (None, 0)
    op, ldo = _rows(h_out, rows, n, res_dtype, dev, "h_out") if h_out is not None else (None, 0)
    xp, ldx = _rows(x, rows, n, dtype, dev, "x") if x is not None else (None, 0)
    gp, ldg = None, 0
    if gate is not None:
        if gate.dim() == 2:
            gp, ldg = _rows(gate, rows, n, dtype, dev, "gate")
        else:
            gp = _vector(gate, n, dtype, dev, "gate")
    if kind not in _NORM_KINDS:
        raise ValueError(f"kind must be 'rms' or 'layer', not {kind!r}")
    a = celty_norm(_NORM_KINDS[kind], w_post is not None if post is None else bool(post), eps, alpha,
                   _vector(w_pre, n, dtype, dev, "w_pre"), _vector(b_pre, n, dtype, dev, "b_pre"),
                   _vector(w_post, n, dtype, dev, "w_post"), _vector(b_post, n, dtype, dev, "b_post"), gp, ldg)
    status = _norm(rows, n, a, code, res, hp, ldh, bp, ldb, op, ldo, xp, ldx, _stream_on(stream, dev))
    if status:
        _check(status, "celty_block_norm")


# ---------------------------------------------------------------------------
# The key/value cache
# ---------------------------------------------------------------------------
class Kv4Cache:
    """A key/value cache in 4 bits: four device tensors and their descriptor."""

    def __init__(self, n_pages: int, kv_heads: int, head_dim: int, page_tokens: int = 64, device=None):
        torch = _torch()
        z = dict(device=torch.device("cuda") if device is None else torch.device(device))
        self._set(torch.zeros(n_pages, kv_heads, page_tokens, head_dim // 2, dtype=torch.uint8, **z),
                  torch.zeros(n_pages, kv_heads, page_tokens // 8, head_dim, dtype=torch.int32, **z),
                  torch.zeros(n_pages, kv_heads, page_tokens, 2, dtype=torch.float16, **z),
                  torch.zeros(n_pages, kv_heads, page_tokens, 2, dtype=torch.float16, **z))

    @classmethod
    def from_tensors(cls, k_codes, v_codes, k_params, v_params) -> "Kv4Cache":
        """A cache over existing tensors (the layouts of celty_kv4_cache)."""
        self = object.__new__(cls)
        self._set(k_codes, v_codes, k_params, v_params)
        return self

    def _set(self, k_codes, v_codes, k_params, v_params):
        torch = _torch()
        if k_codes.dim() != 4:
            raise ValueError("k_codes must be 4-D (pages, heads, tokens, head_dim / 2)")
        P, H, page, half = k_codes.shape
        dev = _gpu(k_codes, "k_codes")
        for name, t, shape, dtype in (("k_codes", k_codes, (P, H, page, half), torch.uint8),
                                      ("v_codes", v_codes, (P, H, page // 8, 2 * half), torch.int32),
                                      ("k_params", k_params, (P, H, page, 2), torch.float16),
                                      ("v_params", v_params, (P, H, page, 2), torch.float16)):
            _on(t, dev, name)
            if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape}")
        if 2 * half not in (64, 128) or page < 32 or page & (page - 1):
            raise ValueError(f"head_dim {2 * half} must be 64 or 128, page_tokens {page} a power of two of at least 32")
        self.k_codes, self.v_codes, self.k_params, self.v_params = k_codes, v_codes, k_params, v_params
        self.n_pages, self.kv_heads, self.page_tokens, self.head_dim, self.device = P, H, page, 2 * half, k_codes.device
        self._dev = dev
        self._desc = celty_kv4_cache(2 * half, H, page, P, k_codes.data_ptr(), v_codes.data_ptr(), k_params.data_ptr(),
                                     v_params.data_ptr())

    def desc(self) -> celty_kv4_cache:
        return self._desc


class Kv4Seqs:
    """The sequences of a call: block_table [n_seqs, max_pages], kv_len
    [n_seqs] (the call's new tokens included) and q_start [n_seqs + 1], the
    first of the call's tokens of each sequence (None: one token each); int32
    device tensors, read when the kernels run."""

    def __init__(self, block_table, kv_len, q_start=None):
        torch = _torch()
        if block_table.dim() != 2 or block_table.dtype != torch.int32 or (block_table.shape[1] > 1 and block_table.stride(1) != 1):
            raise ValueError("block_table must be a 2-D int32 tensor with contiguous rows")
        n, cols = block_table.shape
        dev = _gpu(block_table, "block_table")
        self.n_seqs, self._dev, self._desc = n, dev, None
        self.block_table, self.kv_len, self.q_start = block_table, kv_len, q_start
        self._args = (n, cols, max(block_table.stride(0), cols) if n > 1 else cols, block_table.data_ptr(),
                      _vector(kv_len, n, torch.int32, dev, "kv_len"),
                      _vector(q_start, n + 1, torch.int32, dev, "q_start"))
        if n > 1 and block_table.stride(0) < cols:
            raise ValueError("block_table's rows overlap")

    def desc(self, n_tokens: int) -> celty_kv4_seqs:
        d = self._desc
        if d is None or d.n_tokens != n_tokens:
            n, cols, stride, table, kv_len, q_start = self._args
            if q_start is None and n_tokens != n:
                raise ValueError(f"{n_tokens} tokens for {n} sequences need q_start")
            d = self._desc = celty_kv4_seqs(n, n_tokens, cols, stride, table, kv_len, q_start)
        return d


def _heads(t, heads: Optional[int], cache: Kv4Cache, name: str, like=None) -> celty_heads:
    if t.get_device() != cache._dev:
        _on(t, cache._dev, name)
    if t.dim() != 3 or t.size(2) != cache.head_dim or (heads is not None and t.size(1) != heads):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected (tokens, {heads if heads else 'heads'}, {cache.head_dim})")
    if like is not None and (t.dtype is not like.dtype or t.shape != like.shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)} and dtype {t.dtype}, expected {tuple(like.shape)} and {like.dtype}")
    token, head, step = t.stride()
    if step != 1:
        raise ValueError(f"{name} must have contiguous channels")
    return celty_heads(t.data_ptr(), token if t.size(0) > 1 else 0, head if t.size(1) > 1 else 0)


def _same_gpu(cache: Kv4Cache, seqs: Kv4Seqs) -> None:
    if seqs._dev != cache._dev:
        raise ValueError(f"the sequences are on cuda:{seqs._dev}, the cache on cuda:{cache._dev}")


def _move(f, where, cache: Kv4Cache, seqs: Kv4Seqs, k, v, stream):
    kh = _heads(k, cache.kv_heads, cache, "k")
    vh = _heads(v, cache.kv_heads, cache, "v", k)
    _same_gpu(cache, seqs)
    status = f(cache._desc, seqs.desc(k.size(0)), _dtype_code(k.dtype, "k"), kh, vh, _stream_on(stream, cache._dev))
    if status:
        _check(status, where)


def celty_kv4_append(cache: Kv4Cache, seqs: Kv4Seqs, k, v, stream=None) -> None:
    """Quantise new keys and values (tokens x kv_heads x head_dim) into the cache."""
    _move(_append, "celty_kv4_append", cache, seqs, k, v, stream)


def celty_kv4_gather(cache: Kv4Cache, seqs: Kv4Seqs, k, v, stream=None) -> None:
    """Read the same tokens back into k and v as the numbers the cache stands for."""
    _move(_gather, "celty_kv4_gather", cache, seqs, k, v, stream)


def celty_kv4_attention_workspace_bytes(cache: Kv4Cache, seqs: Kv4Seqs, n_tokens: int, heads: int) -> int:
    s = seqs.desc(int(n_tokens))
    return int(_attention_ws(ctypes.byref(cache._desc), ctypes.byref(s), int(heads)))


def new_kv4_workspace(cache: Kv4Cache, seqs: Kv4Seqs, n_tokens: int, heads: int):
    """A zero-filled device workspace for celty_kv4_attention (uint8 tensor)."""
    n = celty_kv4_attention_workspace_bytes(cache, seqs, n_tokens, heads)
    if n == 0:
        raise ValueError("sizes that celty_kv4_attention refuses")
    return _torch().zeros(n, dtype=_torch().uint8, device=cache.device)


def celty_kv4_attention(cache: Kv4Cache, seqs: Kv4Seqs, q, out, workspace, scale: Optional[float] = None, window: int = 0,
                        stream=None) -> None:
    """Causal attention of q (tokens x heads x head_dim) over the cache into
    out.  scale defaults to 1 / sqrt(head_dim); window > 0 limits each token to
    that many positions, its own included."""
    qh = _heads(q, None, cache, "q")
    oh = _heads(out, None, cache, "out", q)
    _same_gpu(cache, seqs)
    if scale is None:
        scale = 1.0 / math.sqrt(cache.head_dim)
    status = _attention(cache._desc, seqs.desc(q.size(0)), _dtype_code(q.dtype, "q"), q.size(1), qh, oh, scale, window,
                        _vector(workspace, 0, _torch().uint8, cache._dev, "workspace"), workspace.numel(),
                        _stream_on(stream, cache._dev))
    if status:
        _check(status, "celty_kv4_attention")


# ---------------------------------------------------------------------------
# Sampling
# ---------------------------------------------------------------------------
def celty_sample_workspace_bytes(rows: int, V: int) -> int:
    return int(_sample_ws(int(rows), int(V)))


def new_sample_workspace(logits):
    """A device workspace for celty_sample over logits' shape (uint8 tensor)."""
    return _torch().empty(celty_sample_workspace_bytes(*logits.shape), dtype=_torch().uint8, device=logits.device)


def celty_sample(logits, noise, tokens, workspace, temperature=None, top_k=None, top_p=None, min_p=None, stream=None) -> None:
    """One token (int32) per row of logits; noise holds independent draws of
    the exponential distribution (None: the largest logit).  temperature,
    top_p and min_p are float32 and top_k int32 device vectors of one value
    per row, or None."""
    torch = _torch()
    if logits.dim() != 2:
        raise ValueError("logits must be 2-D (rows x vocabulary)")
    rows, V = logits.shape
    dev = _gpu(logits, "logits")
    lp, ldl = _rows(logits, rows, V, logits.dtype, dev, "logits")
    np_, ldn = _rows(noise, rows, V, torch.float32, dev, "noise") if noise is not None else (None, 0)
    f = celty_filters(_vector(temperature, rows, torch.float32, dev, "temperature"), _vector(top_k, rows, torch.int32, dev, "top_k"),
                      _vector(top_p, rows, torch.float32, dev, "top_p"), _vector(min_p, rows, torch.float32, dev, "min_p"))
    status = _sample(rows, V, _dtype_code(logits.dtype, "logits", _FLOATS), lp, ldl, np_, ldn, f,
                     _vector(tokens, rows, torch.int32, dev, "tokens"), _vector(workspace, 0, torch.uint8, dev, "workspace"),
                     workspace.numel(), _stream_on(stream, dev))
    if status:
        _check(status, "celty_sample")


__all__ = [
    "NORM_RMS", "NORM_LAYER", "celty_norm", "celty_kv4_cache", "celty_kv4_seqs", "celty_heads", "celty_filters",
    "celty_block_norm", "Kv4Cache", "Kv4Seqs", "celty_kv4_append", "celty_kv4_gather", "celty_kv4_attention",
    "celty_kv4_attention_workspace_bytes", "new_kv4_workspace", "celty_sample", "celty_sample_workspace_bytes",
    "new_sample_workspace",
]
