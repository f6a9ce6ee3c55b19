"""Operators of the language model's serving layer, which reads the kept
tokens: norm, 4-bit products, append to a paged cache, attention over it.

As in the rest of the binding, the functions only check and marshal torch
tensors.  Each takes tensors of the current GPU, enqueues on torch's current
stream (or ``stream``) and returns without waiting; outputs that are not given
are allocated.  8-bit tensors are torch.float8_e4m3fn throughout.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Optional

import torch

from . import CP_BF16, CP_E4M3, CP_F16, CP_F32, _check, _need, _workspace, library

__all__ = ["rms_norm", "RmsNormResult", "w4_matvec", "kv_append", "paged_attention"]

E4M3 = torch.float8_e4m3fn
_CODE = {torch.float32: CP_F32, torch.bfloat16: CP_BF16, torch.float16: CP_F16, E4M3: CP_E4M3}
_HALF = (torch.bfloat16, torch.float16)


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _on(stream, dev) -> int:
    if dev.type != "cuda":
        raise ValueError(f"tensors must be on the GPU, got {dev}")
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _scales(t, name, n, dev, eight):
    if t is not None:
        if not eight:
            raise ValueError(f"{name} goes with 8-bit values")
        _need(t, name, torch.float32, (n,), dev)


class RmsNormResult(NamedTuple):
    out: torch.Tensor                  # [rows, d], the input's type or float8_e4m3fn
    scale: Optional[torch.Tensor]      # [rows] float32 with an 8-bit output
    residual: Optional[torch.Tensor]   # [rows, d], x + residual rounded


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, residual: Optional[torch.Tensor] = None,
             quantize: bool = False, out: Optional[torch.Tensor] = None, out_scale: Optional[torch.Tensor] = None,
             residual_out: Optional[torch.Tensor] = None, stream=None) -> RmsNormResult:
    """Root-mean-square norm of the rows of x (+ residual), times weight.

    quantize=True rounds to float8_e4m3fn with a scale per row (max / 448), the
    input that w4_matvec takes with x_scale.  residual_out may be residual
    itself (an update in place)."""
    if x.dim() != 2:
        raise ValueError("x must be [rows, d]")
    rows, d = x.shape
    dev, t = x.device, x.dtype
    if t not in _HALF and t != torch.float32:
        raise TypeError(f"x must be bfloat16, float16 or float32, got {t}")
    _need(x, "x", t, (rows, d), dev)
    _need(weight, "weight", t, (d,), dev)
    ot = E4M3 if quantize else t
    if out is None:
        out = torch.empty((rows, d), dtype=ot, device=dev)
    else:
        _need(out, "out", ot, (rows, d), dev)
    if residual is None:
        residual_out = None
    else:
        _need(residual, "residual", t, (rows, d), dev)
        if residual_out is None:
            residual_out = torch.empty((rows, d), dtype=t, device=dev)
        else:
            _need(residual_out, "residual_out", t, (rows, d), dev)
    if not quantize:
        out_scale = None
    elif out_scale is None:
        out_scale = torch.empty(rows, dtype=torch.float32, device=dev)
    else:
        _need(out_scale, "out_scale", torch.float32, (rows,), dev)
    _check(library().coverprune_rms_norm(_at(x), _CODE[t], rows, d, _at(residual), _at(weight), eps, _at(out), _CODE[ot],
                                         _at(out_scale), _at(residual_out), _on(stream, dev)))
    return RmsNormResult(out, out_scale, residual_out)


def w4_matvec(x: torch.Tensor, weight: torch.Tensor, scale: torch.Tensor, zero: Optional[torch.Tensor] = None,
              x_scale: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
              out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x [m, k] times 4-bit weights [n, k]: y[i, o] = sum_j x[i, j] (code[o, j] - zero) scale.

    weight: [n, k / 2] uint8, two codes a byte, the even j in the low half;
    scale: [n, k / group] bfloat16 or float16; zero: [n, k / group] uint8 codes
    (8 without).  x has scale's type, or is float8_e4m3fn with x_scale [m].
    out_dtype: scale's type (default) or float32."""
    if x.dim() != 2 or weight.dim() != 2 or scale.dim() != 2:
        raise ValueError("x, weight and scale must be matrices")
    m, k = x.shape
    n, groups = scale.shape
    dev, t = x.device, scale.dtype
    if t not in _HALF:
        raise TypeError(f"scale must be bfloat16 or float16, got {t}")
    if x.dtype != t and x.dtype != E4M3:
        raise TypeError(f"x must be {t} or {E4M3}, got {x.dtype}")
    if groups < 1 or k % groups != 0:
        raise ValueError(f"scale has {groups} groups for k = {k}")
    _need(x, "x", x.dtype, (m, k), dev)
    _need(weight, "weight", torch.uint8, (n, k // 2), dev)
    _need(scale, "scale", t, (n, groups), dev)
    if zero is not None:
        _need(zero, "zero", torch.uint8, (n, groups), dev)
    if (x_scale is not None) != (x.dtype == E4M3):
        raise ValueError("x_scale goes with an 8-bit x, and only with it")
    if x_scale is not None:
        _need(x_scale, "x_scale", torch.float32, (m,), dev)
    yt = t if out_dtype is None else out_dtype
    if yt != t and yt != torch.float32:
        raise TypeError(f"out_dtype must be {t} or float32, got {yt}")
    if out is None:
        out = torch.empty((m, n), dtype=yt, device=dev)
    else:
        _need(out, "out", yt, (m, n), dev)
    _check(library().coverprune_w4_matvec(_at(x), _CODE[x.dtype], _at(x_scale), _at(weight), _at(scale), _at(zero), m, n, k,
                                          k // groups, _CODE[t], _at(out), _CODE[yt], _on(stream, dev)))
    return out


def _heads(x, name, t, tokens, d, dev):
    """A [tokens, heads, d] view whose heads are contiguous; returns its head count and token stride."""
    if x.dim() != 3 or x.shape[0] != tokens or x.shape[2] != d:
        raise ValueError(f"{name} must be [{tokens}, heads, {d}], got {tuple(x.shape)}")
    if x.dtype != t:
        raise TypeError(f"{name} must be {t}, got {x.dtype}")
    if x.device != dev:
        raise ValueError(f"{name} must be on {dev}, got {x.device}")
    heads = x.shape[1]
    stride, head_stride, one = x.stride()
    if (one != 1 and d > 1) or (head_stride != d and heads > 1):
        raise ValueError(f"{name}: a token's heads must be contiguous")
    if tokens < 2:
        stride = heads * d
    elif stride < heads * d:
        raise ValueError(f"{name}: tokens overlap")
    return heads, stride


def _caches(k_cache, v_cache, t, hk, d, dev, k_scale, v_scale):
    if k_cache.dim() != 4:
        raise ValueError("the caches must be [pages, heads, page_size, d]")
    pages, _, page, _ = k_cache.shape
    c = k_cache.dtype
    if c != t and c != E4M3:
        raise TypeError(f"the caches must be {t} or {E4M3}, got {c}")
    _need(k_cache, "k_cache", c, (pages, hk, page, d), dev)
    _need(v_cache, "v_cache", c, (pages, hk, page, d), dev)
    _scales(k_scale, "k_scale", hk, dev, c == E4M3)
    _scales(v_scale, "v_scale", hk, dev, c == E4M3)
    return c, pages, page


def kv_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor,
              inv_freq: Optional[torch.Tensor], k_cache: torch.Tensor, v_cache: torch.Tensor, interleaved: bool = False,
              magnitude: float = 1.0, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
              q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """Rotate queries and keys by their positions and put keys and values into
    the paged caches; returns the rotated queries (None without q).

    q, k, v: [tokens, heads, d] bfloat16 or float16, possibly views of one
    projection's output; positions [tokens] int32 (a kept token keeps the one
    it had before the prune); slots [tokens] int64, page * page_size + offset
    (negative: not stored); inv_freq [rot / 2] float32, rot <= d elements of
    each head are rotated (None: none); caches [pages, heads, page_size, d] of
    k's type, or float8_e4m3fn holding value / k_scale[head], v_scale[head]."""
    t = k.dtype
    if t not in _HALF:
        raise TypeError(f"k must be bfloat16 or float16, got {t}")
    if k.dim() != 3:
        raise ValueError("k must be [tokens, heads, d]")
    tokens, hk, d = k.shape
    dev = k.device
    _, ks = _heads(k, "k", t, tokens, d, dev)
    hv, vs = _heads(v, "v", t, tokens, d, dev)
    if hv != hk:
        raise ValueError(f"v has {hv} heads, k has {hk}")
    hq, qs = 0, 0
    if q is not None:
        hq, qs = _heads(q, "q", t, tokens, d, dev)
        if q_out is None:
            q_out = torch.empty((tokens, hq, d), dtype=t, device=dev)
        else:
            _need(q_out, "q_out", t, (tokens, hq, d), dev)
    else:
        q_out = None
    _need(positions, "positions", torch.int32, (tokens,), dev)
    _need(slots, "slots", torch.int64, (tokens,), dev)
    half = 0
    if inv_freq is not None:
        half = inv_freq.shape[0] if inv_freq.dim() == 1 else -1
        _need(inv_freq, "inv_freq", torch.float32, (half,), dev)
    c, pages, page = _caches(k_cache, v_cache, t, hk, d, dev, k_scale, v_scale)
    _check(library().coverprune_kv_append(_at(q), qs, _at(k), ks, _at(v), vs, _CODE[t], tokens, hq, hk, d, _at(positions),
                                          _at(slots), _at(inv_freq), 2 * half, bool(interleaved), magnitude, _at(q_out),
                                          _at(k_cache), _at(v_cache), _CODE[c], pages, page, _at(k_scale), _at(v_scale),
                                          _on(stream, dev)))
    return q_out


def paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor,
                    lengths: torch.Tensor, max_length: Optional[int] = None, window: int = 0,
                    scale: Optional[float] = None, k_scale: Optional[torch.Tensor] = None,
                    v_scale: Optional[torch.Tensor] = None, return_lse: bool = False, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of one new token of each sequence over its paged keys and
    values; returns out [batch, heads, d], or (out, lse) with return_lse.

    q [batch, heads, d]; caches as kv_append fills them; table [batch, width]
    int32 pages of each sequence in order; lengths [batch] int32, the new token
    included (0: the result is 0).  max_length is the longest length, known to
    the host (default: all that the table can hold, which cuts short sequences
    into more pieces than they need).  window > 0: only the last `window`
    tokens.  scale defaults to 1 / sqrt(d)."""
    t = q.dtype
    if t not in _HALF:
        raise TypeError(f"q must be bfloat16 or float16, got {t}")
    if q.dim() != 3 or table.dim() != 2 or k_cache.dim() != 4:
        raise ValueError("q must be [batch, heads, d], table [batch, width], the caches [pages, heads, page_size, d]")
    batch, hq, d = q.shape
    dev, hk, width = q.device, k_cache.shape[1], table.shape[1]
    _need(q, "q", t, (batch, hq, d), dev)
    c, pages, page = _caches(k_cache, v_cache, t, hk, d, dev, k_scale, v_scale)
    _need(table, "table", torch.int32, (batch, width), dev)
    _need(lengths, "lengths", torch.int32, (batch,), dev)
    if out is None:
        out = torch.empty((batch, hq, d), dtype=t, device=dev)
    else:
        _need(out, "out", t, (batch, hq, d), dev)
    if lse is not None:
        _need(lse, "lse", torch.float32, (batch, hq), dev)
    elif return_lse:
        lse = torch.empty((batch, hq), dtype=torch.float32, device=dev)
    if max_length is None:
        max_length = width * page
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    lib = library()
    if workspace is None:
        need = lib.coverprune_paged_attention_workspace(batch, hq, hk, d, max_length, window)
        if need:
            workspace = _workspace(need, dev)
    _check(lib.coverprune_paged_attention(_at(q), _CODE[t], batch, hq, hk, d, _at(k_cache), _at(v_cache), _CODE[c], pages, page,
                                          _at(k_scale), _at(v_scale), _at(table), width, _at(lengths), max_length, window,
                                          scale, _at(out), _at(lse), _at(workspace),
                                          0 if workspace is None else workspace.numel(), _on(stream, dev)))
    return (out, lse) if return_lse else out
