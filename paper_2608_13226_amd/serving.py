"""Operators of the language model's serving layer, which reads the kept
tokens: norm, 4-bit products, append to a paged cache, attention over it; and
those that keep the cache small: 4 bits, the tokens' accumulated weights, eviction.

As in the rest of the binding, the functions only check and marshal torch
tensors; here that part is compiled (csrc/binding.cpp), because a decode step
is a handful of calls of a few microseconds each.  Each takes tensors of the
current GPU, enqueues on torch's current stream (or ``stream``) and returns
without waiting; outputs that are not given are allocated.  8-bit tensors are
torch.float8_e4m3fn throughout, 4-bit caches uint8 (two codes a byte) with
uint8 exponents of 32 dims each.  Wrong types raise TypeError, wrong shapes,
strides and devices ValueError, what the library itself refuses
CoverPruneError.  There are no backward passes: tensors that require a gradient
raise ValueError, except under torch.no_grad().
"""
from __future__ import annotations

import os
from typing import NamedTuple, Optional

import torch

from . import HERE, CoverPruneError, library

__all__ = ["rms_norm", "RmsNormResult", "w4_matvec", "kv_append", "paged_attention", "kv_append4", "kv_gather",
           "paged_attention4", "paged_attention_mass", "kv_evict", "KvEvictResult"]


class _Unloaded:
    """Stands for the compiled half until the first call, which loads it."""

    def __getattr__(self, name):
        global _native
        library()
        if not os.path.exists(os.path.join(HERE, "_serving.so")):
            raise CoverPruneError(f"{os.path.join(HERE, '_serving.so')} is missing: build it with "
                                  f"`python -m paper_2608_13226_amd.build`")
        from . import _serving
        _serving.init(CoverPruneError, _raw_stream, _device)
        _native = _serving
        return getattr(_serving, name)


def _any_raw_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# torch's own functions for the handle of a device's current stream and for the
# current device, where it has them: a fifth of the time of making a Stream object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _any_raw_stream)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_native = _Unloaded()


class RmsNormResult(NamedTuple):
    out: torch.Tensor                  # [rows, d], the input's type or float8_e4m3fn
    scale: Optional[torch.Tensor]      # [rows] float32 with an 8-bit output
    residual: Optional[torch.Tensor]   # [rows, d], x + residual rounded


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, residual: Optional[torch.Tensor] = None,
             quantize: bool = False, out: Optional[torch.Tensor] = None, out_scale: Optional[torch.Tensor] = None,
             residual_out: Optional[torch.Tensor] = None, stream=None) -> RmsNormResult:
    """Root-mean-square norm of the rows of x (+ residual), times weight.

    x, residual [rows, d] and weight [d] are bfloat16, float16 or float32.
    quantize=True rounds to float8_e4m3fn with a scale per row (max / 448), the
    input that w4_matvec takes with x_scale.  residual_out may be residual
    itself (an update in place)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return rms_norm(x, weight, eps, residual, quantize, out, out_scale, residual_out)
    return RmsNormResult._make(_native.rms_norm(x, weight, eps, residual, quantize, out, out_scale, residual_out))


def w4_matvec(x: torch.Tensor, weight: torch.Tensor, scale: torch.Tensor, zero: Optional[torch.Tensor] = None,
              x_scale: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
              out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x [m, k] times 4-bit weights [n, k]: y[i, o] = sum_j x[i, j] (code[o, j] - zero) scale.

    weight: [n, k / 2] uint8, two codes a byte, the even j in the low half;
    scale: [n, k / group] bfloat16 or float16, groups of a multiple of 32;
    zero: [n, k / group] uint8 codes (8 without).  x has scale's type, or is
    float8_e4m3fn with x_scale [m] float32.  out_dtype: scale's type (default)
    or float32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return w4_matvec(x, weight, scale, zero, x_scale, out_dtype, out)
    return _native.w4_matvec(x, weight, scale, zero, x_scale, out_dtype, out)


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
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_append(q, k, v, positions, slots, inv_freq, k_cache, v_cache, interleaved, magnitude, k_scale, v_scale, q_out)
    return _native.kv_append(q, k, v, positions, slots, inv_freq, k_cache, v_cache, interleaved, magnitude, k_scale, v_scale, q_out)


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
    if stream is not None:
        with torch.cuda.stream(stream):
            return paged_attention(q, k_cache, v_cache, table, lengths, max_length, window, scale, k_scale, v_scale, return_lse,
                                   out, lse, workspace)
    return _native.paged_attention(q, k_cache, v_cache, table, lengths, max_length, window, scale, k_scale, v_scale, return_lse,
                                   out, lse, workspace)


def kv_append4(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor,
               inv_freq: Optional[torch.Tensor], k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor,
               v_scale: torch.Tensor, interleaved: bool = False, magnitude: float = 1.0, q_out: Optional[torch.Tensor] = None,
               stream=None) -> Optional[torch.Tensor]:
    """kv_append to a cache of 4 bits; returns the rotated queries (None without q).

    Arguments as for kv_append, but the caches are uint8 [pages, heads,
    page_size, d / 2], two codes a byte, with exponents k_scale and v_scale, uint8
    [pages, heads, page_size, d / 32]; d is a multiple of 32.  Each 32 dims share a
    power of two, the smallest that six times reaches their largest; codes are
    0, .5, 1, 1.5, 2, 3, 4, 6 times it and a sign, to nearest."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_append4(q, k, v, positions, slots, inv_freq, k_cache, v_cache, k_scale, v_scale, interleaved, magnitude, q_out)
    return _native.kv_append4(q, k, v, positions, slots, inv_freq, k_cache, v_cache, k_scale, v_scale, interleaved, magnitude, q_out)


def kv_gather(k_cache: torch.Tensor, v_cache: torch.Tensor, slots: torch.Tensor, dtype: Optional[torch.dtype] = None,
              k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
              k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None, stream=None):
    """Cached keys and values as dense rows: returns (k, v), [tokens, heads, d] each.

    Caches and scales as kv_append and kv_append4 take them; slots [tokens] int64
    (negative, or past the caches: zeros).  dtype: the caches' own type, and for 8
    and 4 bits bfloat16 (default) or float16."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_gather(k_cache, v_cache, slots, dtype, k_scale, v_scale, k_out, v_out)
    return _native.kv_gather(k_cache, v_cache, slots, dtype, k_scale, v_scale, k_out, v_out)


def paged_attention4(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                     table: torch.Tensor, lengths: torch.Tensor, max_length: Optional[int] = None, window: int = 0,
                     scale: Optional[float] = None, return_lse: bool = False, out: Optional[torch.Tensor] = None,
                     lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """paged_attention over a cache of 4 bits, as kv_append4 fills it (caches
    [pages, heads, page_size, d / 2] and scales [pages, heads, page_size, d / 32], uint8)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return paged_attention4(q, k_cache, v_cache, k_scale, v_scale, table, lengths, max_length, window, scale, return_lse,
                                    out, lse, workspace)
    return _native.paged_attention4(q, k_cache, v_cache, k_scale, v_scale, table, lengths, max_length, window, scale, return_lse,
                                    out, lse, workspace)


def paged_attention_mass(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor,
                         lengths: torch.Tensor, mass: torch.Tensor, max_length: Optional[int] = None, window: int = 0,
                         scale: Optional[float] = None, k_scale: Optional[torch.Tensor] = None,
                         v_scale: Optional[torch.Tensor] = None, return_lse: bool = False, out: Optional[torch.Tensor] = None,
                         lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention over a cache of any type that also adds to each cached token's
    mass the weight that it got; returns out, or (out, lse) with return_lse.

    mass [batch, kv_heads, span] float32, span at least max_length, is updated in
    place: mass[b, h, j] += sum over the query heads of h of softmax_j.  The
    other arguments as for paged_attention; uint8 caches are 4-bit ones, their
    scales the exponents.  max_length defaults to all that the table can hold, or
    span where that is less."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return paged_attention_mass(q, k_cache, v_cache, table, lengths, mass, max_length, window, scale, k_scale, v_scale,
                                        return_lse, out, lse, workspace)
    return _native.paged_attention_mass(q, k_cache, v_cache, table, lengths, mass, max_length, window, scale, k_scale, v_scale,
                                        return_lse, out, lse, workspace)


class KvEvictResult(NamedTuple):
    kept: torch.Tensor                 # [batch, kv_heads, keep] int32, the token now at each place; -1 past the new length
    lengths: torch.Tensor              # [batch] int32, at most keep
    mass: torch.Tensor                 # [batch, kv_heads, span] float32 in the new order, 0 past the new length


def kv_evict(k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, mass: torch.Tensor,
             keep: int, recent: int = 0, sink: int = 0, max_length: Optional[int] = None, k_scale: Optional[torch.Tensor] = None,
             v_scale: Optional[torch.Tensor] = None, kept: Optional[torch.Tensor] = None,
             mass_out: Optional[torch.Tensor] = None, lengths_out: Optional[torch.Tensor] = None,
             workspace: Optional[torch.Tensor] = None, stream=None) -> KvEvictResult:
    """Leave `keep` tokens of each sequence and head in the cache: the first
    `sink`, the last `recent`, and of the others those of largest mass (as
    paged_attention_mass adds it up).

    The caches (and the exponents k_scale and v_scale of 4-bit ones) are updated
    in place: kept tokens from place keep - recent on fill the places that fall vacant
    before it, then the last `recent` follow in order.  A sequence's pages must be its
    own.  mass_out may be mass itself; lengths_out may not be lengths.  Attention with a
    window no longer goes by age afterwards."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_evict(k_cache, v_cache, table, lengths, mass, keep, recent, sink, max_length, k_scale, v_scale, kept, mass_out,
                            lengths_out, workspace)
    return KvEvictResult._make(_native.kv_evict(k_cache, v_cache, table, lengths, mass, keep, recent, sink, max_length, k_scale,
                                                v_scale, kept, mass_out, lengths_out, workspace))
