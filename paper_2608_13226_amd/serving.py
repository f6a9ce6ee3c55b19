"""Operators of the language model's serving layer, which reads the kept
tokens: norm, 4-bit products, append to a paged cache, attention over it.

As in the rest of the binding, the functions only check and marshal torch
tensors; here that part is compiled (csrc/binding.cpp), because a decode step
is a handful of calls of a few microseconds each.  Each takes tensors of the
current GPU, enqueues on torch's current stream (or ``stream``) and returns
without waiting; outputs that are not given are allocated.  8-bit tensors are
torch.float8_e4m3fn throughout.  Wrong types raise TypeError, wrong shapes,
strides and devices ValueError, what the library itself refuses
CoverPruneError.  There are no backward passes: tensors that require a gradient
raise ValueError, except under torch.no_grad().
"""
from __future__ import annotations

import os
from typing import NamedTuple, Optional

import torch

from . import HERE, CoverPruneError, library

__all__ = ["rms_norm", "RmsNormResult", "w4_matvec", "kv_append", "paged_attention"]


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
